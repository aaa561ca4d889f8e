// ripple_paged_tree_attn for bf16 queries, on the 5th-generation tensor cores.
//
// A team of 7 warps (9 over 8-bit pages; two teams a CTA, one CTA an SM) has the 128 rows of a
// matrix product for up to 128 query rows of a KV head and takes its run's blocks of 64 keys:
// S = Q . K^T (128 x 64) into TMEM, softmax by a thread a row, P back into TMEM over S, O += P . V
// (128 x d) in TMEM. A draft of n tokens with G heads a KV head has n G query rows. With 32 of them
// or fewer the product's rows hold four copies, with 64 two, and every copy takes its share of a
// block's keys (the others' probabilities are 0), so that the four softmax warps share the work
// however few rows there are; the copies are joined when a group is done. The products' rows cost
// nothing that the cache's bytes do not: a block is 32 KB, 1400 cycles of an SM's share of HBM, and
// 512 of its tensor cores.
//
// Of a team, 4 warps: queries, softmax and outputs; one issues the MMAs; one fetches keys, one
// values (8-bit pages: two each): a block by TMA (a box a page, with the 128-byte swizzle that the
// MMAs read), or, where rows of it are missing or pages have fewer than 8, by 16-byte copies to the
// same places. Scores of the next block are on their way while a block's softmax runs; S and P of
// two blocks and O fill half of the TMEM. The teams share nothing: one's softmax runs while the
// other's blocks are on their way. (Two CTAs of one team each do not find a place on an SM at
// the same time, though registers, shared memory and TMEM have room.)
//
// A wait that runs out ends the call: its role and then the others leave, the softmax warps of a
// team together, each fetching warp once what it issued has landed.
//
// Measured, D 128, 8 KV heads: 48 sequences of up to 32768 rows, 2 to 12 tokens of 32 heads 163 us
// (1.01 GB, 91% of the copy rate; with one team a CTA and no copies of the query rows 285); 3 of
// about 31000 rows with 64 tokens of 64 heads 191 us (196 GFLOP, 1.03 PFLOP/s): there the chain
// scores - softmax - product of a block, two of them an SM, leaves the tensor pipe half idle (and
// 128 registers a thread are not enough: 180 bytes spilt); 8-bit pages, 32 sequences of up to 32768
// rows, 16 tokens 172 us (419 MB, 36%): bound by the fetching warps' instructions (of a block's 3500
// cycles their loads, scales and tables take 1250, the widening 950; 18 warps leave 96 registers a
// thread, 110 to 240 bytes spilt). One sequence of 900 rows and 4 tokens 14.4 us: the launch,
// lengths, table, queries, two blocks, the join of the copies and of the shares, one after the other.
//
// P in one bf16 part: the output is rounded to bf16 as well, and a probability's rounding
// (2^-8) enters the output as part of a mean. The sum is of the unrounded ones, in fp32.
//
// 8-bit pages come into a ring of their own, two blocks ahead, and two warps each for keys and
// values make them fp16 values: a code times its row's scale over a reference of the block's, the
// largest scale of its rows before the draft. That is exact for rows up to 2^kBelow below it and
// 2^kAbove above. Rows beyond (hardly ever there) are left for further passes over the block, with
// references in steps of that, and count for nothing in this one. So no row takes anything from
// another, whatever a hidden one holds, or one without weight. The keys' reference multiplies the
// scores; the values' counts with the probability, 2^(x + e), relative to the largest such weight
// that the query row has seen, which is held as 2^7 to 2^15 in fp16: a weight loses 2^-32 of that
// one at most at the lower end (times 2^11 where their rows' scales are as far apart). The sum of
// the probabilities has the scores' own maximum, in fp32. A query row is multiplied by the power of
// two that brings its largest element to [2^14, 2^15).
// (Scales relative to the largest of any row of the block and, of values, so far: 161 us for the
// batch above, 172 now, but a hidden row could cost the others all their bits. Scales by rows in the
// softmax: 182 to 243, the block's scores then wait for them in a thread that has no registers left.)
#include "paged_tree.cuh"
#include "tc_ptx.cuh"

#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <float.h>

#include <atomic>

namespace ripple {
namespace {

constexpr int KB = kTreeTcKeys;
constexpr int kRows = kTreeTcRows;
// Warps 0-3, 4-7: softmax of the teams; 8, 9: their MMAs; from 10 on: keys and values of one team,
// then of the other, a warp each, two for 8-bit pages. (A warp reaches the TMEM lanes 32 (warp
// % 4) on.)
constexpr int kTeams = 2;
__host__ __device__ constexpr int threads(bool codes) { return 32 * (10 + kTeams * (codes ? 4 : 2)); }
// Blocks that a group's queries and outputs take as long as (their copies' join in the main). us for
// 2, 4, 7, 10, 14, D 128, 4 heads a KV head: 48 sequences of up to 32768 rows and 2 to 12 tokens
// 188, 164, 163.5, 165, 168; 8-bit pages, 32 sequences of 16 tokens 210, 185, 172, 176, 181.
constexpr int kGroupCost = 7;
constexpr int kRing = 2;       // blocks of 8-bit rows on their way or being widened
constexpr uint32_t kTeamCols = 256;  // of TMEM: S and P of two blocks (64 each), O (d) from 128 on
constexpr uint32_t kOCol = 128;
constexpr float kSlack = 8.f;
constexpr unsigned kAll = 0xffffffffu;
constexpr int kMaxDevices = 64;
constexpr int kDrafts = 4; // parts with drafted tokens that the values may be ahead
constexpr int kSlots = 8;  // of the rows that are there (known up to two blocks ahead)
constexpr int kScaled = 3; // of passes over 8-bit blocks (widened at most two ahead of the softmax)
// log2 of how far a row's scale may be from the reference to be put into fp16 values: codes reach
// from 2^-9 (of 4 bits) to 448, fp16 from 2^-24 to 65504.
constexpr int kBelow = 8, kAbove = 3, kWindow = kBelow + kAbove + 1;

// What the fetching warps tell one another and the softmax about blocks.
template <bool kCodes>
struct Told {
  uint64_t draft_done[kDrafts];        // by parts with drafted tokens (values may be parts ahead)
  unsigned long long bad[kDrafts];     // drafted tokens whose values are not all finite, by parts
  unsigned long long present[kSlots];  // rows of a block that are there
  // (among the softmax's warps) what the values of a part have in a quarter of the dims that is not
  // finite: 1: infinity, 2: -infinity, 4: NaN
  uint32_t not_finite[32];
};
template <>
struct Told<true> {
  uint16_t factor[2][kRing][KB];       // what the ring's keys, values are multiplied by, fp16
  bool more[2][kRing];                 // another pass over the same rows follows
  unsigned long long present[kScaled]; // rows that count in the pass
  unsigned long long nan[kScaled];     // those of them whose values are NaN
  float key[kScaled], value[kScaled];  // the references: the keys', log2 of the values'
  int again[kScaled];                  // 1: another pass over the same rows follows; 2: see nan
};
template <bool kCodes>
struct alignas(16) Sync {
  Told<kCodes> told;
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2];
  uint64_t ring_full[2][kRing];                         // of keys, of values
  uint64_t s_full[2], p_full[2], pv_done[2];            // of even and odd blocks
  uint64_t q_full, mma_done;
  uint32_t tmem;
  int abort;                           // a role has given up waiting
  float inv[64];                       // of a group's query rows (with copies), and where they go
  int out_row[64];
};

template <int D, bool kCodes>
struct Smem {
  static constexpr int SK = kCodes ? 1 : 2, SV = 2;  // stages of 16-bit blocks of keys, of values
  static constexpr int Q = kRows * D * 2, TILE = KB * D * 2;
  static constexpr int RAW = KB * D;             // a block of 8-bit rows
  static constexpr int HALF_Q = kRows * 128, HALF = KB * 128;  // of 64 dims
  static constexpr int K0 = Q, V0 = Q + SK * TILE, RING = V0 + SV * TILE;
  static constexpr int TEAM = RING + (kCodes ? 2 * kRing * RAW : 0);
  static constexpr int BYTES = kTeams * (TEAM + (int)sizeof(Sync<kCodes>));
  static_assert(TEAM % 1024 == 0 && BYTES <= 227 * 1024, "shared memory per CTA");
};

// The pools as TMA sees them: boxes of 64 dims (8-bit: a row) x rows of a page.
struct Maps {
  CUtensorMap k, v;
};
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap *map, int x, int y, int z,
                                            int w, uint64_t *bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"((uint64_t)map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar))
      : "memory");
}
// The thread's arrival on `bar` once its copies so far have landed.
__device__ __forceinline__ void copies_arrive(uint64_t *bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// Bounded wait: gives up after the bound, or when another role has. A poll suspends the thread
// for a quarter of the bound at most; not at all where that is little, since the least that the
// hardware suspends a thread for is then more.
__device__ __forceinline__ bool try_wait_for(uint64_t *bar, uint32_t parity, uint32_t ns) {
  uint32_t ok;
  if (ns < 1000) {
    asm volatile(
        "{\n .reg .pred p;\n"
        " mbarrier.test_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2;\n"
        " selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return ok != 0;
  }
  asm volatile(
      "{\n .reg .pred p;\n"
      " mbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2, %3;\n"
      " selp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity), "r"(ns)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool wait_bar(uint64_t *bar, int phase, const TreeParams &p, int *abort) {
  if (try_wait_for(bar, phase & 1, p.suspend_ns)) return true;
  const long long t0 = clock64();
  for (;;) {
    if (try_wait_for(bar, phase & 1, p.suspend_ns)) return true;
    if (*(volatile int *)abort) return false;
    if (clock64() - t0 > p.wait_cycles) {
      *(volatile int *)abort = 1;
      report(p.status, RIPPLE_ETIMEOUT);
      return false;
    }
  }
}

__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src),
               "r"(there ? 16 : 0)
               : "memory");
}
__device__ __forceinline__ void copies_landed() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ void st_shared16(uint32_t to, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(a), "r"(b), "r"(c), "r"(d)
               : "memory");
}
__device__ __forceinline__ uint4 ld_shared16(uint32_t at) {
  uint4 r;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
               : "r"(at)
               : "memory");
  return r;
}
// D[tmem] (+)= A[tmem] . B[smem], bf16, fp32 accumulation.
__device__ __forceinline__ void mma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc,
                                            uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, "
      "%11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, "
      "%28, %29, %30, %31, %32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
      "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
      "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
      "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, "
      "%11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
      : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, "
      "%11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
        "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_wait_st() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
// N columns of the thread's lane: 16, 32 or 64.
template <int N>
__device__ __forceinline__ void tmem_load(uint32_t at, uint32_t (&r)[N]) {
  if constexpr (N == 16)
    tmem_ld16(at, r);
  else
#pragma unroll
    for (int i = 0; i < N / 32; ++i) tmem_ld32(at + 32 * i, reinterpret_cast<uint32_t(&)[32]>(r[32 * i]));
  tmem_wait_ld();
}
template <int N>
__device__ __forceinline__ void tmem_store(uint32_t at, const uint32_t (&r)[N]) {
  if constexpr (N == 8)
    tmem_st8(at, r);
  else if constexpr (N == 16)
    tmem_st16(at, r);
  else
    tmem_st32(at, r);
}
// Two values as a pair of 16 bits, bf16 or (8-bit pages) fp16.
template <bool kHalf>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  if (kHalf) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
  }
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&h);
}
// Which of two bf16 values are infinite or NaN, as masks of their halves.
__device__ __forceinline__ uint32_t not_finite(uint32_t pair) {
  return ((pair & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) |
         ((pair & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}
constexpr uint16_t kNanFactor = 0x7fff;
// 16 codes times a factor as fp16.
__device__ __forceinline__ void widen(const uint4 &u, uint16_t factor, uint32_t (&o)[8]) {
  const __half2 scale = __half2half2(__ushort_as_half(factor));
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(
        (__nv_fp8x2_storage_t)(w[i / 2] >> (16 * (i & 1))), __NV_E4M3);
    const __half2 x = __hmul2(__half2(h), scale);
    o[i] = *reinterpret_cast<const uint32_t *>(&x);
  }
}
__device__ __forceinline__ float pow2(int e) {  // -126 <= e <= 127
  return __int_as_float((e + 127) << 23);
}

// kCodes: 8-bit pages. C: copies of the query rows.
template <int D, bool kCodes, int C>
__global__ void __launch_bounds__(threads(kCodes), 1)
    tree_tc_kernel(const __grid_constant__ TreeParams p, const __grid_constant__ Maps maps) {
  using S = Smem<D, kCodes>;
  using W = TreeWalk<KB, kGroupCost, 0>;
  constexpr int SK = S::SK, SV = S::SV;
  constexpr int RT = kRows / C;   // query rows of the tile
  constexpr int KC = KB / C;      // keys of a block that a copy takes
  extern __shared__ __align__(1024) uint8_t smem[];
  const int lane = threadIdx.x & 31, cta_warp = threadIdx.x >> 5;
  constexpr int kFetch = kCodes ? 4 : 2;  // warps of a team that fetch
  const int team = cta_warp < 8 ? cta_warp / 4 : cta_warp < 10 ? cta_warp - 8 : (cta_warp - 10) / kFetch;
  // 0-3: softmax, 4: MMAs, 5: keys, 6: values
  const int warp = cta_warp < 8    ? cta_warp % 4
                   : cta_warp < 10 ? 4
                                   : 5 + (cta_warp - 10) % kFetch / (kFetch / 2);
  const bool second = kCodes && cta_warp >= 10 && (cta_warp - 10) % 2 == 1;  // of two that fetch
  const int tid = 32 * warp + lane;
  uint8_t *const tiles = smem + team * S::TEAM;
  Sync<kCodes> *const syncs = (Sync<kCodes> *)(smem + kTeams * S::TEAM), *const sy = syncs + team;
  // (as many CTAs as SMs, or one for each team's work: teams beside one another in different CTAs)
  // Short caches: p.teams teams of a cluster (or one) have equal shares of a group.
  const int teams = p.teams;
  const int work = teams > 1 ? kTeams * (int)blockIdx.x + team : (int)(blockIdx.x + team * gridDim.x);
  const int run = teams > 0 ? work : work / p.tiles, tile = teams > 0 ? 0 : work % p.tiles;
  if (warp == 4 && lane == 0) {
    sy->abort = 0;
    for (int i = 0; i < kRing; ++i) {
      mbar_init(&sy->ring_full[0][i], 32);
      mbar_init(&sy->ring_full[1][i], 32);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sy->k_full[i], 16 * kFetch);
      mbar_init(&sy->v_full[i], 16 * kFetch);
      mbar_init(&sy->k_empty[i], 1);
      mbar_init(&sy->v_empty[i], 1);
      mbar_init(&sy->s_full[i], 1);
      mbar_init(&sy->p_full[i], 4);
      mbar_init(&sy->pv_done[i], 1);
    }
    mbar_init(&sy->q_full, 4);
    if constexpr (!kCodes)
      for (int i = 0; i < kDrafts; ++i) mbar_init(&sy->told.draft_done[i], 32);
    mbar_init(&sy->mma_done, 1);
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  if (cta_warp == 8) {
    tmem_alloc(&syncs->tmem, kTeams * kTeamCols);
    tmem_relinquish();
  }
  pdl_wait();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = syncs->tmem + team * kTeamCols;
  if (blockIdx.x == 0)
    for (int b = threadIdx.x; b < p.g.B; b += threads(kCodes)) TreeSeq::check(p, b);

  const uint32_t qs = smem_u32(tiles), ks = qs + S::K0, vs = qs + S::V0;
  W w;
  const bool any = teams > 0 ? w.share(p, work / teams, work % teams, teams) : w.start(p, run, lane);
  int n = 0;  // blocks of this CTA so far
  bool ok = true;
  auto wait_for = [&](uint64_t *bar, int phase) {  // by a whole warp
    return __all_sync(kAll, wait_bar(bar, phase, p, &sy->abort));
  };

  if (warp >= 5) {
    // -------------------------------------------------- keys, values
    const bool keys = warp == 5;
    const int ST = keys ? SK : SV;
    uint64_t *const full = keys ? sy->k_full : sy->v_full, *const empty = keys ? sy->k_empty : sy->v_empty;
    const uint32_t stages = keys ? ks : vs;
    const uint8_t *const pool = (const uint8_t *)(keys ? p.k_pages : p.v_pages);
    const CUtensorMap *const map = keys ? &maps.k : &maps.v;
    constexpr int kElem = kCodes ? 1 : 2;
    constexpr int kPieces = D * kElem / 16;     // of a row in its page
    constexpr int kRowsWarp = 32 / kPieces;     // rows of a copy of the warp
    constexpr int kSteps = KB / kRowsWarp;
    const int sub = lane / kPieces, pc = lane % kPieces;
    const int page_rows = 1 << p.g.shift, box = min(page_rows, KB);
    // entries of the block table for the rows lane and lane + 32 of the next block
    int entry[2];
    auto look_up = [&](int row0) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int row = row0 + lane + 32 * i;
        entry[i] = -1;
        if (row < w.end)
          entry[i] = p.table[guard((long long)w.b * p.g.max_pages + (row >> p.g.shift), 1,
                                   (long long)p.g.B * p.g.max_pages, p.status)];
      }
    };
    // The block at row0 on its way to `to`: by TMA where all its rows are there (and `allowed`);
    // returns whether so. Then `bar` has this thread's arrival and gets the bytes; otherwise the
    // thread's copies have been issued.
    unsigned long long present;
    auto fetch = [&](int row0, uint32_t to, uint64_t *bar, bool allowed) {
      bool there[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        there[i] = (unsigned)entry[i] < (unsigned)p.g.n_pages;
        if (!there[i] && row0 + lane + 32 * i < w.end) report(p.status, RIPPLE_EBOUNDS);
      }
      const uint32_t lo = __ballot_sync(kAll, there[0]), hi = __ballot_sync(kAll, there[1]);
      present = (unsigned long long)hi << 32 | lo;
      if constexpr (!kCodes)
        if (keys && lane == 0) sy->told.present[n % kSlots] = present;
      __syncwarp();
      if (allowed && p.tma && present == ~0ull) {
        if (lane == 0) mbar_arrive_expect_tx(bar, KB * D * kElem);
        __syncwarp();
        // a lane a page: the entry of its first row
        const int boxes = KB / box, first = lane * box;
        const int e0 = __shfl_sync(kAll, entry[0], first & 31);
        const int e1 = __shfl_sync(kAll, entry[1], first & 31);
        if (lane < boxes) {
          const int page = first < 32 ? e0 : e1, slot = (row0 + first) & (page_rows - 1);
          if constexpr (kCodes) {
            tma_load_4d(to + first * D, map, 0, slot, w.h, page, bar);
          } else {
#pragma unroll
            for (int half = 0; half < D / 64; ++half)
              tma_load_4d(to + half * S::HALF + first * 128, map, 64 * half, slot, w.h, page, bar);
          }
        }
        __syncwarp();
        if (lane != 0) mbar_arrive(bar);
        return true;
      }
      long long place[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int row = row0 + lane + 32 * i;
        place[i] = there[i] ? (entry[i] * p.g.page_stride + w.h * p.g.head_stride +
                               (row & (page_rows - 1)) * p.g.row_stride) * kElem
                            : -1;
      }
#pragma unroll 8
      for (int i = 0; i < kSteps; ++i) {
        const int row = i * kRowsWarp + sub;
        const long long at = __shfl_sync(kAll, i * kRowsWarp < 32 ? place[0] : place[1], row & 31);
        copy16(kCodes ? to + row * D + 16 * pc
                      : to + (pc >> 3) * S::HALF + row * 128 + (((pc & 7) ^ (row & 7)) << 4),
               pool + (at >= 0 ? at + 16 * pc : 0), at >= 0);
      }
      return false;
    };
    // Values of drafted tokens that are not finite are left out of the products (a hidden one's
    // weight is 0, and 0 times them is NaN) and added to the outputs of the rows that see them: who
    // they are is told with the part's last block.
    int drafts = 0;  // parts with drafted tokens
    unsigned long long bad = 0;
    // (8-bit pages have their own way: Told<true>::nan)
    auto tell_bad = [&]() {
      if constexpr (!kCodes) {
        const uint32_t lo = __reduce_or_sync(kAll, (uint32_t)bad);
        const uint32_t hi = __reduce_or_sync(kAll, (uint32_t)(bad >> 32));
        if (lane == 0) sy->told.bad[drafts % kDrafts] = (unsigned long long)hi << 32 | lo;
        bad = 0;
        mbar_arrive(&sy->told.draft_done[drafts % kDrafts]);
        ++drafts;
      }
    };
    int ring_n = 0, issued = 0;  // blocks that have gone through the ring, that were put there
    for (bool more = any; more && ok; more = w.next(p)) {
      const TreeSeq seq(p, w.b);
      if (seq.tokens * p.G - tile * RT <= 0 || w.count == 0) continue;
      look_up(w.begin);
      if constexpr (!kCodes) {
        for (int row0 = w.begin; row0 < w.end; row0 += KB, ++n) {
          const int stage = n % ST;
          if (n >= ST && !(ok = wait_for(&empty[stage], n / ST - 1))) break;
          const bool draft = !keys && w.end > seq.prefix && row0 + KB > seq.prefix;
          const uint32_t to = stages + stage * S::TILE;
          const bool by_tma = fetch(row0, to, &full[stage], !draft);
          if (row0 + KB < w.end) look_up(row0 + KB);
          if (by_tma) continue;
          copies_landed();
          if (draft) {
            const int first = (int)max(0LL, seq.prefix - row0);  // row of the block
#pragma unroll 4
            for (int i = first / kRowsWarp; i < kSteps; ++i) {
              const int row = i * kRowsWarp + sub;
              const uint32_t at = to + (pc >> 3) * S::HALF + row * 128 + (((pc & 7) ^ (row & 7)) << 4);
              const uint4 u = ld_shared16(at);
              const uint32_t b[4] = {not_finite(u.x), not_finite(u.y), not_finite(u.z), not_finite(u.w)};
              if (row >= first && (b[0] | b[1] | b[2] | b[3]) != 0) {
                st_shared16(at, u.x & ~b[0], u.y & ~b[1], u.z & ~b[2], u.w & ~b[3]);
                bad |= 1ull << (row0 + row - seq.prefix & 63);
              }
            }
            if (row0 + KB >= w.end) tell_bad();
          }
          fence_proxy_async_smem();  // for the tensor cores' reads
          mbar_arrive(&full[stage]);
        }
      } else {
        uint64_t *const ring_full = sy->ring_full[keys ? 0 : 1];
        const uint32_t ring = qs + S::RING + (keys ? 0 : kRing * S::RAW);
        // What both warps agree on: they go on to a block, or neither does.
        const int pair_bar = 3 + 2 * team + (keys ? 0 : 1);
        auto both = [&](bool mine) {
          int all;
          asm volatile(
              "{\n .reg .pred p, q;\n setp.ne.b32 q, %1, 0;\n"
              " barrier.cta.red.and.pred p, %2, 64, q;\n selp.s32 %0, 1, 0, p;\n}\n"
              : "=r"(all)
              : "r"((int)mine), "r"(pair_bar)
              : "memory");
          return all != 0;
        };
        // The first warp fetches blocks into the ring, block i of it being n + i - ring_n of the team.
        auto issue = [&](int row0, int i) {
          const int slot = i % kRing;
          issued = i + 1;
          if (!fetch(row0, ring + slot * S::RAW, &ring_full[slot], true)) copies_arrive(&ring_full[slot]);
          if (row0 + KB < w.end) look_up(row0 + KB);
        };
        // The second brings the scales of keys and values, bytes of the rows lane and lane + 32,
        // loaded a block before they are put beside the ring (and not looked at until then: what
        // does waits for them, 243 us for the batch above).
        int coming[2][2] = {{0, 0}, {0, 0}}, there = 0;  // which of the two rows are in the cache
        uint32_t bytes = 0;                     // of this block: keys from bit 0, values from 16 on
        int id[2] = {0, 0};                     // the pass that a row belongs to (0: none any more)
        int ref[2] = {127, 127}, now = 0;       // bytes of the first pass's references; this pass
        uint32_t rows[2] = {0, 0};              // of the pass
        bool several = false, follows = false;  // passes over the block; another after this one
        constexpr int kFirst = 32 << 8 | 32;    // windows up or down, and 32, of keys and values
        auto byte_of = [&](int kind, int k) { return (int)(bytes >> (16 * kind + 8 * k) & 0xffu); };
        auto load_scales = [&](int row0) {
          there = 0;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int page = entry[k], row = row0 + lane + 32 * k;
            if ((unsigned)page < (unsigned)p.g.n_pages) {
              const long long at =
                  page * p.scale_page + w.h * p.scale_head + (row & (page_rows - 1)) * p.scale_row;
              coming[0][k] = p.k_scales[at];
              coming[1][k] = p.v_scales[at];
              there |= 1 << k;
            }
          }
          if (row0 + KB < w.end) look_up(row0 + KB);
        };
        // Passes over the block at row0: rows by how many windows their scales lie from the
        // references. (Neither these nor the passes' order hang on drafted rows; NaN is of the
        // first.)
        auto sort_rows = [&](int row0) {
          bytes = coming[0][0] | coming[0][1] << 8 | coming[1][0] << 16 | coming[1][1] << 24;
          const int before = (int)(seq.prefix - row0) - lane;  // rows before the draft from the lane's on
#pragma unroll
          for (int kind = 0; kind < 2; ++kind) {
            int top = 0;
#pragma unroll
            for (int k = 0; k < 2; ++k)
              if (byte_of(kind, k) != 255 && before > 32 * k) top = max(top, byte_of(kind, k));
            top = __reduce_max_sync(kAll, top);
            ref[kind] = top > 0 ? top : 127;
          }
          bool apart = false;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            id[k] = there >> k & 1 ? kFirst : 0;
#pragma unroll
            for (int kind = 0; kind < 2; ++kind)
              apart |= id[k] != 0 &&
                       (unsigned)(byte_of(kind, k) - ref[kind] + kBelow) >= (unsigned)kWindow;
          }
          several = __any_sync(kAll, apart);
          if (several) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              int at[2];
#pragma unroll
              for (int kind = 0; kind < 2; ++kind) {
                const int byte = byte_of(kind, k);  // (32 windows are more than a byte has)
                at[kind] = byte == 255 ? 32 : (byte - ref[kind] + kBelow + 32 * kWindow) / kWindow;
              }
              if (id[k] != 0) id[k] = at[0] << 8 | at[1];
            }
          }
        };
        // The next pass, beside the ring's block i.
        auto put_scales = [&](int i) {
          if constexpr (kCodes) {
            now = kFirst;
            follows = false;
            if (several) {
              constexpr unsigned kNone = ~0u;
              const unsigned a = id[0] == 0 ? kNone : id[0], b = id[1] == 0 ? kNone : id[1];
              now = (int)__reduce_min_sync(kAll, min(a, b));
              follows = __any_sync(kAll, (id[0] != 0 && id[0] != now) ||
                                             (id[1] != 0 && id[1] != now));
            }
            const int kind = keys ? 0 : 1;
            const int centre = ref[kind] + ((keys ? now >> 8 : now & 0xff) - 32) * kWindow;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int byte = byte_of(kind, k);
              sy->told.factor[kind][i % kRing][lane + 32 * k] =
                  id[k] != now ? 0
                  : byte == 255  ? (keys ? kNanFactor : 0)
                                 : (15 + byte - centre) << 10;
              rows[k] = __ballot_sync(kAll, id[k] == now);
            }
            if (lane == 0) sy->told.more[kind][i % kRing] = follows;
          }
        };
        // What the softmax gets, once the pass three before it has been read.
        auto tell_scales = [&]() {
          if constexpr (kCodes) {
            const int slot = n % kScaled;
            const bool nan[2] = {id[0] == now && byte_of(1, 0) == 255,
                                 id[1] == now && byte_of(1, 1) == 255};
            const bool any_nan = __any_sync(kAll, nan[0] || nan[1]);
            if (any_nan) {
              const uint32_t lo = __ballot_sync(kAll, nan[0]), hi = __ballot_sync(kAll, nan[1]);
              if (lane == 0) sy->told.nan[slot] = (unsigned long long)hi << 32 | lo;
            }
            if (lane == 0) {
              const int key = ref[0] + ((now >> 8) - 32) * kWindow;
              sy->told.present[slot] = (unsigned long long)rows[1] << 32 | rows[0];
              sy->told.key[slot] = key >= 255 ? FLT_MAX : pow2(key - 127);
              sy->told.value[slot] = (float)(ref[1] + ((now & 0xff) - 32) * kWindow - 127);
              sy->told.again[slot] = (int)follows | (any_nan ? 2 : 0);
            }
          }
        };
        if (!second) {
          issue(w.begin, ring_n);
          if (w.begin + KB < w.end) issue(w.begin + KB, ring_n + 1);
        } else {
          load_scales(w.begin);
          sort_rows(w.begin);
          put_scales(ring_n);
          if (w.begin + KB < w.end) load_scales(w.begin + KB);
        }
        for (int row0 = w.begin; row0 < w.end; ++n) {
          const int slot = ring_n % kRing, stage = n % ST;
          ok = both(wait_for(&ring_full[slot], ring_n / kRing) &&
                    (n < ST || wait_for(&empty[stage], n / ST - 1)));
          if (!ok) break;
          bool more = false;
          if constexpr (kCodes) more = sy->told.more[keys ? 0 : 1][slot];
          if (keys && second) tell_scales();
          const uint32_t from = ring + slot * S::RAW, to = stages + stage * S::TILE;
          // the steps of one warp, kAt at a time: their loads together, then the rest
          constexpr int kMine = kSteps / 2, kAt = 4;
          static_assert(kMine % kAt == 0, "");
#pragma unroll 1
          for (int i0 = 0; i0 < kMine; i0 += kAt) {
            const int first = (second ? kMine : 0) + i0;
            uint4 u[kAt];
            uint16_t by[kAt];
#pragma unroll
            for (int i = 0; i < kAt; ++i) {
              const int row = (first + i) * kRowsWarp + sub;
              if constexpr (kCodes) by[i] = sy->told.factor[keys ? 0 : 1][slot][row];
              u[i] = ld_shared16(from + row * D + 16 * pc);
            }
#pragma unroll
            for (int i = 0; i < kAt; ++i) {
              const int row = (first + i) * kRowsWarp + sub;
              uint32_t o[8];
              widen(u[i], by[i], o);
              const int c = 2 * pc;  // of 16-byte pieces in the stage
              const uint32_t at = to + (c >> 3) * S::HALF + row * 128;
              st_shared16(at + (((c & 7) ^ (row & 7)) << 4), o[0], o[1], o[2], o[3]);
              st_shared16(at + ((((c & 7) + 1) ^ (row & 7)) << 4), o[4], o[5], o[6], o[7]);
            }
          }
          fence_proxy_async_smem();  // for the tensor cores' reads
          mbar_arrive(&full[stage]);
          named_bar_sync(pair_bar, 64);  // the ring's place has been read
          if (more) {
            if (second) {
#pragma unroll
              for (int k = 0; k < 2; ++k) id[k] = id[k] == now ? 0 : id[k];
              put_scales(ring_n);
            }
            continue;
          }
          if (!second) {
            if (row0 + 2 * KB < w.end) issue(row0 + 2 * KB, ring_n + 2);
          } else if (row0 + KB < w.end) {
            sort_rows(row0 + KB);
            put_scales(ring_n + 1);
            if (row0 + 2 * KB < w.end) load_scales(row0 + 2 * KB);
          }
          row0 += KB;
          ++ring_n;
        }
      }
    }
    copies_landed();
    // What TMA still has on its way lands before the CTA leaves: this warp may be done where
    // another role has given up on it.
    if (!kCodes) {
      for (int i = max(0, n - ST); i < n; ++i) mbar_wait(&full[i % ST], i / ST & 1, nullptr);
    } else if (!ok) {  // (else every block has been waited for; the second warp has issued none)
      for (int i = max(0, issued - kRing); i < issued; ++i)
        mbar_wait(&sy->ring_full[keys ? 0 : 1][i % kRing], i / kRing & 1, nullptr);
    }
  } else if (warp == 4) {
    // -------------------------------------------------- MMAs (the whole warp waits, one lane issues)
    constexpr uint32_t kType = kCodes ? ~((1u << 7) | (1u << 10)) : ~0u;  // fp16 in place of bf16
    constexpr uint32_t id_qk = idesc_bf16(kRows, KB) & kType;
    constexpr uint32_t id_pv = (idesc_bf16(kRows, D) & kType) | (1u << 16);  // V: d is the contiguous one
    const uint64_t qd = sw128_desc(qs);
    // scores of block i: S(i). The products P . V of the blocks up to n - 1 have been issued, and
    // all of them have to be done: P of block i - 2 lies where S(i) goes, and a barrier that has
    // gone on by two phases cannot be waited for.
    auto scores = [&](int i) {
      const int st = i % SK;
      if (!wait_for(&sy->k_full[st], i / SK)) return false;
      if (n > 0 && !wait_for(&sy->pv_done[(n - 1) & 1], (n - 1) / 2)) return false;
      tc_fence_after();
      if (elect_one()) {
        const uint64_t kd = sw128_desc(ks + st * S::TILE);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          const uint64_t step = (uint64_t)((kk & 3) * 32 >> 4);
          mma_bf16(tmem + (i & 1) * KB, qd + ((kk >> 2) * S::HALF_Q >> 4) + step,
                   kd + ((kk >> 2) * S::HALF >> 4) + step, id_qk, kk > 0);
        }
        mma_commit(&sy->k_empty[st]);
        mma_commit(&sy->s_full[i & 1]);
      }
      __syncwarp();
      return true;
    };
    // (8-bit pages: another pass over the rows of block n follows; known once its keys are there)
    auto again = [&]() {
      if constexpr (kCodes) return (sy->told.again[n % kScaled] & 1) != 0;
      else return false;
    };
    int part = 0;
    for (bool more = any; more && ok; more = w.next(p)) {
      const TreeSeq seq(p, w.b);
      if (seq.tokens * p.G - tile * RT <= 0 || w.count == 0) continue;
      const int count = w.count;
      if (!(ok = wait_for(&sy->q_full, part++))) break;
      ok = scores(n);
      bool begun = false;  // O has a block
      for (int i = 0; i < count && ok; ++n, begun = true) {
        if (!again()) ++i;
        if (i < count && !(ok = scores(n + 1))) break;
        const int st = n % SV;
        if (!wait_for(&sy->p_full[n & 1], n / 2) || !wait_for(&sy->v_full[st], n / SV)) {
          ok = false;
          break;
        }
        tc_fence_after();
        if (elect_one()) {
          const uint64_t vd = sw128_desc_mn(vs + st * S::TILE, S::HALF, 1024);
#pragma unroll
          for (int kk = 0; kk < KB / 16; ++kk)  // 16 keys: 8 columns of P, 2 KB of V
            mma_bf16_ts(tmem + kOCol, tmem + (n & 1) * KB + kk * 8, vd + (kk * 2048 >> 4), id_pv,
                        kk > 0 || begun);
          // (the copies are joined in the last block's stage)
          if (C == 1 || i < count) mma_commit(&sy->v_empty[st]);
          mma_commit(&sy->pv_done[n & 1]);
        }
        __syncwarp();
      }
    }
    if (elect_one()) mma_commit(&sy->mma_done);
    __syncwarp();
    mbar_wait(&sy->mma_done, 0, nullptr);
  } else {
    // ------------------------------------ queries, softmax and outputs, a thread a row of the products
    const uint32_t lanes = tmem + ((uint32_t)(32 * warp) << 16);
    int2 rec = make_int2(0, 0);
    const int copy = tid / RT, r = tid % RT;
    const int key0 = copy * KC;
    // The queries of the part at `w`, once the products with the ones before are done. The row's
    // products are multiplied by row_scale.
    float row_scale = 0.f;
    // A warp has 32 rows of the products, a row's 16-byte pieces on neighbouring lanes.
    auto fetch_queries = [&](const W &w, const TreeSeq &seq) {
      constexpr int kQPieces = D / 8, kAtOnce = 32 / kQPieces, kSteps = 32 / kAtOnce;
      const int n_rows = min(seq.tokens * p.G - tile * RT, RT);
      const int mine = tile * RT + (r < n_rows ? r : 0), tok = mine / p.G;
      const int head = w.h * p.G + mine - tok * p.G;
      // where the thread's own row lies (-1: it is none)
      const long long at = r < n_rows ? head * p.q_head + (p.starts == nullptr
                                                               ? w.b * p.q_seq + tok * p.q_token
                                                               : (long long)(seq.first + tok) * p.q_token)
                                      : -1;
      const int pc = lane % kQPieces, sub = lane / kQPieces;
      float scale = p.scale2;
      auto place = [&](int row) {  // of the piece of a row of the warp
        return qs + (pc >> 3) * S::HALF_Q + (32 * warp + row) * 128 + (((pc & 7) ^ (row & 7)) << 4);
      };
      if constexpr (!kCodes) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          const int row = i * kAtOnce + sub;
          const long long from = __shfl_sync(kAll, at, row);
          copy16(place(row), (const __nv_bfloat16 *)p.q + (from >= 0 ? from + 8 * pc : 0), from >= 0);
        }
        copies_landed();
      } else {
        constexpr int kAt = kSteps < 8 ? kSteps : 8;  // loaded at a time
        int up = 0;                                   // of the thread's own row
#pragma unroll 1
        for (int i0 = 0; i0 < kSteps; i0 += kAt) {
          uint4 x[kAt];
#pragma unroll
          for (int i = 0; i < kAt; ++i) {
            const long long from = __shfl_sync(kAll, at, (i0 + i) * kAtOnce + sub);
            x[i] = make_uint4(0, 0, 0, 0);
            if (from >= 0)
              x[i] = __ldg(reinterpret_cast<const uint4 *>((const __nv_bfloat16 *)p.q + from) + pc);
          }
#pragma unroll
          for (int i = 0; i < kAt; ++i) {
            const int row = (i0 + i) * kAtOnce + sub;
            const uint32_t u[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
            float most = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k)
              most = fmaxf(most, fmaxf(fabsf(__uint_as_float(u[k] << 16)),
                                       fabsf(__uint_as_float(u[k] & 0xffff0000u))));
#pragma unroll
            for (int o = 1; o < kQPieces; o <<= 1) most = fmaxf(most, __shfl_xor_sync(kAll, most, o));
            // (infinities keep the others finite; what is below 2^-86 may be lost)
            const int e = most == 0.f ? 0 : min(14 - ((__float_as_int(most) >> 23) - 127), 100);
            const float f = pow2(e);
            uint32_t o[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
              o[k] = pack16<true>(__uint_as_float(u[k] << 16) * f, __uint_as_float(u[k] & 0xffff0000u) * f);
            st_shared16(place(row), o[0], o[1], o[2], o[3]);
            const int of_row = __shfl_sync(kAll, e, lane % kAtOnce * kQPieces);
            if (lane / kAtOnce == i0 + i) up = of_row;
          }
        }
        scale *= pow2(-up);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sy->q_full);
      row_scale = scale;
    };
    // A barrier of the team's four warps, and whether all of their threads say so. (That none has given
    // up, before barriers that all of them have to reach.)
    auto all_say = [&](bool mine) {
      int all;
      asm volatile(
          "{\n .reg .pred p, q;\n setp.ne.b32 q, %1, 0;\n"
          " barrier.cta.red.and.pred p, %2, 128, q;\n selp.s32 %0, 1, 0, p;\n}\n"
          : "=r"(all)
          : "r"((int)mine), "r"(1 + team)
          : "memory");
      return all != 0;
    };
    bool have_queries = false;
    int drafts = 0;  // parts with drafted tokens
    for (bool more = any; more && ok; more = w.next(p)) {
      const TreeSeq seq(p, w.b);
      if (w.count == 0) continue;
      const bool here = w.block == 0, whole = w.whole();
      if (teams == 0 && here && !whole) rec = make_int2(w.b * p.g.Hkv + w.h, w.runs_of_group(run));
      const int n_rows = min(seq.tokens * p.G - tile * RT, RT);
      if (n_rows <= 0) continue;
      if (!have_queries) fetch_queries(w, seq);
      const bool live = r < n_rows, warp_live = 32 * warp % RT < n_rows;
      // query row r of the tile: token, output row
      auto token_of = [&](int i) { return (tile * RT + i) / p.G; };
      auto out_row = [&](int i) {
        return (long long)(seq.first + token_of(i)) * p.Hq + w.h * p.G + (tile * RT + i) % p.G;
      };
      uint64_t mask = 0;
      if (live) mask = p.masks == nullptr ? ~0ull >> (63 - token_of(r)) : p.masks[seq.first + token_of(r)];
      // adds what the values of the drafted tokens in `which` have that is not finite to the dims
      // from d0 on
      auto add_bad = [&](unsigned long long which, int d0, float *o, int dims) {
        for (unsigned long long left = which; left != 0; left &= left - 1) {
          const long long at_row = seq.prefix + __ffsll(left) - 1;
          const int page = p.table[guard((long long)w.b * p.g.max_pages + (at_row >> p.g.shift), 1,
                                         (long long)p.g.B * p.g.max_pages, p.status)];
          const int v_slot = (int)(at_row & ((1 << p.g.shift) - 1));
          const __nv_bfloat16 *v = (const __nv_bfloat16 *)p.v_pages + page * p.g.page_stride +
                                   w.h * p.g.head_stride + v_slot * p.g.row_stride + d0;
          for (int i = 0; i < dims; ++i) {
            const float x = __bfloat162float(v[i]);
            if (!(fabsf(x) < INFINITY)) o[i] += x;
          }
        }
      };
      // told.not_finite for the dims from d0 on, by the team's 128 threads: over the part's rows before
      // the draft, 16 bytes' quarter (four dims) of every 128 / pieces-th row a thread.
      auto find_not_finite = [&](int d0, int pieces) {
        if constexpr (!kCodes) {
          if (tid < 4 * pieces) sy->told.not_finite[tid] = 0;
          named_bar_sync(1 + team, 128);
          const int pc = tid % pieces, step = 128 / pieces;
          const int end = (int)min((long long)w.end, seq.prefix);
          uint32_t found[4] = {0, 0, 0, 0};
#pragma unroll 1
          for (int row = w.begin + tid / pieces; row < end; row += step) {
            const int page = p.table[guard((long long)w.b * p.g.max_pages + (row >> p.g.shift), 1,
                                           (long long)p.g.B * p.g.max_pages, p.status)];
            if ((unsigned)page >= (unsigned)p.g.n_pages) continue;
            const uint2 u = *reinterpret_cast<const uint2 *>(
                (const __nv_bfloat16 *)p.v_pages + page * p.g.page_stride + w.h * p.g.head_stride +
                (row & ((1 << p.g.shift) - 1)) * p.g.row_stride + d0 + 4 * pc);
            const uint32_t bits[4] = {u.x << 16, u.x & 0xffff0000u, u.y << 16, u.y & 0xffff0000u};
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if ((bits[i] & 0x7f800000u) == 0x7f800000u)
                found[i] |= (bits[i] & 0x7fffffu) != 0 ? 4 : bits[i] >> 31 ? 2 : 1;
          }
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (found[i] != 0) atomicOr(&sy->told.not_finite[4 * pc + i], found[i]);
          named_bar_sync(1 + team, 128);
        }
      };
      // Of four outputs of that quarter, from its dim d on, those that are NaN: the sum of what the
      // values have that is not finite; others stay.
      auto put_not_finite = [&](int d, float (&o)[4]) {
        if constexpr (!kCodes) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t has = sy->told.not_finite[d + i];
            if (o[i] != o[i] && (has == 1 || has == 2)) o[i] = has == 1 ? INFINITY : -INFINITY;
          }
        }
      };
      // m: what the probabilities are relative to, a maximum, in log2. ew (8-bit pages): of their
      // products with the values' scales, over m; the largest is held as 2^kTop or up to 2^kSlack more
      constexpr float kTop = 7.f;
      float m = -INFINITY, l = 0.f, ew = 0.f;
      bool begun = false;     // O has a block
      bool poisoned = false;  // 8-bit pages: a value that the row sees is NaN
      for (int row0 = w.begin; row0 < w.end && ok; ++n, begun = true) {
        if (!(ok = wait_for(&sy->s_full[n & 1], n / 2))) break;
        bool more = false;  // 8-bit pages: another pass over the same rows follows
        if (warp_live) {
          tc_fence_after();
          const uint32_t s_at = lanes + (n & 1) * KB;
          // (8-bit pages without copies: a thread has no room for 64 scores, and reads them again)
          constexpr int NH = kCodes && C == 1 ? 2 : 1, HK = KC / NH;
          uint32_t u[HK];
          const int slot = n % (kCodes ? kScaled : kSlots);
          const unsigned long long present = sy->told.present[slot];
          const bool masked = present != ~0ull || row0 + KB > seq.prefix;
          unsigned long long seen = ~0ull;
          if (masked) {
            // the draft's token j is the block's key j - j0
            const long long j0 = row0 - seq.prefix;
            seen = (present & (j0 <= -64 ? ~0ull
                               : j0 < 0  ? mask << -j0 | ((1ull << -j0) - 1)
                               : j0 < 64 ? mask >> j0
                                         : 0ull)) >> key0;
          }
          auto load_scores = [&](int half) {
            tmem_load<HK>(s_at + key0 + half * HK, u);
            if (masked) {
              const unsigned long long on = seen >> (half * HK);
#pragma unroll
              for (int i = 0; i < HK; ++i)
                if (!(on >> i & 1)) u[i] = 0xff800000u;  // -infinity
            }
          };
          // O of the blocks before times a, once they are in it; false: the wait ran out
          auto rescale = [&](bool grow, float a) {
            if (!__any_sync(kAll, grow) || !begun) return true;
            if (!wait_for(&sy->pv_done[(n - 1) & 1], (n - 1) / 2)) return false;
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
              uint32_t o[32];
              tmem_load<32>(lanes + kOCol + c, o);
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * a);
              tmem_store<32>(lanes + kOCol + c, o);
            }
            return true;
          };
          // 8-bit pages: both references, where the largest score or weight (`most`, log2, over the
          // maximum `over` so far) may be beyond what they allow; they move together
          bool grow = false;
          float a_o = 1.f;
          auto raise = [&](float mb, auto most) {
            float was = m == -INFINITY ? -INFINITY : ew;  // (none before the first score)
            float over = m == -INFINITY ? 0.f : m;
            if (mb > m + kSlack) {
              const float fall = m - mb;
              l *= fast_exp2(fall);
              was += fall;
              m = over = mb;
              grow = true;
            }
            const float y = most(over);
            if (grow || y > ew + kSlack) {
              // (above 2^-120, the least scale, so that the outputs' factor is an fp32 value)
              ew = fminf(fmaxf(ceilf(fmaxf(was, y)), -112.f), 128.f);
              a_o = fast_exp2(was - ew);
              grow = true;
            }
          };
          float key_scale = 1.f, value = 0.f;
          if constexpr (kCodes) {
            key_scale = sy->told.key[slot];
            value = sy->told.value[slot];
            if ((sy->told.again[slot] & 2) != 0)
              poisoned |= (seen & sy->told.nan[slot] >> key0 & (~0ull >> (64 - KC))) != 0;
          }
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int half = 0; half < NH; ++half) {
            load_scores(half);
#pragma unroll
            for (int i = 0; i < HK; ++i) mx[i & 3] = fmaxf(mx[i & 3], __uint_as_float(u[i]));
          }
          float mb = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
          float rs = row_scale;
          // (a positive number; scores have 2^-95 at most where fp32 has no smaller factor)
          if (kCodes) rs = fminf(fmaxf(rs * key_scale, FLT_MIN), FLT_MAX);
          mb *= rs;  // (> 0)
          if constexpr (!kCodes) {
            if (mb > m + kSlack) {
              a_o = fast_exp2(m - mb);
              m = mb;
              l *= a_o;
              grow = true;
            }
          } else {
            if (mb > m + kSlack || (mb - (m == -INFINITY ? 0.f : m)) + value > ew + kSlack)
              raise(mb, [&](float over) { return (mb - over) + value; });
          }
          if (!(ok = rescale(grow, a_o))) break;
          // scores of -infinity alone leave no finite maximum; the fused multiply-add, which leaves
          // out the score's rounding, must not meet a maximum whose own rounding counts
          // (8-bit pages: by threads, so that no row's scores hang on another's)
          const float sub = m == -INFINITY ? 0.f : m;
          float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
          const bool far = kCodes ? fabsf(sub) >= 65536.f : __any_sync(kAll, fabsf(sub) >= 65536.f);
          // 8-bit pages: the weights over the probabilities, log2. The sum is of the weights, brought
          // back, but where that is so much that either may be no fp32 value.
          const float up = kCodes ? value + (kTop - ew) : 0.f;
          const bool apart = kCodes && fabsf(up) > 90.f;
#pragma unroll
          for (int half = 0; half < NH; ++half) {
            if (NH > 1) load_scores(half);  // (P lies over scores that have been read)
            uint32_t pr[HK / 2];
            if (!far && !apart) {
#pragma unroll
              for (int i = 0; i < HK; i += 2) {
                float2 y = __ffma2_rn(make_float2(__uint_as_float(u[i]), __uint_as_float(u[i + 1])),
                                      make_float2(rs, rs), make_float2(up - sub, up - sub));
                y.x = fast_exp2(y.x);
                y.y = fast_exp2(y.y);
                sum[i / 2 & 1] = __fadd2_rn(sum[i / 2 & 1], y);
                pr[i / 2] = pack16<kCodes>(y.x, y.y);
              }
            } else {
#pragma unroll
              for (int i = 0; i < HK; i += 2) {
                // (rounded apart, as the maximum was: fused they may be far above it)
                const float2 y = make_float2(__fsub_rn(__fmul_rn(__uint_as_float(u[i]), rs), sub),
                                             __fsub_rn(__fmul_rn(__uint_as_float(u[i + 1]), rs), sub));
                float2 z = make_float2(fast_exp2(y.x), fast_exp2(y.y));
                sum[i / 2 & 1] = __fadd2_rn(sum[i / 2 & 1], z);
                if (kCodes) z = make_float2(fast_exp2(y.x + up), fast_exp2(y.y + up));
                pr[i / 2] = pack16<kCodes>(z.x, z.y);
              }
            }
            if (kCodes) __syncwarp();
            // the copy's own keys; the other copies' have no weight here
#pragma unroll
            for (int k = 0; k < C; ++k) {
              uint32_t of[HK / 2];
#pragma unroll
              for (int i = 0; i < HK / 2; ++i) of[i] = C == 1 || k == copy ? pr[i] : 0u;
              tmem_store<HK / 2>(s_at + (C == 1 ? half : k) * (HK / 2), of);
            }
          }
          const float all = (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
          l += kCodes && !far && !apart ? all * fast_exp2(-up) : all;
          tmem_wait_st();
          tc_fence_before();
        }
        if constexpr (kCodes) more = (sy->told.again[n % kScaled] & 1) != 0;
        if (!more) row0 += KB;
        __syncwarp();
        if (lane == 0) mbar_arrive(&sy->p_full[n & 1]);
      }
      // the next part's queries: its first scores are computed while this one's outputs are written
      if (ok) {
        W next = w;
        have_queries = false;
        if (next.next(p)) {
          const TreeSeq next_seq(p, next.b);
          if (next_seq.tokens * p.G - tile * RT > 0 && next.count > 0) {
            fetch_queries(next, next_seq);
            have_queries = true;
          }
        }
      }
      ok = ok && wait_for(&sy->pv_done[(n - 1) & 1], (n - 1) / 2);
      unsigned long long bad = 0;
      if constexpr (!kCodes) {
        if (ok && w.end > seq.prefix) {
          ok = wait_for(&sy->told.draft_done[drafts % kDrafts], drafts / kDrafts);
          bad = sy->told.bad[drafts % kDrafts];
          ++drafts;
        }
      }
      // (a wait can end well for one warp and badly for another)
      if constexpr (C > 1) ok = all_say(ok);
      if (!ok) break;
      tc_fence_after();
      const float o_scale = kCodes ? pow2((int)(ew - kTop)) : 1.f;
      const long long slot =
          (teams > 0 ? (long long)work : (2LL * run + (here ? 1 : 0)) * p.tiles + tile) * p.tile_rows;
      // four outputs of query row i, whose output row is `at`: the output, or the partial
      auto put = [&](int i, long long at, int d, const float4 &x) {
        if (whole)
          put4((__nv_bfloat16 *)p.out + at * D + d, x);
        else
          put4(p.ws_o + (slot + i) * D + d, x);
      };
      auto put_stats = [&](int i, float m, float l) {
        if (!whole)
          p.ws_ml[slot + i] = make_float2(m, l);
        else if (p.lse != nullptr)
          p.lse[out_row(i)] = tree_lse(m, l);
      };
      auto inverse = [&](float l) {  // 0: no row counts
        return l != l ? l : !whole ? 1.f : l != 0.f ? 1.f / l : 0.f;
      };
      if constexpr (C == 1) {
        if (warp_live) {
          const float inv = poisoned ? __int_as_float(0x7fffffff) : inverse(l) * o_scale;
          const long long at = live ? out_row(r) : 0;
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            __syncwarp();
            uint32_t u[32];
            tmem_load<32>(lanes + kOCol + c, u);
            if (!live) continue;
            float o[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = __uint_as_float(u[i]) * inv;
            if (!kCodes && (bad & mask) != 0) add_bad(bad & mask, c, o, 32);
#pragma unroll
            for (int i = 0; i < 32; i += 4)
              put(r, at, c + i, make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]));
          }
          if (live) put_stats(r, m, l);
        }
      } else {
        // the copies, in the last block's values' stage: their statistics, then a quarter of the
        // dims at a time, a row of the products each thread's, 16 bytes at places by the row's
        // low bits
        uint8_t *const stage = tiles + S::V0 + (n - 1) % SV * S::TILE;
        constexpr int CD = D / 4, CP = CD / 4;
        float2 *const stats = (float2 *)stage;
        stats[tid] = make_float2(m, l);
        named_bar_sync(1 + team, 128);
        float top = m;
#pragma unroll
        for (int k = 0; k < C; ++k) top = fmaxf(top, stats[k * RT + r].x);
        const float sub = top == -INFINITY ? 0.f : top;
        float den = 0.f;
#pragma unroll
        for (int k = 0; k < C; ++k) den += fast_exp2(stats[k * RT + r].x - sub) * stats[k * RT + r].y;
        const float f = poisoned ? __int_as_float(0x7fffffff) : fast_exp2(m - sub) * o_scale;
        if (copy == 0) {
          sy->inv[r] = inverse(den);
          sy->out_row[r] = live ? (int)(out_row(r) - (long long)seq.first * p.Hq) : 0;
          if (live) put_stats(r, top, den);
        }
        named_bar_sync(1 + team, 128);
#pragma unroll 1
        for (int c = 0; c < D; c += CD) {
          uint32_t u[CD];
          tmem_load<CD>(lanes + kOCol + c, u);
#pragma unroll
          for (int i = 0; i < CP; ++i)
            *reinterpret_cast<float4 *>(stage + tid * CD * 4 + ((i ^ (tid & (CP - 1))) << 4)) =
                make_float4(__uint_as_float(u[4 * i]) * f, __uint_as_float(u[4 * i + 1]) * f,
                            __uint_as_float(u[4 * i + 2]) * f, __uint_as_float(u[4 * i + 3]) * f);
          named_bar_sync(1 + team, 128);
          // A value before the draft that is not finite makes a NaN of the copies that do not have
          // its key (0 times it): then the outputs are the sum of what is not finite (if the
          // probabilities are numbers). What that is takes a look at all of the part's values, once
          // for all rows, and a second time over the outputs.
#pragma unroll 1
          for (int look = 0; look < 2; ++look) {
            bool nan = false;
            for (int e = tid; e < n_rows * CP; e += 128) {
              const int i = e / CP, pc = e % CP;
              float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
              for (int k = 0; k < C; ++k) {
                const int row = k * RT + i;
                const float4 y = *reinterpret_cast<const float4 *>(
                    stage + row * CD * 4 + ((pc ^ (row & (CP - 1))) << 4));
                x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
              }
              const float inv = sy->inv[i];
              float o[4] = {x.x * inv, x.y * inv, x.z * inv, x.w * inv};
              if (!kCodes && inv == inv && !((x.x + x.y) + (x.z + x.w) == (x.x + x.y) + (x.z + x.w))) {
                nan = true;
                if (look > 0) put_not_finite(4 * pc, o);
              }
              if (!kCodes && bad != 0) {
                const int tok = token_of(i);
                const unsigned long long sees =
                    p.masks == nullptr ? ~0ull >> (63 - tok) : p.masks[seq.first + tok];
                if ((bad & sees) != 0) add_bad(bad & sees, c + 4 * pc, o, 4);
              }
              put(i, sy->out_row[i] + (long long)seq.first * p.Hq, c + 4 * pc,
                  make_float4(o[0], o[1], o[2], o[3]));
            }
            // (a barrier too: the stage has been read)
            if (all_say(!nan) || look > 0) break;
            find_not_finite(c, CP);
          }
        }
        fence_proxy_async_smem();  // (the stage is written by TMA next)
        named_bar_sync(1 + team, 128);
        if (tid == 0) mbar_arrive(&sy->v_empty[(n - 1) % SV]);
      }
      tc_fence_before();  // O is read before the next group's first block is said to be ready
    }
    if (teams == 0 && tile == 0 && tid == 0 && run < p.n_runs) p.rec[run] = ok ? rec : make_int2(0, 0);
    tc_fence_before();
  }
  __syncthreads();
  tc_fence_after();
  if (cta_warp == 8) tmem_dealloc(syncs->tmem, kTeams * kTeamCols);
  if (teams == 0) return;

  // the shares' partials joined in order, a row of 16 bytes of outputs a thread; and the outputs of
  // idle sequences
  if (teams > 1) {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  }
  const int members = teams > 1 ? teams / kTeams * threads(kCodes) : threads(kCodes);
  const int me =
      threadIdx.x + (teams > 1 ? (int)blockIdx.x % (teams / kTeams) * threads(kCodes) : 0);
  for (int g = 0; g < (teams > 1 ? 1 : kTeams); ++g) {
    const int group = teams > 1 ? work / teams : (int)(blockIdx.x + g * gridDim.x);
    if (group >= p.g.B * p.g.Hkv) break;
    const int b = group / p.g.Hkv, h = group % p.g.Hkv;
    const TreeSeq seq(p, b);
    const int blocks = W::blocks_of(seq), rows = seq.tokens * p.G;
    const bool idle = seq.len == 0;
    if (!idle && (teams == 1 || blocks == 1)) continue;  // (whole shares have been written)
    constexpr int kCols = D / 4;
    for (int e = me; e < rows * kCols; e += members) {
      const int i = e / kCols, col = e % kCols;
      float m = -INFINITY, den = 0.f;
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int k0 = 0; k0 < (idle ? 0 : teams); k0 += 8) {
        float2 ml[8];
        float4 o[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int of = k0 + k;
          ml[k] = make_float2(-INFINITY, 0.f);
          o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (of < teams && (long long)blocks * of / teams < (long long)blocks * (of + 1) / teams) {
            const long long at = ((long long)group * teams + of) * p.tile_rows + i;
            ml[k] = __ldcg(&p.ws_ml[at]);
            o[k] = __ldcg(reinterpret_cast<const float4 *>(p.ws_o + at * D) + col);
          }
        }
        float mn = m;
#pragma unroll
        for (int k = 0; k < 8; ++k) mn = fmaxf(mn, ml[k].x);
        const float subm = mn == -INFINITY ? 0.f : mn, a = fast_exp2(m - subm);
        sum = make_float4(sum.x * a, sum.y * a, sum.z * a, sum.w * a);
        den *= a;
        m = mn;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float f = fast_exp2(ml[k].x - subm);
          if (ml[k].y == 0.f) continue;  // (no row counts; a share without blocks)
          sum.x += f * o[k].x;
          sum.y += f * o[k].y;
          sum.z += f * o[k].z;
          sum.w += f * o[k].w;
          den += f * ml[k].y;
        }
      }
      const long long at = (long long)(seq.first + i / p.G) * p.Hq + h * p.G + i % p.G;
      const float inv = den != 0.f ? 1.f / den : 0.f;  // 0: no row counts
      put4((__nv_bfloat16 *)p.out + at * D + 4 * col,
           make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv));
      if (p.lse != nullptr && col == 0) p.lse[at] = tree_lse(m, den);
    }
  }
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *,
                                  const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                  const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
  static std::atomic<EncodeTiledFn> fn{nullptr};
  EncodeTiledFn f = fn.load(std::memory_order_relaxed);
  if (f == nullptr) {
    void *ptr = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &ptr, 12000, cudaEnableDefault,
                                         &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess) {
      f = (EncodeTiledFn)ptr;
      fn.store(f, std::memory_order_relaxed);
    }
  }
  return f;
}

// A pool as [pages][heads][rows][dims] in boxes of up to KB rows of one page and head; false
// where its strides are none that a tensor map can have (the copies then go by 16 bytes).
bool encode(CUtensorMap *map, const PagedGeom &g, const void *pool, bool codes) {
  const EncodeTiledFn fn = encode_fn();
  if (fn == nullptr) return false;
  const int elem = codes ? 1 : 2;
  const cuuint64_t dims[4] = {(cuuint64_t)g.D, (cuuint64_t)1 << g.shift, (cuuint64_t)g.Hkv,
                              (cuuint64_t)g.n_pages};
  cuuint64_t strides[3] = {(cuuint64_t)g.row_stride * elem, (cuuint64_t)g.head_stride * elem,
                           (cuuint64_t)g.page_stride * elem};
  for (int i = 0; i < 3; ++i) {
    if (dims[i + 1] == 1) strides[i] = (cuuint64_t)g.D * elem;  // (of no use, but it has to be one)
    if (strides[i] == 0 || strides[i] >= (1ull << 40)) return false;
  }
  const cuuint32_t box[4] = {(cuuint32_t)(codes ? g.D : 64), (cuuint32_t)std::min(1 << g.shift, KB), 1, 1};
  const cuuint32_t one[4] = {1, 1, 1, 1};
  return fn(map, codes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4,
            const_cast<void *>(pool), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
            codes ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool kCodes, int C>
cudaError_t launch(TreeParams p, int dev, int sms, cudaStream_t st) {
  static std::atomic<bool> attr_set[kMaxDevices];
  constexpr int smem = Smem<D, kCodes>::BYTES;
  Maps maps;
  // (boxes of fewer than 8 rows would not lie on the swizzle's 1 KB)
  p.tma = p.g.shift >= 3 && encode(&maps.k, p.g, p.k_pages, kCodes) &&
          encode(&maps.v, p.g, p.v_pages, kCodes);
  p.suspend_ns = (uint32_t)std::min<long long>(p.wait_cycles / 4, 1000000);
  if (!attr_set[dev].load(std::memory_order_acquire)) {
    const cudaError_t e = cudaFuncSetAttribute(
        tree_tc_kernel<D, kCodes, C>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    attr_set[dev].store(true, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg = {};
  const int works = p.teams > 0 ? p.g.B * p.g.Hkv * p.teams : p.n_runs * p.tiles;
  cfg.gridDim = dim3(p.teams > 1 ? works / kTeams
                                 : std::min(works, std::max(sms, (works + kTeams - 1) / kTeams)));
  cfg.blockDim = dim3(threads(kCodes));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = p.teams > 1 ? p.teams / kTeams : 1;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.teams > kTeams ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, tree_tc_kernel<D, kCodes, C>, p, maps);
  count_launches(1);
  return e;
}

template <int D, bool kCodes>
cudaError_t launch_copies(const TreeParams &p, int dev, int sms, cudaStream_t st) {
  const int rows = p.max_tokens * p.G;
  if (rows <= kRows / 4) return launch<D, kCodes, 4>(p, dev, sms, st);
  if (rows <= kRows / 2) return launch<D, kCodes, 2>(p, dev, sms, st);
  return launch<D, kCodes, 1>(p, dev, sms, st);
}

}  // namespace

cudaError_t launch_tree_tc(const TreeParams &p, bool codes, int dev, int sms, cudaStream_t st) {
  if (codes)
    return p.g.D == 128 ? launch_copies<128, true>(p, dev, sms, st)
                        : launch_copies<64, true>(p, dev, sms, st);
  return p.g.D == 128 ? launch_copies<128, false>(p, dev, sms, st)
                      : launch_copies<64, false>(p, dev, sms, st);
}

}  // namespace ripple
