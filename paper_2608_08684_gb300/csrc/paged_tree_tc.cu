// ripple_paged_tree_attn for bf16 queries, on the 5th-generation tensor cores.
//
// A CTA (288 threads, two on an SM) has up to 128 query rows of a KV head and takes its run's
// blocks of 64 keys: S = Q . K^T (128 x 64) into TMEM, softmax by a thread a row, P as bf16
// back into TMEM over S, O += P . V (128 x d) in TMEM. A draft of n tokens with G heads a KV
// head has n G rows; up to 128 the padding costs nothing that the cache's bytes do not: a
// block is 32 KB, 1400 cycles of an SM's share of HBM, and 512 of its tensor cores.
//
// Warps 0-3: softmax and outputs; warp 4: issues the MMAs; warps 5, 6 fetch keys (and a
// group's queries), 7, 8 values: a block by TMA (a box a page, with the 128-byte swizzle that
// the MMAs read), or, where rows of it are missing or pages have fewer than 8, by 16-byte copies to
// the same places. 8-bit pages come into a ring of their own, two blocks ahead, and these
// warps make them the bf16 values that they stand for, exactly, so that all else is the same.
// Scores of the next block are on their way while a block's softmax runs; S and P of two
// blocks and O fill half of the TMEM, the other CTA's the other half.
//
// P in one bf16 part: the output is rounded to bf16 as well, and a probability's rounding
// (2^-9) enters the output as part of a mean. The sum is of the unrounded ones, in fp32.
#include "paged_tree.cuh"
#include "tc_ptx.cuh"

#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <atomic>

namespace ripple {
namespace {

constexpr int KB = kTreeTcKeys;
constexpr int kRows = kTreeTcRows;
constexpr int kThreads = 288;
constexpr int kFetchers = 64;  // threads that fetch keys, and values
constexpr int kRing = 3;       // blocks of 8-bit rows on their way or being widened
constexpr uint32_t kTmemCols = 256;  // S and P of two blocks (64 each), O (d) from 128 on
constexpr uint32_t kOCol = 128;
constexpr float kSlack = 8.f;
constexpr unsigned kAll = 0xffffffffu;
constexpr int kMaxDevices = 64;
constexpr int kSlots = 4;  // of the blocks' present rows

struct Sync {
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2];
  uint64_t ring_full[2][kRing];                         // of keys, of values
  uint64_t s_full[2], p_full[2], pv_done[2], mma_done;  // (of even and odd blocks)
  unsigned long long present[kSlots];  // rows of a block that are there
  unsigned long long bad;              // drafted tokens whose values are not all finite
  uint32_t tmem;
  int abort;                           // a role has given up waiting
  uint8_t scale[2][kRing][KB];         // of the ring's rows
};

template <int D, bool kCodes>
struct Smem {
  static constexpr int STAGES = kCodes ? 1 : 2;  // of bf16 blocks of keys, and of values
  static constexpr int Q = kRows * D * 2, TILE = KB * D * 2;
  static constexpr int RAW = KB * D;             // a block of 8-bit rows
  static constexpr int HALF_Q = kRows * 128, HALF = KB * 128;  // of 64 dims
  static constexpr int K0 = Q, V0 = Q + STAGES * TILE, RING = V0 + STAGES * TILE;
  static constexpr int SYNC = RING + (kCodes ? 2 * kRing * RAW : 0);
  static constexpr int BYTES = SYNC + (int)sizeof(Sync);
  static_assert(2 * (BYTES + 1024) <= 228 * 1024, "two CTAs an SM");
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
// for a quarter of the bound at most.
__device__ __forceinline__ bool try_wait_for(uint64_t *bar, uint32_t parity, uint32_t ns) {
  uint32_t ok;
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
__device__ __forceinline__ void copies_landed() {
  asm volatile("cp.async.wait_all;" ::: "memory");
  fence_proxy_async_smem();  // for the tensor cores' reads
}
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
__device__ __forceinline__ void tmem_wait_st() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&h);
}
// Which of two bf16 values are infinite or NaN, as masks of their halves.
__device__ __forceinline__ uint32_t not_finite(uint32_t pair) {
  return ((pair & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) |
         ((pair & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}
// The value of a scale byte as a factor; 255 is NaN.
__device__ __forceinline__ float scale_of_byte(int s) {
  return s == 255 ? __int_as_float(0x7fffffff) : __int_as_float(s << 23);  // (7..247)
}
// 16 codes times their scale as bf16, exactly.
__device__ __forceinline__ void widen(const uint4 &u, float scale, uint32_t (&o)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i / 2] >> (16 * (i & 1))), __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    o[i] = pack_bf16x2(f.x * scale, f.y * scale);
  }
}

// kCodes: 8-bit pages.
template <int D, bool kCodes>
__global__ void __launch_bounds__(kThreads, 2)
    tree_tc_kernel(const __grid_constant__ TreeParams p, const __grid_constant__ Maps maps) {
  using S = Smem<D, kCodes>;
  constexpr int ST = S::STAGES;
  using W = TreeWalk<KB>;
  extern __shared__ __align__(1024) uint8_t tiles[];
  Sync *const sy = (Sync *)(tiles + S::SYNC);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int run = blockIdx.x / p.tiles, tile = blockIdx.x % p.tiles;
  if (tid == 0) {
    sy->abort = 0;
    for (int i = 0; i < kRing; ++i) {
      mbar_init(&sy->ring_full[0][i], kFetchers);
      mbar_init(&sy->ring_full[1][i], kFetchers);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sy->k_full[i], kFetchers);
      mbar_init(&sy->v_full[i], kFetchers);
      mbar_init(&sy->k_empty[i], 1);
      mbar_init(&sy->v_empty[i], 1);
      mbar_init(&sy->s_full[i], 1);
      mbar_init(&sy->p_full[i], 4);
      mbar_init(&sy->pv_done[i], 1);
    }
    mbar_init(&sy->mma_done, 1);
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  if (warp == 4) {
    tmem_alloc(&sy->tmem, kTmemCols);
    tmem_relinquish();
  }
  pdl_wait();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sy->tmem;
  if (blockIdx.x == 0)
    for (int b = tid; b < p.g.B; b += kThreads) TreeSeq::check(p, b);

  const uint32_t qs = smem_u32(tiles), ks = qs + S::K0, vs = qs + S::V0;
  W w;
  const long long total = w.start(p, run, lane);
  const bool any = total > 0;
  int n = 0;  // blocks of this CTA so far
  bool ok = true;

  auto wait_for = [&](uint64_t *bar, int phase) {  // by a whole warp
    return __all_sync(kAll, wait_bar(bar, phase, p, &sy->abort));
  };

  if (warp >= 5) {
    // -------------------------------------------------- keys (and queries), values
    const bool keys = warp < 7;
    const int th = tid - (keys ? 160 : 224), wk = th >> 5;
    uint64_t *const full = keys ? sy->k_full : sy->v_full, *const empty = keys ? sy->k_empty : sy->v_empty;
    const uint32_t stages = keys ? ks : vs;
    const uint8_t *const pool = (const uint8_t *)(keys ? p.k_pages : p.v_pages);
    const CUtensorMap *const map = keys ? &maps.k : &maps.v;
    constexpr int kElem = kCodes ? 1 : 2;
    constexpr int kPieces = D * kElem / 16;     // of a row in its page
    constexpr int kRowsWarp = 32 / kPieces;     // rows of a warp's copy
    constexpr int kSteps = KB / (2 * kRowsWarp);
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
      if (!kCodes && keys && th == 0) sy->present[n % kSlots] = present;
      if (allowed && p.tma && present == ~0ull) {
        if (th == 0) mbar_arrive_expect_tx(bar, KB * D * kElem);
        if (wk == 0) {
          __syncwarp();
          // a lane a page: the entry of its first row
          const int boxes = KB / box, first = lane * box;
          const int e0 = __shfl_sync(kAll, entry[0], first & 31), e1 = __shfl_sync(kAll, entry[1], first & 31);
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
        }
        if (th != 0) mbar_arrive(bar);
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
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const int row = (2 * i + wk) * kRowsWarp + sub;
        const long long at = __shfl_sync(kAll, row < 32 ? place[0] : place[1], row & 31);
        copy16(kCodes ? to + row * D + 16 * pc
                      : to + (pc >> 3) * S::HALF + row * 128 + (((pc & 7) ^ (row & 7)) << 4),
               pool + (at >= 0 ? at + 16 * pc : 0), at >= 0);
      }
      return false;
    };
    // What both warps of keys (of values) agree on: they fetch a block, or neither does, so that
    // what is on its way is waited for by its barrier also when a wait has given up.
    auto both = [&](bool mine) {
      int all;
      asm volatile(
          "{\n .reg .pred p, q;\n setp.ne.b32 q, %1, 0;\n"
          " barrier.cta.red.and.pred p, %2, %3, q;\n selp.s32 %0, 1, 0, p;\n}\n"
          : "=r"(all)
          : "r"((int)mine), "r"(keys ? 2 : 3), "r"(kFetchers)
          : "memory");
      return all != 0;
    };
    int ring_n = 0, issued = 0;  // blocks that have gone through the ring, that were put there
    for (bool more = any; more && ok; more = w.next(p)) {
      const TreeSeq seq(p, w.b);
      const int n_rows = min(seq.tokens * p.G - tile * kRows, kRows);
      if (n_rows <= 0) continue;
      look_up(w.begin);
      // the group's queries, once the scores of the group before are done
      auto fetch_queries = [&]() {
        if (n > 0 && !both(wait_for(&sy->k_empty[(n - 1) % ST], (n - 1) / ST))) return false;
        constexpr int kQPieces = D / 8;
        for (int i = th; i < kRows * kQPieces; i += kFetchers) {
          const int r = i / kQPieces, c = i % kQPieces;
          const bool there = r < n_rows;
          const int row = tile * kRows + (there ? r : 0), tok = row / p.G, head = w.h * p.G + row % p.G;
          const __nv_bfloat16 *q = (const __nv_bfloat16 *)p.q + head * p.q_head +
                                   (p.starts == nullptr ? w.b * p.q_seq + tok * p.q_token
                                                        : (long long)(seq.first + tok) * p.q_token);
          copy16(qs + (c >> 3) * S::HALF_Q + r * 128 + (((c & 7) ^ (r & 7)) << 4), q + 8 * c, there);
        }
        return true;
      };
      if constexpr (!kCodes) {
        for (int row0 = w.begin; row0 < w.end; row0 += KB, ++n) {
          const int stage = n % ST;
          if (n >= ST && !(ok = both(wait_for(&empty[stage], n / ST - 1)))) break;
          // drafted tokens' values that are not finite are left out here (a hidden one's weight is
          // 0, and 0 times them is NaN) and added to the outputs of the rows that see them
          const bool draft = !keys && row0 + KB > seq.prefix, queries = keys && row0 == w.begin;
          const uint32_t to = stages + stage * S::TILE;
          if (queries && !(ok = fetch_queries())) break;
          // (the queries are waited for below, and this thread arrives after that)
          const bool by_tma = fetch(row0, to, &full[stage], !draft && !queries);
          if (row0 + KB < w.end) look_up(row0 + KB);
          if (by_tma) continue;
          asm volatile("cp.async.wait_all;" ::: "memory");
          if (draft) {
#pragma unroll 1
            for (int i = 0; i < kSteps; ++i) {
              const int row = (2 * i + wk) * kRowsWarp + sub;
              const uint32_t at = to + (pc >> 3) * S::HALF + row * 128 + (((pc & 7) ^ (row & 7)) << 4);
              const uint4 u = ld_shared16(at);
              const uint32_t b[4] = {not_finite(u.x), not_finite(u.y), not_finite(u.z), not_finite(u.w)};
              if (row0 + row >= seq.prefix && (b[0] | b[1] | b[2] | b[3]) != 0)
                st_shared16(at, u.x & ~b[0], u.y & ~b[1], u.z & ~b[2], u.w & ~b[3]);
            }
          }
          fence_proxy_async_smem();
          mbar_arrive(&full[stage]);
        }
      } else {
        const uint8_t *const scales = keys ? p.k_scales : p.v_scales;
        uint8_t(*const scale_ring)[KB] = sy->scale[keys ? 0 : 1];
        uint64_t *const ring_full = sy->ring_full[keys ? 0 : 1];
        const uint32_t ring = qs + S::RING + (keys ? 0 : kRing * S::RAW);
        const int my_row = 32 * wk + lane;
        int byte = 0, byte_slot = -1;  // of the thread's row of the block issued last
        auto put_scale = [&]() {
          if (byte_slot >= 0) scale_ring[byte_slot][my_row] = (uint8_t)byte;
          byte_slot = -1;
        };
        // the block at row0 into the ring; its scales are put there when the next one is issued
        unsigned long long ring_present[kRing];
        auto issue = [&](int row0, int i) {
          const int slot = i % kRing;
          issued = i + 1;
          put_scale();
          const int page = wk == 0 ? entry[0] : entry[1], row = row0 + my_row;
          byte = 0;
          if ((unsigned)page < (unsigned)p.g.n_pages)
            byte = scales[page * p.scale_page + w.h * p.scale_head + (row & (page_rows - 1)) * p.scale_row];
          byte_slot = slot;
          if (!fetch(row0, ring + slot * S::RAW, &ring_full[slot], true)) copies_arrive(&ring_full[slot]);
#pragma unroll
          for (int k = 0; k < kRing; ++k)
            if (k == slot) ring_present[k] = present;
          if (row0 + KB < w.end) look_up(row0 + KB);
        };
        issue(w.begin, ring_n);
        if (w.begin + KB < w.end) issue(w.begin + KB, ring_n + 1);
        for (int row0 = w.begin; row0 < w.end; row0 += KB, ++n, ++ring_n) {
          put_scale();
          if (row0 + 2 * KB < w.end) issue(row0 + 2 * KB, ring_n + 2);
          const int slot = ring_n % kRing, stage = n % ST;
          // (then the scales of this block are there as well)
          ok = both(wait_for(&ring_full[slot], ring_n / kRing) &&
                    (n < ST || wait_for(&empty[stage], n / ST - 1)));
          if (!ok) break;
          if (keys && row0 == w.begin && !(ok = fetch_queries())) break;
          if (keys && th == 0) {
#pragma unroll
            for (int k = 0; k < kRing; ++k)
              if (k == slot) sy->present[n % kSlots] = ring_present[k];
          }
          const uint32_t from = ring + slot * S::RAW, to = stages + stage * S::TILE;
          const bool draft = !keys && row0 + KB > seq.prefix;
#pragma unroll
          for (int i = 0; i < kSteps; ++i) {
            const int row = (2 * i + wk) * kRowsWarp + sub;
            float f = scale_of_byte(scale_ring[slot][row]);
            uint4 u = ld_shared16(from + row * D + 16 * pc);
            if (draft && f != f && row0 + row >= seq.prefix) {  // as infinite values of bf16 pages
              f = 0.f;
              u = make_uint4(0, 0, 0, 0);
            }
            uint32_t o[8];
            widen(u, f, o);
            const int c = 2 * pc;  // of 16-byte pieces in the stage
            const uint32_t at = to + (c >> 3) * S::HALF + row * 128;
            st_shared16(at + (((c & 7) ^ (row & 7)) << 4), o[0], o[1], o[2], o[3]);
            st_shared16(at + ((((c & 7) + 1) ^ (row & 7)) << 4), o[4], o[5], o[6], o[7]);
          }
          if (keys && row0 == w.begin) asm volatile("cp.async.wait_all;" ::: "memory");
          fence_proxy_async_smem();
          mbar_arrive(&full[stage]);
          named_bar_sync(keys ? 2 : 3, kFetchers);  // the slot has been read
        }
      }
    }
    copies_landed();
    if (!ok) {  // what TMA still has on its way lands before the CTA leaves
      if (!kCodes) {
        for (int i = max(0, n - ST); i < n; ++i) mbar_wait(&full[i % ST], i / ST & 1, nullptr);
      } else {
        for (int i = max(0, issued - kRing); i < issued; ++i)
          mbar_wait(&sy->ring_full[keys ? 0 : 1][i % kRing], i / kRing & 1, nullptr);
      }
    }
  } else if (warp == 4) {
    // -------------------------------------------------- MMAs (the whole warp waits, one lane issues)
    constexpr uint32_t id_qk = idesc_bf16(kRows, KB);
    constexpr uint32_t id_pv = idesc_bf16(kRows, D) | (1u << 16);  // V: d is the contiguous one
    const uint64_t qd = sw128_desc(qs);
    // scores of block i: S(i). The products P . V of the blocks up to n - 1 have been issued, and
    // all of them have to be done: P of block i - 2 lies where S(i) goes, and a barrier that has
    // gone on by two phases cannot be waited for.
    auto scores = [&](int i) {
      const int st = i % ST;
      if (!wait_for(&sy->k_full[st], i / ST)) return false;
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
    for (bool more = any; more && ok; more = w.next(p)) {
      const TreeSeq seq(p, w.b);
      if (seq.tokens * p.G - tile * kRows <= 0) continue;
      const int count = w.count();
      ok = scores(n);
      for (int i = 0; i < count && ok; ++i, ++n) {
        if (i + 1 < count && !(ok = scores(n + 1))) break;
        const int st = n % ST;
        if (!wait_for(&sy->p_full[n & 1], n / 2) || !wait_for(&sy->v_full[st], n / ST)) {
          ok = false;
          break;
        }
        tc_fence_after();
        if (elect_one()) {
          const uint64_t vd = sw128_desc_mn(vs + st * S::TILE, S::HALF, 1024);
#pragma unroll
          for (int kk = 0; kk < KB / 16; ++kk)  // 16 keys: 8 columns of P, 2 KB of V
            mma_bf16_ts(tmem + kOCol, tmem + (n & 1) * KB + kk * 8, vd + (kk * 2048 >> 4), id_pv,
                        kk > 0 || i > 0);
          mma_commit(&sy->v_empty[st]);
          mma_commit(&sy->pv_done[n & 1]);
        }
        __syncwarp();
      }
    }
    if (elect_one()) mma_commit(&sy->mma_done);
    __syncwarp();
    mbar_wait(&sy->mma_done, 0, nullptr);
  } else {
    // -------------------------------------------------- softmax and outputs, a thread a row
    const uint32_t lanes = tmem + ((uint32_t)(32 * warp) << 16);
    int2 rec = make_int2(0, 0);
    const int runs = (int)min((long long)p.n_runs, total);
    long long t = any ? run_start(total, runs, run) : 0;
    const int r = tid;  // row of the tile
    for (bool more = any; more && ok; t += w.count(), more = w.next(p)) {
      const TreeSeq seq(p, w.b);
      const bool here = w.block == 0, ends = w.block + w.count() == w.blocks();
      if (here && !ends)
        rec = make_int2(w.b * p.g.Hkv + w.h, run_of(total, runs, t + w.blocks() - 1) - run + 1);
      const int n_rows = min(seq.tokens * p.G - tile * kRows, kRows);
      if (n_rows <= 0) continue;
      const int row = tile * kRows + r, tok = row / p.G;
      const bool live = r < n_rows, warp_live = 32 * warp < n_rows;
      uint64_t mask = 0;
      if (live) mask = p.masks == nullptr ? ~0ull >> (63 - tok) : p.masks[seq.first + tok];
      // drafted tokens of this part whose values are not finite
      unsigned long long bad = 0;
      if (w.end > seq.prefix) {
        if (tid == 0) sy->bad = 0;
        named_bar_sync(1, 128);
        for (int j = warp; j < seq.tokens; j += 4) {
          const long long at_row = seq.prefix + j;
          if (at_row < w.begin || at_row >= w.end) continue;
          const int page = p.table[guard((long long)w.b * p.g.max_pages + (at_row >> p.g.shift), 1,
                                         (long long)p.g.B * p.g.max_pages, p.status)];
          if ((unsigned)page >= (unsigned)p.g.n_pages) continue;
          const int slot = (int)(at_row & ((1 << p.g.shift) - 1));
          bool found;
          if constexpr (kCodes) {
            found = p.v_scales[page * p.scale_page + w.h * p.scale_head + slot * p.scale_row] == 255;
          } else {
            const uint32_t *v = reinterpret_cast<const uint32_t *>(
                (const __nv_bfloat16 *)p.v_pages + page * p.g.page_stride + w.h * p.g.head_stride +
                slot * p.g.row_stride);
            uint32_t any_bad = 0;
#pragma unroll
            for (int i = 0; i < D / 64; ++i) any_bad |= not_finite(v[lane + 32 * i]);
            found = any_bad != 0;
          }
          if (__any_sync(kAll, found) && lane == 0) atomicOr(&sy->bad, 1ull << j);
        }
        named_bar_sync(1, 128);
        bad = sy->bad & mask;
      }
      float m = -INFINITY, l = 0.f;
      bool begun = false;  // O has a block
      for (int row0 = w.begin; row0 < w.end && ok; row0 += KB, ++n, begun = true) {
        if (!(ok = wait_for(&sy->s_full[n & 1], n / 2))) break;
        if (warp_live) {
          tc_fence_after();
          const uint32_t s_at = lanes + (n & 1) * KB;
          const unsigned long long present = sy->present[n % kSlots];
          const bool masked = present != ~0ull || row0 + KB > seq.prefix;
          unsigned long long seen = ~0ull;
          if (masked) {
            // the draft's token j is the block's key j - j0
            const long long j0 = row0 - seq.prefix;
            seen = present & (j0 <= -64 ? ~0ull
                              : j0 < 0  ? mask << -j0 | ((1ull << -j0) - 1)
                              : j0 < 64 ? mask >> j0
                                        : 0ull);
          }
          // 32 scores of the row (read twice: a thread has no room for 64 beside the rest)
          uint32_t u[32];
          auto load_scores = [&](int half) {
            tmem_ld32(s_at + 32 * half, u);
            tmem_wait_ld();
            if (masked) {
              const uint32_t on = (uint32_t)(seen >> (32 * half));
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (!(on >> i & 1)) u[i] = 0xff800000u;  // -infinity
            }
          };
          float mb = -INFINITY;
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            load_scores(half);
#pragma unroll
            for (int i = 0; i < 32; ++i) mb = fmaxf(mb, __uint_as_float(u[i]));
          }
          mb *= p.scale2;  // (>= 0)
          float a = 1.f;
          const bool grow = mb > m + kSlack;
          if (grow) {
            a = fast_exp2(m - mb);
            m = mb;
            l *= a;
          }
          if (__any_sync(kAll, grow) && begun) {
            // O of the blocks before, once they are in it
            if (!(ok = wait_for(&sy->pv_done[(n - 1) & 1], (n - 1) / 2))) break;
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
              uint32_t o[32];
              tmem_ld32(lanes + kOCol + c, o);
              tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * a);
              tmem_st32(lanes + kOCol + c, o);
            }
          }
          // scores of -infinity alone leave no finite maximum; the fused multiply-add, which
          // leaves out the score's rounding, must not meet a maximum whose own rounding counts
          const float sub = m == -INFINITY ? 0.f : m;
          const bool rounded = fabsf(sub) >= 65536.f;
          float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int half = 0; half < 2; ++half) {  // (P lies over scores that have been read)
            load_scores(half);
            uint32_t pr[16];
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              float e[2];
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                const float sc = __uint_as_float(u[i + k]);
                const float y = rounded ? sc * p.scale2 - sub : fmaf(sc, p.scale2, -sub);
                e[k] = fast_exp2(y);
                sum[(i / 2) & 3] += e[k];
              }
              pr[i / 2] = pack_bf16x2(e[0], e[1]);
            }
            tmem_st16(s_at + 16 * half, pr);
          }
          l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
          tmem_wait_st();
          tc_fence_before();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&sy->p_full[n & 1]);
      }
      if (!ok || !(ok = wait_for(&sy->pv_done[(n - 1) & 1], (n - 1) / 2))) break;
      if (!warp_live) continue;
      tc_fence_after();
      const bool whole = here && ends;
      const long long slot = ((2LL * run + (here ? 1 : 0)) * p.tiles + tile) * p.tile_rows + r;
      const long long at = (long long)(seq.first + tok) * p.Hq + w.h * p.G + row % p.G;
      const float inv = !whole ? 1.f : l != 0.f ? 1.f / l : 0.f;  // 0: no row counts
#pragma unroll 1
      for (int c = 0; c < D; c += 32) {
        __syncwarp();
        uint32_t o[32];
        tmem_ld32(lanes + kOCol + c, o);
        tmem_wait_ld();
        if (!live) continue;
        if (bad != 0) {
          for (unsigned long long left = bad; left != 0; left &= left - 1) {
            const long long at_row = seq.prefix + __ffsll(left) - 1;
            const int page = p.table[guard((long long)w.b * p.g.max_pages + (at_row >> p.g.shift), 1,
                                           (long long)p.g.B * p.g.max_pages, p.status)];
            const int v_slot = (int)(at_row & ((1 << p.g.shift) - 1));
            const __nv_bfloat16 *v = (const __nv_bfloat16 *)p.v_pages + page * p.g.page_stride +
                                     w.h * p.g.head_stride + v_slot * p.g.row_stride + c;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              const float x = kCodes ? __int_as_float(0x7fffffff) : __bfloat162float(v[i]);
              if (!(fabsf(x) < INFINITY)) o[i] = __float_as_uint(__uint_as_float(o[i]) + x);
            }
          }
        }
#pragma unroll
        for (int i = 0; i < 32; i += 8) {
          float y[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) y[k] = __uint_as_float(o[i + k]) * inv;
          if (whole) {
            *reinterpret_cast<uint4 *>((__nv_bfloat16 *)p.out + at * D + c + i) =
                make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]),
                           pack_bf16x2(y[6], y[7]));
          } else {
            put4(p.ws_o + slot * D + c + i, make_float4(y[0], y[1], y[2], y[3]));
            put4(p.ws_o + slot * D + c + i + 4, make_float4(y[4], y[5], y[6], y[7]));
          }
        }
      }
      if (live) {
        if (!whole)
          p.ws_ml[slot] = make_float2(m, l);
        else if (p.lse != nullptr)
          p.lse[at] = tree_lse(m, l);
      }
      tc_fence_before();  // O is read before the next group's first block is said to be ready
    }
    if (tile == 0 && tid == 0) p.rec[run] = ok ? rec : make_int2(0, 0);
    tc_fence_before();
  }
  __syncthreads();
  tc_fence_after();
  if (warp == 4) tmem_dealloc(tmem, kTmemCols);
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

template <int D, bool kCodes>
cudaError_t launch(TreeParams p, int dev, cudaStream_t st) {
  static std::atomic<bool> attr_set[kMaxDevices];
  constexpr int smem = Smem<D, kCodes>::BYTES;
  Maps maps;
  // (boxes of fewer than 8 rows would not lie on the swizzle's 1 KB)
  p.tma = p.g.shift >= 3 && encode(&maps.k, p.g, p.k_pages, kCodes) &&
          encode(&maps.v, p.g, p.v_pages, kCodes);
  p.suspend_ns = (uint32_t)std::min<long long>(p.wait_cycles / 4, 1000000);
  if (!attr_set[dev].load(std::memory_order_acquire)) {
    const cudaError_t e = cudaFuncSetAttribute(
        tree_tc_kernel<D, kCodes>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    attr_set[dev].store(true, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.n_runs * p.tiles);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, tree_tc_kernel<D, kCodes>, p, maps);
  count_launches(1);
  return e;
}

}  // namespace

cudaError_t launch_tree_tc(const TreeParams &p, bool codes, int dev, cudaStream_t st) {
  if (codes) return p.g.D == 128 ? launch<128, true>(p, dev, st) : launch<64, true>(p, dev, st);
  return p.g.D == 128 ? launch<128, false>(p, dev, st) : launch<64, false>(p, dev, st);
}

}  // namespace ripple
