// ripple_paged_decode_attn: attention of one new token per sequence over a paged cache.
//
// Work: the cache rows of every (sequence, KV head) group are cut into blocks of 4 KB (K
// and V each), and the blocks of all groups, in order, into runs, one CTA of one warp
// each, eight per SM. Lengths are read on the device (graphs are replayed with new ones);
// every CTA finds its run by a sum over the sequences. The first runs, one for every
// place on the GPU, hold most of the blocks, later ones less and less (Runs): SMs differ
// by a tenth in the bandwidth they get, and the later runs go where a place is free first.
// (One run of equal length for every warp: 158 us for 62 sequences of 3800 rows, 965 MB,
// of which the slowest SMs took 144 and the fastest 120.) What a run covers does not
// depend on where it goes, so results do not either.
//
// A warp is on its own: it fetches its blocks with asynchronous 16-byte copies into a
// ring, two blocks ahead, whatever the page size and layout (a lane looks up the page of
// one row of the block, one block before it is fetched), and keeps a running maximum and
// sum. Copies of 16 bytes and not bulk copies, because a block's rows need a layout that
// ldmatrix reads without bank conflicts, and pages may be one row. Rows behind a length
// and rows whose page is none are filled with zeros and left out by their place, so that
// what lies there never counts.
//
// bf16: warp-level matrix instructions (mma.sync: a step is bound by its bytes, and its few
// rows would leave tcgen05's 128-row tiles empty), probabilities in three bf16 parts so
// that nothing is lost against fp32, short chains in the accumulators because matrix
// instructions cut their sums off. fp32: the CUDA cores.
//
// A group that lies in one run is written there. Of the others every run leaves a partial
// in the workspace (a run has two at most: of the group it begins within and of the one
// it ends within), and the run with the group's first block a record of them; a second
// launch, a programmatic dependent of the first, joins them in order.
//
// Short caches (tables with room for few blocks a warp, as compressed caches have): a
// cluster of up to eight CTAs of four warps takes a group, the warps equal parts of it,
// and joins them through shared memory: one launch, no sums over the sequences and no
// workspace (short_cluster).
#include <math.h>

#include <atomic>

#include "common.cuh"
#include "kernels.cuh"
#include "paged.cuh"
#include "warp_attn.cuh"

namespace ripple {
namespace {

constexpr int kMaxGroup = 16;
constexpr int kBlockBytes = 4096;  // of K (and of V) a block
constexpr int kStages = 3;         // blocks in the ring
constexpr int kWarpsPerSm = 8;
// A running maximum (log2 units) moves only when a score exceeds it by more than this.
constexpr float kSlack = 8.f;
constexpr unsigned kAll = 0xffffffffu;
constexpr int kMaxDevices = 64;

// The runs: kPhases times one for every place (warp) on the GPU, the phases' shares of the
// blocks in 1/256. Few blocks, and few groups (of which each would be left in hundreds of
// partials), are one phase.
// Shares measured (us; D 128, 8 KV heads): 64 sequences of 3800 rows, 4 heads a group, with
// ends at 170 and 225: 148.8, 190 and 236: 147.8, 210 and 245: 146.0, one phase 152.9; of 64 to
// 32768 rows 152.7, 151.9, 150.7, one phase 156.6; 9 of 12970 rows 66.0, 66.3, 68.3.
constexpr int kPhases = 3;
__device__ __forceinline__ int share_before(int phase) {
  return phase == 0 ? 0 : phase == 1 ? 190 : phase == 2 ? 236 : 256;
}
// Blocks per place, at most. One phase and three (us, 64 sequences of equal lengths, bf16 with
// 4 and 8 heads a group, fp32 with one head of 64): 24 blocks 45.8 and 48.0, 48.6 and 54.3, 42.6
// and 45.3; 30 blocks 53.6 and 55.6, 57.9 and 62.8, 51.1 and 52.9; 34 blocks 59.4 and 61.1, 62.5
// and 68.2, 56.4 and 58.0; 48 blocks 79.3 and 79.3, 82.9 and 87.4, 76.3 and 76.4; 96 blocks 146.7
// and 142.8, 152.5 and 151.9, 140.8 and 137.2. (Three phases gain above about 48 blocks, and
// with 8 heads a group above 90.)
constexpr int kOnePhase = 32;
// One phase and three (us, 8 KV heads, 48 blocks a place): 1 sequence 79.7 and 93.4, 2 79.1
// and 87.5, 4 (32 groups) 77.3 and 82.2, 7 (56) 78.2 and 81.0, 8 (64) 61.6 and 65.0 (with twice
// the rows 113.5 and 113.7), 9 (72) 64.2 and 66.3, with twice the rows 117.9 and 116.8, 16 (128)
// with twice the rows 130.9 and 128.8.
constexpr int kFewGroups = 64;

struct PagedDecParams {
  PagedGeom g;
  int Hq, G;
  float scale2;
  const void *q;
  long long q_seq, q_head;  // strides, elements
  const void *k_pages, *v_pages;
  const int32_t *table, *lens;
  float *out, *lse;
  int32_t *status;
  int places, n_runs;  // warps that find a place at once (short caches: CTAs of a cluster), runs
  int2 *rec;      // [n_runs] the group that begins in the run and goes on, and its runs (0: none)
  float *ws_o;    // [2 * n_runs][G][D] partial outputs: of the group begun before, begun here
  float2 *ws_ml;  // [2 * n_runs][G] their maximum and sum
};

template <typename T, int D, int G>
struct Cfg {
  static constexpr bool kMma = sizeof(T) == 2;
  static constexpr int ROW_BYTES = D * (int)sizeof(T);
  static constexpr int PIECES = ROW_BYTES / 16;
  static constexpr int RB = kBlockBytes / ROW_BYTES;  // rows of a block: 8, 16 or 32
  // fp32: lanes per row (a lane's queries and outputs stay at 64 registers each), rows per
  // warp step and steps of a block
  static constexpr int S0 = G * D / 64 > G ? G * D / 64 : G;
  static constexpr int S = S0 > ROW_BYTES / 128 ? S0 : ROW_BYTES / 128;
  static constexpr int R = 32 / S;
  static constexpr int STEPS = RB / R;
  static constexpr int PPL = PIECES / S;  // 16-byte pieces of a row a lane has
  // where a piece of a row lies in the block: rows are multiples of 128 bytes, so eight rows
  // of ldmatrix, or the rows of a quarter warp, must differ in the piece
  static __device__ __forceinline__ int swizzle(int row) {
    return kMma ? row & 7 : (row * S) & 7;
  }
  static_assert(kMma || (S <= 32 && STEPS >= 1 && STEPS * R == RB && PPL >= 1), "lane layout");
};

__device__ __forceinline__ int clamp_len(const PagedDecParams &p, int b) {
  const long long room = (long long)p.g.max_pages << p.g.shift;
  const int n = p.lens[b];
  return n <= 0 ? 0 : (int)(n < room ? n : room);
}
// Where the runs of `total` blocks begin.
struct Runs {
  long long total;
  int places, phases;
  __device__ __forceinline__ Runs(long long total_, int places_, int n_runs) : total(total_) {
    const bool one = total <= (long long)kOnePhase * places_ || n_runs < kPhases * places_;
    places = one ? (int)min((long long)min(places_, n_runs), total) : places_;
    phases = one ? 1 : kPhases;
  }
  __device__ __forceinline__ int count() const { return places * phases; }
  __device__ __forceinline__ long long phase_start(int i) const {
    return phases == 1 ? (i == 0 ? 0 : total) : total * share_before(i) / 256;
  }
  __device__ __forceinline__ long long start(int run) const {
    if (run >= count()) return total;
    const int ph = run / places;
    const long long a = phase_start(ph), n = phase_start(ph + 1) - a;
    return a + n * (run - ph * places) / places;
  }
  // The run that has block t.
  __device__ __forceinline__ int of(long long t) const {
    int ph = 0;
    while (ph + 1 < phases && t >= phase_start(ph + 1)) ++ph;
    const long long a = phase_start(ph), n = phase_start(ph + 1) - a;
    return ph * places + (int)(((t - a + 1) * places - 1) / n);
  }
};

// A walk over the parts of groups in a warp's run. RB: rows of a block.
template <int RB>
struct Walk {
  int b, h, len;
  int block;           // the part's first in its group
  int begin, end;      // the part's rows
  long long left;      // blocks of the run, the part's included
  static __device__ __forceinline__ int blocks_of(int len) { return len / RB + (len % RB != 0); }
  __device__ __forceinline__ int blocks() const { return blocks_of(len); }
  __device__ __forceinline__ int count() const {
    return (int)min((long long)(blocks() - block), left);
  }
  __device__ __forceinline__ void set() {
    begin = block * RB;
    end = (int)min((long long)len, (long long)(block + count()) * RB);
  }
  // To the next part; false at the end of the run.
  __device__ __forceinline__ bool next(const PagedDecParams &p) {
    left -= count();
    if (left <= 0) return false;
    block = 0;
    if (++h >= p.g.Hkv) {
      h = 0;
      do len = clamp_len(p, ++b);
      while (len == 0);  // left > 0: there are more
    }
    set();
    return true;
  }
};

// The cache rows pass L2 once; what is read again (tables, partials) stays.
__device__ __forceinline__ uint64_t evict_first() {
  uint64_t p;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
  return p;
}
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool there, uint64_t policy) {
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;" ::"r"(dst),
               "l"(src), "r"(there ? 16 : 0), "l"(policy)
               : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
// A warp's fetching side: the walk, the next block of this warp in its part, and the page
// of the lane's row in that block.
template <typename T, int D, int G>
struct Fetch {
  using C = Cfg<T, D, G>;
  Walk<C::RB> w;
  int at;      // the next block's first row
  bool live;   // there is a next block
  int entry;   // block-table entry of the block, or of row at + lane % RB where it has several
  uint64_t policy;
  __device__ __forceinline__ void look_up(const PagedDecParams &p, int lane) {
    const int row = (1 << p.g.shift) >= C::RB ? at : at + lane % C::RB;
    entry = -1;
    if (row < w.end)
      entry = p.table[guard((long long)w.b * p.g.max_pages + (row >> p.g.shift), 1,
                            (long long)p.g.B * p.g.max_pages, p.status)];
  }
  // Copies the block into `stage` and goes on; returns its live rows as bits. A lane copies
  // piece lane % PIECES of every kRowsPer-th row.
  __device__ __forceinline__ uint32_t issue(const PagedDecParams &p, uint8_t (*stage)[kBlockBytes],
                                            int lane) {
    constexpr int kCopies = kBlockBytes / 512, kRowsPer = 32 / C::PIECES;
    const int r0 = lane / C::PIECES, pc = lane % C::PIECES;
    uint32_t rows = 0;
    if (live) {
      const uint32_t ks = smem_u32(stage[0]) + r0 * C::ROW_BYTES;
      const uint32_t vs = smem_u32(stage[1]) + r0 * C::ROW_BYTES;
      auto place = [&](int j) {  // in a stage, of the lane's copy j
        return j * 512u + ((pc ^ C::swizzle(j * kRowsPer + r0)) << 4);
      };
      const long long in_page = (at & ((1 << p.g.shift) - 1)) * p.g.row_stride + w.h * p.g.head_stride;
      if ((1 << p.g.shift) >= C::RB) {  // the block lies in one page
        const int n = min(C::RB, w.end - at);
        const bool ok = (unsigned)entry < (unsigned)p.g.n_pages;
        if (!ok && lane == 0) report(p.status, RIPPLE_EBOUNDS);
        rows = ok ? 0xffffffffu >> (32 - n) : 0u;
        const long long off =
            ok ? entry * p.g.page_stride + in_page + r0 * p.g.row_stride + pc * (16 / (int)sizeof(T))
               : 0;
        const T *k = (const T *)p.k_pages + off, *v = (const T *)p.v_pages + off;
        const long long step = kRowsPer * p.g.row_stride;
        if (rows == 0xffffffffu >> (32 - C::RB)) {
#pragma unroll
          for (int j = 0; j < kCopies; ++j, k += step, v += step) {
            copy16(ks + place(j), k, true, policy);
            copy16(vs + place(j), v, true, policy);
          }
        } else {
#pragma unroll
          for (int j = 0; j < kCopies; ++j, k += step, v += step) {
            const bool has = rows >> (j * kRowsPer + r0) & 1;
            copy16(ks + place(j), has ? k : (const T *)p.k_pages, has, policy);
            copy16(vs + place(j), has ? v : (const T *)p.v_pages, has, policy);
          }
        }
      } else {  // a page for each lane's row
        const int row = at + lane % C::RB;
        const bool there = row < w.end, ok = there && (unsigned)entry < (unsigned)p.g.n_pages;
        if (there && !ok) report(p.status, RIPPLE_EBOUNDS);
        rows = __ballot_sync(kAll, ok) & (0xffffffffu >> (32 - C::RB));
        const long long off = ok ? entry * p.g.page_stride +
                                       (row & ((1 << p.g.shift) - 1)) * p.g.row_stride +
                                       w.h * p.g.head_stride
                                 : 0;
#pragma unroll
        for (int j = 0; j < kCopies; ++j) {
          const int r = j * kRowsPer + r0;
          const long long o = __shfl_sync(kAll, off, r) + pc * (16 / (int)sizeof(T));
          const bool has = rows >> r & 1;
          copy16(ks + place(j), (const T *)p.k_pages + o, has, policy);
          copy16(vs + place(j), (const T *)p.v_pages + o, has, policy);
        }
      }
      at += C::RB;
      if (at >= w.end) {
        live = w.next(p);
        at = w.begin;
      }
      if (live) look_up(p, lane);
    }
    copy_commit();
    return rows;
  }
};

// ------------------------------------------------------------ a warp's rows, bf16
// Scores S[row][key] = Q . K^T with the heads as rows (accumulator lane (g, t): row g, keys
// 2t, 2t + 1), online softmax on those lanes, O[row][dim] += P . V with the probabilities, as
// they lie, as the A operand. Their three parts fill the operand's 16 rows: up to 4 heads
// repeat in rows 4-7 and take rows 0-3 (high), 4-7 (middle) and 8-15 (half of the low part,
// twice) of one MMA; up to 8 take rows 0-7 (high), 8-15 (middle) and a second MMA (half of
// the low part on all 16); up to 16 take one MMA per part.
template <typename T, int D, int G>
struct Rows {
  using C = Cfg<T, D, G>;
  static_assert(C::kMma, "");
  static constexpr int NB = D / 8;
  static constexpr int H = G > 8 ? 2 : 1;  // heads of a lane: g and g + 8
  uint32_t qa[D / 16][2 * H];
  float2 acc[NB][H];
  float m[H], l[H];

  __device__ __forceinline__ void start(const PagedDecParams &p, const Walk<C::RB> &w, int lane) {
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int i = 0; i < H; ++i) {
      const int head = (G > 4 ? g : g & 3) + 8 * i;
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int b = 0; b < NB; ++b) acc[b][i] = make_float2(0.f, 0.f);
      const uint32_t *q = reinterpret_cast<const uint32_t *>(
          (const T *)p.q + w.b * p.q_seq + (w.h * p.G + min(head, p.G - 1)) * p.q_head);
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        const uint32_t lo = q[k * 8 + t], hi = q[k * 8 + 4 + t];
        qa[k][2 * i] = head < p.G ? lo : 0u;
        qa[k][2 * i + 1] = head < p.G ? hi : 0u;
      }
    }
  }

  // 16 rows at ks, vs (rows of a block from a multiple of 16 on); kMask: some are not there.
  template <bool kMask>
  __device__ __forceinline__ void step(float scale2, uint32_t ks, uint32_t vs, uint32_t live,
                                       int lane) {
    const int g = lane >> 2, t = lane & 3, r8 = lane & 7;
    float sc[2][2 * H];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 2 * H; ++e) sc[i][e] = 0.f;
    const uint32_t kx = (lane >> 3) ^ r8, ka = ks + r8 * C::ROW_BYTES;
#pragma unroll
    for (int k2 = 0; k2 < D / 32; ++k2) {
      uint32_t kb[2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i)
        ldmatrix4(ka + i * 8 * C::ROW_BYTES + ((kx ^ (k2 * 4)) << 4), kb[i]);
      float part[2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) part[i][e] = 0.f;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t(&a)[2 * H] = qa[2 * k2 + h];
          mma_bf16(part[i], a[0], H > 1 ? a[2 * H - 2] : 0u, a[1], H > 1 ? a[2 * H - 1] : 0u,
                   kb[i][2 * h], kb[i][2 * h + 1]);
        }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 2 * H; ++e) sc[i][e] += part[i][e];
    }
    Parts pp[H][2];
#pragma unroll
    for (int u = 0; u < H; ++u) {
      // this lane's keys of block i: 8 i + 2 t + e
      float x[2][2];
      bool on[2][2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          on[i][e] = !kMask || (live >> (8 * i + 2 * t + e) & 1);
          x[i][e] = on[i][e] ? sc[i][2 * u + e] * scale2 : -INFINITY;
        }
      const float mb = fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[1][0], x[1][1]));
      if (__any_sync(kAll, mb > m[u] + kSlack)) {
        float mr = fmaxf(mb, __shfl_xor_sync(kAll, mb, 1));
        mr = fmaxf(mr, __shfl_xor_sync(kAll, mr, 2));
        if (mr > m[u] + kSlack) {
          const float a = fast_exp2(m[u] - mr);
          l[u] *= a;
#pragma unroll
          for (int b = 0; b < NB; ++b) acc[b][u] = __fmul2_rn(acc[b][u], make_float2(a, a));
          m[u] = mr;
        }
        __syncwarp();
      }
      // scores of -infinity alone leave no finite maximum; the fused multiply-add, which leaves
      // out the rounding of the score, must not meet a maximum whose own rounding is a large
      // part of 1; a row that is not there counts for nothing by its place, so that a NaN score
      // of one that is reaches the output
      const float sub = m[u] == -INFINITY ? 0.f : m[u];
      const bool rounded = fabsf(sub) >= 65536.f;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float w[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float y = rounded ? x[i][e] - sub : fmaf(sc[i][2 * u + e], scale2, -sub);
          w[e] = on[i][e] ? fast_exp2(y) : 0.f;
          l[u] += w[e];
        }
        pp[u][i] = three_parts<(G <= 8)>(w[0], w[1]);
      }
    }
    const uint32_t vx = (lane >> 4) ^ r8, va = vs + (r8 + ((lane >> 3) & 1) * 8) * C::ROW_BYTES;
#pragma unroll
    for (int b2 = 0; b2 < NB / 2; ++b2) {
      uint32_t vb[4];  // keys 0-7 and 8-15 of 8 dims, then of the next 8
      ldmatrix4_trans(va + ((vx ^ (b2 * 2)) << 4), vb);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t v0 = vb[2 * e], v1 = vb[2 * e + 1];
        float part[4] = {0.f, 0.f, 0.f, 0.f};
        if constexpr (G > 8) {
          mma_bf16(part, pp[0][0].l, pp[H - 1][0].l, pp[0][1].l, pp[H - 1][1].l, v0, v1);
          mma_bf16(part, pp[0][0].m, pp[H - 1][0].m, pp[0][1].m, pp[H - 1][1].m, v0, v1);
          mma_bf16(part, pp[0][0].h, pp[H - 1][0].h, pp[0][1].h, pp[H - 1][1].h, v0, v1);
          acc[2 * b2 + e][0] = __fadd2_rn(acc[2 * b2 + e][0], make_float2(part[0], part[1]));
          acc[2 * b2 + e][H - 1] = __fadd2_rn(acc[2 * b2 + e][H - 1], make_float2(part[2], part[3]));
        } else {
          const Parts &p0 = pp[0][0], &p1 = pp[0][1];
          if (G > 4) mma_bf16(part, p0.l, p0.l, p1.l, p1.l, v0, v1);
          const bool high = G > 4 || g < 4;
          mma_bf16(part, high ? p0.h : p0.m, G > 4 ? p0.m : p0.l, high ? p1.h : p1.m,
                   G > 4 ? p1.m : p1.l, v0, v1);
          acc[2 * b2 + e][0] = __fadd2_rn(acc[2 * b2 + e][0],
                                          make_float2(part[0] + part[2], part[1] + part[3]));
        }
      }
    }
  }

  __device__ __forceinline__ void block(const PagedDecParams &p, uint8_t (*stage)[kBlockBytes],
                                        uint32_t live, int lane) {
    const uint32_t ks = smem_u32(stage[0]), vs = smem_u32(stage[1]);
#pragma unroll 1
    for (int i = 0; i < C::RB / 16; ++i) {
      const uint32_t part = live >> (16 * i) & 0xffffu, at = i * 16 * C::ROW_BYTES;
      if (part == 0xffffu)
        step<false>(p.scale2, ks + at, vs + at, part, lane);
      else if (part != 0)
        step<true>(p.scale2, ks + at, vs + at, part, lane);
    }
  }

  // The warp's rows done: full sums, each head's parts added up.
  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int u = 0; u < H; ++u) {
      l[u] += __shfl_xor_sync(kAll, l[u], 1);
      l[u] += __shfl_xor_sync(kAll, l[u], 2);
    }
    if (G <= 4) {
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        acc[b][0].x += __shfl_xor_sync(kAll, acc[b][0].x, 16);
        acc[b][0].y += __shfl_xor_sync(kAll, acc[b][0].y, 16);
      }
    }
  }
  // The outputs of a group that is done.
  __device__ __forceinline__ void normalise() {
#pragma unroll
    for (int u = 0; u < H; ++u) {
      const float inv = l[u] != 0.f ? 1.f / l[u] : 0.f;  // 0: no row counts
#pragma unroll
      for (int b = 0; b < NB; ++b) acc[b][u] = __fmul2_rn(acc[b][u], make_float2(inv, inv));
    }
  }
  // f(head, its maximum, its sum), once per head
  template <typename F>
  __device__ __forceinline__ void stats(int lane, F f) {
    const int g = lane >> 2;
#pragma unroll
    for (int u = 0; u < H; ++u)
      if (g + 8 * u < G && (lane & 3) == 0) f(g + 8 * u, m[u], l[u]);
  }
  // f(head, dim, its output and the next dim's)
  template <typename F>
  __device__ __forceinline__ void outputs(int lane, F f) {
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int u = 0; u < H; ++u)
      if (g + 8 * u < G) {
#pragma unroll
        for (int b = 0; b < NB; ++b) f(g + 8 * u, b * 8 + 2 * t, acc[b][u]);
      }
  }
};

// ------------------------------------------------------------ a warp's rows, fp32
// S lanes share a row, each with PPL 16-byte pieces of it for every head; a step covers
// 32 / S rows. Per row: packed FMAs, a sum over the row's lanes that leaves each lane with
// one head's score, the probability back to all of them.
template <int D, int G>
struct Rows<float, D, G> {
  using C = Cfg<float, D, G>;
  static constexpr int S = C::S, R = C::R, PPL = C::PPL;
  static constexpr int HL = S / G;  // lanes per head after the sum
  float2 q[G][2 * PPL];             // scaled; entry j: head j ^ hq
  float2 acc[G][2 * PPL];
  float m[1], l[1];                 // of head hq over this row group's rows

  __device__ __forceinline__ void start(const PagedDecParams &p, const Walk<C::RB> &w, int lane) {
    const int sl = lane % S, hq = sl / HL;
#pragma unroll
    for (int j = 0; j < G; ++j) {
      const int head = j ^ hq;
      const float *from =
          (const float *)p.q + w.b * p.q_seq + (w.h * p.G + min(head, p.G - 1)) * p.q_head;
#pragma unroll
      for (int k = 0; k < PPL; ++k) {
        const float4 x = *reinterpret_cast<const float4 *>(from + (sl + k * S) * 4);
        const float f = head < p.G ? p.scale2 : 0.f;
        q[j][2 * k] = make_float2(x.x * f, x.y * f);
        q[j][2 * k + 1] = make_float2(x.z * f, x.w * f);
        acc[j][2 * k] = acc[j][2 * k + 1] = make_float2(0.f, 0.f);
      }
    }
    m[0] = -INFINITY;
    l[0] = 0.f;
  }

  __device__ __forceinline__ float4 piece(const uint8_t *base, int row, int pc) const {
    return *reinterpret_cast<const float4 *>(base + row * C::ROW_BYTES +
                                             ((pc ^ C::swizzle(row)) << 4));
  }

  __device__ __forceinline__ void block(const PagedDecParams &, uint8_t (*stage)[kBlockBytes],
                                        uint32_t live, int lane) {
    const int sl = lane % S, rg = lane / S;
    float sc[C::STEPS];
#pragma unroll
    for (int t = 0; t < C::STEPS; ++t) {
      const int row = t * R + rg;
      float2 d[G];
#pragma unroll
      for (int j = 0; j < G; ++j) d[j] = make_float2(0.f, 0.f);
#pragma unroll
      for (int k = 0; k < PPL; ++k) {
        const float4 x = piece(stage[0], row, sl + k * S);
#pragma unroll
        for (int j = 0; j < G; ++j) {
          d[j] = __ffma2_rn(q[j][2 * k], make_float2(x.x, x.y), d[j]);
          d[j] = __ffma2_rn(q[j][2 * k + 1], make_float2(x.z, x.w), d[j]);
        }
      }
      float v[G];
#pragma unroll
      for (int j = 0; j < G; ++j) v[j] = d[j].x + d[j].y;
      reduce_heads<S, G>(v);
      sc[t] = live >> row & 1 ? v[0] : -INFINITY;
    }
    float mb = sc[0];
#pragma unroll
    for (int t = 1; t < C::STEPS; ++t) mb = fmaxf(mb, sc[t]);
    const bool grow = mb > m[0] + kSlack;
    if (__any_sync(kAll, grow)) {
      const float mn = grow ? mb : m[0], a = grow ? fast_exp2(m[0] - mn) : 1.f;
      l[0] *= a;
      float ag[G];
      spread_heads<S, G>(a, ag);
#pragma unroll
      for (int j = 0; j < G; ++j)
#pragma unroll
        for (int e = 0; e < 2 * PPL; ++e)
          acc[j][e] = __fmul2_rn(acc[j][e], make_float2(ag[j], ag[j]));
      m[0] = mn;
    }
    const float sub = m[0] == -INFINITY ? 0.f : m[0];
#pragma unroll
    for (int t = 0; t < C::STEPS; ++t) {
      const int row = t * R + rg;
      const float w = live >> row & 1 ? fast_exp2(sc[t] - sub) : 0.f;
      l[0] += w;
      float wg[G];
      spread_heads<S, G>(w, wg);
#pragma unroll
      for (int k = 0; k < PPL; ++k) {
        const float4 x = piece(stage[1], row, sl + k * S);
#pragma unroll
        for (int j = 0; j < G; ++j) {
          const float2 ww = make_float2(wg[j], wg[j]);
          acc[j][2 * k] = __ffma2_rn(ww, make_float2(x.x, x.y), acc[j][2 * k]);
          acc[j][2 * k + 1] = __ffma2_rn(ww, make_float2(x.z, x.w), acc[j][2 * k + 1]);
        }
      }
    }
  }

  // Merge the row groups: lanes at the same place in their row group have the same head.
  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int o = S; o < 32; o <<= 1) {
      const float mo = __shfl_xor_sync(kAll, m[0], o), lo = __shfl_xor_sync(kAll, l[0], o);
      const float M = fmaxf(m[0], mo);
      const float a = m[0] == -INFINITY ? 0.f : fast_exp2(m[0] - M);
      const float b = mo == -INFINITY ? 0.f : fast_exp2(mo - M);
      l[0] = l[0] * a + lo * b;
      m[0] = M;
      float ga[G], gb[G];
      spread_heads<S, G>(a, ga);
      spread_heads<S, G>(b, gb);
#pragma unroll
      for (int j = 0; j < G; ++j)
#pragma unroll
        for (int e = 0; e < 2 * PPL; ++e) {
          float2 x;
          x.x = __shfl_xor_sync(kAll, acc[j][e].x, o);
          x.y = __shfl_xor_sync(kAll, acc[j][e].y, o);
          acc[j][e] = __ffma2_rn(acc[j][e], make_float2(ga[j], ga[j]),
                                 __fmul2_rn(x, make_float2(gb[j], gb[j])));
        }
    }
  }
  __device__ __forceinline__ void normalise() {
    float inv[G];
    spread_heads<S, G>(l[0] != 0.f ? 1.f / l[0] : 0.f, inv);  // 0: no row counts
#pragma unroll
    for (int j = 0; j < G; ++j)
#pragma unroll
      for (int e = 0; e < 2 * PPL; ++e)
        acc[j][e] = __fmul2_rn(acc[j][e], make_float2(inv[j], inv[j]));
  }
  template <typename F>
  __device__ __forceinline__ void stats(int lane, F f) {
    if (lane < S && lane % HL == 0) f(lane / HL, m[0], l[0]);
  }
  template <typename F>
  __device__ __forceinline__ void outputs(int lane, F f) {
    if (lane >= S) return;
    const int hq = lane / HL;
#pragma unroll
    for (int j = 0; j < G; ++j)
#pragma unroll
      for (int e = 0; e < 2 * PPL; ++e)
        f(j ^ hq, (lane + e / 2 * S) * 4 + e % 2 * 2, acc[j][e]);
  }
};

__device__ __forceinline__ float lse_of(float m, float l) {  // of log2 units; no row: -infinity
  return (m + log2f(l)) * 0.6931471805599453f;
}

template <typename T, int D, int G>
__global__ void __launch_bounds__(32, kWarpsPerSm)
    paged_decode_kernel(const __grid_constant__ PagedDecParams p) {
  using C = Cfg<T, D, G>;
  using W = Walk<C::RB>;
  __shared__ __align__(128) uint8_t ring[kStages][2][kBlockBytes];  // [stage][K, V]
  const int lane = threadIdx.x, run = blockIdx.x;
  pdl_wait();

  // This run: blocks of all groups, lane by lane over the sequences.
  const int per = (p.g.B + 31) / 32;
  const int b0 = min(lane * per, p.g.B), b1 = min(b0 + per, p.g.B);
  long long mine = 0;
  for (int b = b0; b < b1; ++b) {
    mine += (long long)W::blocks_of(clamp_len(p, b)) * p.g.Hkv;
    if (run == 0 && (long long)p.lens[b] > (long long)p.g.max_pages << p.g.shift)
      report(p.status, RIPPLE_EFULL);
  }
  long long incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(kAll, incl, o);
    if (lane >= o) incl += y;
  }
  const Runs runs(__shfl_sync(kAll, incl, 31), p.places, p.n_runs);
  const int rec_at = guard(run, 1, p.n_runs, p.status);
  if (run >= runs.count()) {
    if (lane == 0) p.rec[rec_at] = make_int2(0, 0);
    return;
  }
  const long long t0 = runs.start(run);
  const int owner = __ffs(__ballot_sync(kAll, incl > t0)) - 1;
  int seq = 0;
  long long rest = t0 - (incl - mine);
  if (lane == owner) {
    for (seq = b0;; ++seq) {
      const long long k = (long long)W::blocks_of(clamp_len(p, seq)) * p.g.Hkv;
      if (rest < k) break;
      rest -= k;
    }
  }
  Fetch<T, D, G> fetch;
  fetch.policy = evict_first();
  W &w = fetch.w;
  w.b = __shfl_sync(kAll, seq, owner);
  rest = __shfl_sync(kAll, rest, owner);
  w.len = clamp_len(p, w.b);
  w.h = (int)(rest / w.blocks());
  w.block = (int)(rest % w.blocks());
  w.left = runs.start(run + 1) - t0;
  w.set();
  fetch.live = true;
  fetch.at = w.begin;
  fetch.look_up(p, lane);
  W at = fetch.w;
  uint64_t coming = 0;  // live rows of the blocks on their way, 32 bits each
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i)
    coming |= (uint64_t)fetch.issue(p, ring[i], lane) << (32 * i);
  static_assert(kStages <= 3, "two blocks on their way at most");

  const long long n_rows = (long long)p.g.B * p.Hq;
  int2 rec = make_int2(0, 0);
  int stage = 0;
  long long t = t0;  // the part's first block
  for (bool more = true; more;) {
    Rows<T, D, G> rows;
    rows.start(p, at, lane);
    for (int row = at.begin; row < at.end; row += C::RB) {
      copy_wait<kStages - 2>();
      __syncwarp();  // the block has landed, and the stage before it has been read
      const uint32_t live = (uint32_t)coming;
      const int fill = stage > 0 ? stage - 1 : kStages - 1;
      coming = coming >> 32 | (uint64_t)fetch.issue(p, ring[fill], lane) << (32 * (kStages - 2));
      rows.block(p, ring[stage], live, lane);
      stage = stage + 1 < kStages ? stage + 1 : 0;
    }
    rows.finish();
    const bool ends = at.block + at.count() == at.blocks();
    if (ends && at.block == 0) {
      const long long row0 = guard((long long)at.b * p.Hq + at.h * p.G, p.G, n_rows, p.status);
      rows.normalise();
      rows.outputs(lane, [&](int head, int d, const float2 &o) {
        if (head < p.G) *reinterpret_cast<float2 *>(&p.out[(row0 + head) * D + d]) = o;
      });
      if (p.lse != nullptr)
        rows.stats(lane, [&](int head, float m, float l) {
          if (head < p.G) p.lse[row0 + head] = lse_of(m, l);
        });
    } else {
      const bool here = at.block == 0;  // the group begins in this run
      const long long slot =
          guard(2LL * run + (here ? 1 : 0), 1, 2LL * p.n_runs, p.status) * p.G;
      rows.outputs(lane, [&](int head, int d, const float2 &o) {
        if (head < p.G) *reinterpret_cast<float2 *>(&p.ws_o[(slot + head) * D + d]) = o;
      });
      rows.stats(lane, [&](int head, float m, float l) {
        if (head < p.G) p.ws_ml[slot + head] = make_float2(m, l);
      });
      if (here)
        rec = make_int2(at.b * p.g.Hkv + at.h, runs.of(t + at.blocks() - 1) - run + 1);
    }
    t += at.count();
    more = at.next(p);
  }
  copy_wait<0>();
  if (lane == 0) p.rec[rec_at] = rec;
}

// ------------------------------------------------------------ short caches
constexpr int kShortWarps = 4;
constexpr int kShortThreads = kShortWarps * 32;
constexpr int kMaxCluster = 8;
// Blocks that a warp gets at most, where the clusters leave SMs idle that runs would use, and
// where they do not. Measured (bf16, D 128, 8 KV heads, us, clusters and runs): 1 sequence with
// 4 heads a group: 470 rows 4.2 and 7.0, 2000 rows 6.6 and 8.0, 4000 rows 9.8 and 9.6, 8000 rows
// 15.8 and 11.8; 16 sequences of up to 1000 rows 10.2 and 14.0, up to 4000 rows 30.4 and 33.5;
// 64 of up to 1000 rows 32.3 and 37.5, with 8 heads a group 35.4 and 41.3, 16 heads 43.7 and 53.5.
// The clusters lose where lengths are far apart (64 of 20 to 2000 rows: 27.8 and 26.4) and where
// most warps of many groups have nothing to do (256 of up to 30 rows: 18.9 and 16.6; 150 of
// them 11.3 and 12.8).
// fp32 (blocks of 8 rows of 128 or 16 of 64), where equal lengths and few heads a group agree
// with these bounds: D 128, 8 KV heads, 4 heads a group: 1 sequence of 1000 rows 6.6 and 8.7, of
// 2000 9.1 and 10.6, of 4000 (behind the bound) 14.6 and 13.6; 9 of 4000 38.0 and 46.9, 64 of
// 1000 77.9 and 86.2, 64 of 2000 (behind it) 147.7 and 155.0. With many heads a block costs a
// warp more, and the clusters lose sooner: D 64, 16 heads a group: 1 sequence of 2000 rows 10.6
// and 9.4, of 4000 15.8 and 10.4; and where lengths are far apart: 64 of 66 to 4000 rows, 16 heads
// on one KV head, 29.5 and 21.9; 64 of 33 to 2000, 7 on each of 4, 32.1 and 25.2; 9 of which one
// has 5979 and the next 1792, 7 on each of 4, 15.7 and 14.0 (1437 and 897: 7.9 and 10.9).
constexpr int kShortFew = 8, kShortMany = 32;

template <typename T, int D, int G>
struct ShortSmem {
  struct alignas(16) Partial {  // read and written four outputs at a time
    float o[G][D];
    float2 ml[G];
  };
  static_assert(sizeof(Partial) % 16 == 0, "");
  union Ring {
    alignas(128) uint8_t stage[kStages][2][kBlockBytes];
    Partial part;  // of the warp, when its blocks are done
  };
  Ring ring[kShortWarps];
  int has[kShortWarps];  // the warp has blocks
  Partial parts[1];      // of each of the cluster's CTAs, if there are several: this one's share
  static constexpr int bytes(int ctas) {
    return (int)(sizeof(ShortSmem) - sizeof(Partial) + (ctas > 1 ? ctas * sizeof(Partial) : 0));
  }
};

__device__ __forceinline__ void axpy(float f, const float4 &x, float4 &y) {
  y.x += f * x.x;
  y.y += f * x.y;
  y.z += f * x.z;
  y.w += f * x.w;
}
// To the shared memory of a CTA of the cluster, at the place that `at` has in this one's.
__device__ __forceinline__ uint32_t in_cta(const void *at, int cta) {
  uint32_t to;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(smem_u32(at)), "r"(cta));
  return to;
}
__device__ __forceinline__ void st_cluster(uint32_t to, const float4 &v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to), "f"(v.x), "f"(v.y),
               "f"(v.z), "f"(v.w)
               : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t to, const float2 &v) {
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(v.x), "f"(v.y) : "memory");
}

template <typename T, int D, int G>
__global__ void __launch_bounds__(kShortThreads)
    paged_short_kernel(const __grid_constant__ PagedDecParams p) {
  using C = Cfg<T, D, G>;
  using W = Walk<C::RB>;
  extern __shared__ __align__(128) uint8_t smem_raw[];
  ShortSmem<T, D, G> &s = *reinterpret_cast<ShortSmem<T, D, G> *>(smem_raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int ctas = p.places, shift = __ffs(ctas) - 1;  // of the cluster, a power of two
  const int group = blockIdx.x >> shift, rank = blockIdx.x & (ctas - 1);
  pdl_wait();
  if (ctas > 1) asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  const int b = group / p.g.Hkv, h = group % p.g.Hkv;
  if (h == 0 && rank == 0 && tid == 0 &&
      (long long)p.lens[b] > (long long)p.g.max_pages << p.g.shift)
    report(p.status, RIPPLE_EFULL);
  const int len = clamp_len(p, b), blocks = W::blocks_of(len);
  const int worker = rank * kShortWarps + warp, workers = ctas * kShortWarps;
  const int first = blocks * worker / workers, last = blocks * (worker + 1) / workers;
  if (first < last) {
    Fetch<T, D, G> fetch;
    fetch.policy = evict_first();
    fetch.w.b = b;
    fetch.w.h = h;
    fetch.w.len = len;
    fetch.w.block = first;
    fetch.w.left = last - first;
    fetch.w.set();
    fetch.live = true;
    fetch.at = fetch.w.begin;
    fetch.look_up(p, lane);
    const W at = fetch.w;
    uint8_t(*ring)[2][kBlockBytes] = s.ring[warp].stage;
    uint64_t coming = 0;
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i)
      coming |= (uint64_t)fetch.issue(p, ring[i], lane) << (32 * i);
    Rows<T, D, G> rows;
    rows.start(p, at, lane);
    int stage = 0;
    for (int row = at.begin; row < at.end; row += C::RB) {
      copy_wait<kStages - 2>();
      __syncwarp();
      const uint32_t live = (uint32_t)coming;
      const int fill = stage > 0 ? stage - 1 : kStages - 1;
      coming = coming >> 32 | (uint64_t)fetch.issue(p, ring[fill], lane) << (32 * (kStages - 2));
      rows.block(p, ring[stage], live, lane);
      stage = stage + 1 < kStages ? stage + 1 : 0;
    }
    rows.finish();
    copy_wait<0>();
    __syncwarp();
    auto &part = s.ring[warp].part;
    rows.outputs(lane, [&](int head, int d, const float2 &o) {
      *reinterpret_cast<float2 *>(&part.o[head][d]) = o;
    });
    rows.stats(lane, [&](int head, float m, float l) { part.ml[head] = make_float2(m, l); });
  }
  if (lane == 0) s.has[warp] = first < last;
  __syncthreads();
  if (ctas > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");  // all of them run

  // parts[i], i < n, joined in order, column by column of four outputs (from begin to end);
  // those without rows (there(i) false) left out
  const int cols = p.G * D / 4;
  auto join = [&](int n, auto part_of, auto there, int begin, int end, auto put) {
    for (int col = begin + tid; col < end; col += kShortThreads) {
      const int head = col * 4 / D, d = col * 4 % D;
      float m = -INFINITY, den = 0.f;
      for (int i = 0; i < n; ++i)
        if (there(i)) m = fmaxf(m, part_of(i).ml[head].x);
      const float sub = m == -INFINITY ? 0.f : m;
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int i = 0; i < n; ++i) {
        if (!there(i)) continue;
        const float2 ml = part_of(i).ml[head];
        const float f = fast_exp2(ml.x - sub);
        axpy(f, *reinterpret_cast<const float4 *>(&part_of(i).o[head][d]), sum);
        den += f * ml.y;
      }
      put(col, head, d, sum, m, den);
    }
  };
  const long long row0 =
      guard((long long)b * p.Hq + h * p.G, p.G, (long long)p.g.B * p.Hq, p.status);
  auto write = [&](int, int head, int d, const float4 &o, float m, float den) {
    const float inv = den != 0.f ? 1.f / den : 0.f;  // 0: no row counts
    *reinterpret_cast<float4 *>(&p.out[(row0 + head) * D + d]) =
        make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    if (p.lse != nullptr && d == 0) p.lse[row0 + head] = lse_of(m, den);
  };
  using Partial = typename ShortSmem<T, D, G>::Partial;
  auto of_warps = [&](int i) -> const Partial & { return s.ring[i].part; };
  auto has = [&](int i) { return s.has[i] != 0; };
  if (ctas == 1) {
    join(kShortWarps, of_warps, has, 0, cols, write);
    return;
  }
  // to the CTA whose share of the columns it is; D, the padded G and ctas are powers of two
  const int share_shift = __ffs(G * D / 4) - 1 - shift;
  join(kShortWarps, of_warps, has, 0, cols,
       [&](int col, int head, int d, const float4 &o, float m, float den) {
         const int to = col >> share_shift;
         st_cluster(in_cta(&s.parts[rank].o[head][d], to), o);
         if (d == 0 || (col & ((1 << share_shift) - 1)) == 0)
           st_cluster(in_cta(&s.parts[rank].ml[head], to), make_float2(m, den));
       });
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  join(ctas, [&](int i) -> const Partial & { return s.parts[i]; },
       [](int) { return true; }, min(rank << share_shift, cols),
       min((rank + 1) << share_shift, cols), write);
}

// Joins the partials of the groups that begin in this CTA's kJoinRuns runs and go on, one
// head of the group per blockIdx.y: a group of many partials by the whole CTA, the others
// by as many warps each as there are for them. And the outputs of the sequences without
// rows.
constexpr int kJoinThreads = 256;
constexpr int kJoinWarps = kJoinThreads / 32;
constexpr int kJoinRuns = 32;
constexpr int kMany = 32;  // partials

struct Joined {
  float m, den;
  float4 sum;
  __device__ __forceinline__ void clear() {
    m = -INFINITY;
    den = 0.f;
    sum = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  __device__ __forceinline__ void scale_to(float mn) {  // a larger maximum
    const float a = fast_exp2(m - (mn == -INFINITY ? 0.f : mn));
    sum = make_float4(sum.x * a, sum.y * a, sum.z * a, sum.w * a);
    den *= a;
    m = mn;
  }
  __device__ __forceinline__ void add(float f, float l, const float4 &o) {
    sum.x += f * o.x;
    sum.y += f * o.y;
    sum.z += f * o.z;
    sum.w += f * o.w;
    den += f * l;
  }
  __device__ __forceinline__ void add(const Joined &x) {
    const float mn = fmaxf(m, x.m);
    scale_to(mn);
    add(fast_exp2(x.m - (mn == -INFINITY ? 0.f : mn)), x.den, x.sum);
  }
  // Partials first, first + step, .. of those of the group that begins in `run`.
  __device__ __forceinline__ void add_partials(const PagedDecParams &p, int D, int run, int parts,
                                               int first, int step, int head, int col) {
    constexpr int kAt = 8;  // loaded at a time
    for (int k0 = first; k0 < parts; k0 += kAt * step) {
      float2 ml[kAt];
      float4 o[kAt];
#pragma unroll
      for (int i = 0; i < kAt; ++i) {
        const int k = min(k0 + i * step, parts - 1);
        const long long slot =
            guard(2LL * (run + k) + (k == 0 ? 1 : 0), 1, 2LL * p.n_runs, p.status) * p.G + head;
        ml[i] = __ldcg(&p.ws_ml[slot]);
        o[i] = __ldcg(reinterpret_cast<const float4 *>(p.ws_o + slot * D) + col);
      }
      float mn = m;
#pragma unroll
      for (int i = 0; i < kAt; ++i) mn = fmaxf(mn, ml[i].x);  // (repeats change no maximum)
      scale_to(mn);
      const float sub = mn == -INFINITY ? 0.f : mn;
#pragma unroll
      for (int i = 0; i < kAt; ++i)
        if (k0 + i * step < parts) add(fast_exp2(ml[i].x - sub), ml[i].y, o[i]);
    }
  }
  __device__ __forceinline__ void write(const PagedDecParams &p, int D, int group, int head,
                                        int col) const {
    const long long row =
        guard((long long)(group / p.g.Hkv) * p.Hq + group % p.g.Hkv * p.G + head, 1,
              (long long)p.g.B * p.Hq, p.status);
    const float inv = den != 0.f ? 1.f / den : 0.f;  // 0: no row counts
    reinterpret_cast<float4 *>(p.out + row * D)[col] =
        make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv);
    if (p.lse != nullptr && col == 0) p.lse[row] = lse_of(m, den);
  }
};

template <int D>
__global__ void __launch_bounds__(kJoinThreads, 3)
    paged_join_kernel(const __grid_constant__ PagedDecParams p) {
  constexpr int kCols = D / 4;
  __shared__ Joined part[kJoinThreads];
  __shared__ int3 few[kJoinRuns], many[kJoinRuns];  // run, group, partials
  __shared__ int n_few, n_many;
  const int tid = threadIdx.x, warp = tid >> 5, head = blockIdx.y;
  if (tid == 0) n_few = n_many = 0;
  __syncthreads();
  pdl_wait();
  const int run = blockIdx.x * kJoinRuns + tid;
  if (tid < kJoinRuns && run < p.n_runs) {
    const int2 r = __ldcg(&p.rec[run]);
    // (listed in any order: each group is joined by itself)
    if (r.y > kMany)
      many[atomicAdd(&n_many, 1)] = make_int3(run, r.x, r.y);
    else if (r.y > 0)
      few[atomicAdd(&n_few, 1)] = make_int3(run, r.x, r.y);
  }
  __syncthreads();
  // `warps` warps a group, each stripe of D / 4 threads of them taking every stripes-th partial
  auto join = [&](const int3 *groups, int n, int warps) {
    const int stripes = warps * 32 / kCols, at_once = kJoinWarps / warps;
    const int in = tid % (warps * 32), col = in % kCols, stripe = in / kCols;
    for (int i0 = 0; i0 < n; i0 += at_once) {
      const int i = i0 + warp / warps;
      Joined j;
      j.clear();
      if (i < n) j.add_partials(p, D, groups[i].x, groups[i].z, stripe, stripes, head, col);
      if (stripes > 1) {
        part[tid] = j;
        __syncthreads();
        if (stripe == 0)
          for (int k = 1; k < stripes; ++k) j.add(part[tid + k * kCols]);
        __syncthreads();
      }
      if (i < n && stripe == 0) j.write(p, D, groups[i].y, head, col);
    }
  };
  join(many, n_many, kJoinWarps);
  join(few, n_few, n_few <= 1 ? kJoinWarps : n_few <= 2 ? 4 : n_few <= 4 ? 2 : 1);
  for (int b = blockIdx.x; b < p.g.B; b += gridDim.x) {
    if (clamp_len(p, b) > 0) continue;
    for (int e = tid; e < p.g.Hkv * D; e += kJoinThreads) {
      const long long row = guard((long long)b * p.Hq + e / D * p.G + head, 1,
                                  (long long)p.g.B * p.Hq, p.status);
      p.out[row * D + e % D] = 0.f;
      if (p.lse != nullptr && e % D == 0) p.lse[row] = -INFINITY;
    }
  }
}

// ------------------------------------------------------------ host side

// SMs of the device (cached; a repeated look-up is harmless).
int sm_count(int dev) {
  static std::atomic<int> n[kMaxDevices];
  int v = n[dev].load(std::memory_order_relaxed);
  if (v == 0) {
    cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev);
    v = v > 0 ? v : 1;
    n[dev].store(v, std::memory_order_relaxed);
  }
  return v;
}

size_t round_up(size_t x) { return (x + 255) & ~(size_t)255; }

bool decode_args(const ripple_paged_desc *d, int n_q_heads, PagedDecParams *p) {
  if (!paged_geom(d, &p->g)) return false;
  if (n_q_heads < 1 || n_q_heads % d->n_kv_heads != 0) return false;
  p->Hq = n_q_heads;
  p->G = n_q_heads / d->n_kv_heads;
  return p->G <= kMaxGroup;
}

// Runs of a call and the workspace: records, (max, sum), outputs of the partials. The runs are
// bounded by the blocks that the table has room for, so that small caches take few CTAs;
// everything grows with the call. Returns the bytes; fills p's pointers if given a base.
size_t plan(PagedDecParams *p, int dtype, int sms, void *ws) {
  const int rows = kBlockBytes / (p->g.D * (dtype == RIPPLE_BF16 ? 2 : 4));
  const long long room =
      (((long long)p->g.max_pages << p->g.shift) + rows - 1) / rows * p->g.B * p->g.Hkv;
  p->places = sms * kWarpsPerSm;
  const int phases = (long long)p->g.B * p->g.Hkv <= kFewGroups ? 1 : kPhases;
  p->n_runs = (int)std::min<long long>(phases * p->places, room);
  const size_t slots = 2 * (size_t)p->n_runs;
  const size_t rec = round_up(p->n_runs * sizeof(int2));
  const size_t ml = round_up(slots * p->G * sizeof(float2));
  uint8_t *base = (uint8_t *)ws;
  p->rec = (int2 *)base;
  p->ws_ml = (float2 *)(base + rec);
  p->ws_o = (float *)(base + rec + ml);
  return rec + ml + round_up(slots * p->G * p->g.D * sizeof(float));
}

cudaError_t launch_pdl(void (*kernel)(PagedDecParams), dim3 grid, int threads,
                       const PagedDecParams &p, cudaStream_t st, int smem = 0, int cluster = 1) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, p);
  count_launches(1);
  return e;
}

// CTAs of a group's cluster where the table's room is short, 0 where it is not: as many as
// find a place at once, and few blocks for each of their warps.
template <typename T, int D, int G>
int short_cluster(const PagedDecParams &p, int sms) {
  auto places = [&](int ctas) {  // two CTAs an SM where their shared memory has room
    return (2 * (ShortSmem<T, D, G>::bytes(ctas) + 1024) <= 228 * 1024 ? 2LL : 1LL) * sms;
  };
  const long long groups = (long long)p.g.B * p.g.Hkv;
  const long long rows = (long long)p.g.max_pages << p.g.shift;
  int ctas = 1;
  // (one CTA where its warps get a block each at most: a cluster's joins take 0.8 us; 64 rows 3.2
  // and 4.0, 8 sequences of 64 rows 3.4 and 4.3; with two blocks each 4.0 and 4.0, with three 4.7
  // and 4.0)
  if (rows > kShortWarps * Cfg<T, D, G>::RB)
    while (ctas < kMaxCluster && groups * 2 * ctas <= places(2 * ctas)) ctas *= 2;
  // of one block there is nothing to share out: runs, but for groups that all find a place
  // soon (a block each, clusters and runs: 400 groups 6.5 and 8.2 us, 1024 groups of d 64
  // 12.3 and 9.0, 2048 of d 128 18.6 and 10.5)
  if (rows <= Cfg<T, D, G>::RB && groups > 2 * places(1)) return 0;
  const int most = groups * ctas >= sms ? kShortMany : kShortFew;
  return rows <= (long long)ctas * kShortWarps * most * Cfg<T, D, G>::RB ? ctas : 0;
}

template <typename T, int D, int G>
cudaError_t launch(const PagedDecParams &p, int dev, cudaStream_t st) {
  const int ctas = short_cluster<T, D, G>(p, sm_count(dev));
  if (ctas > 0) {
    static std::atomic<bool> attr_set[kMaxDevices];
    constexpr int most = ShortSmem<T, D, G>::bytes(kMaxCluster);
    static_assert(most <= 227 * 1024, "shared memory per CTA");
    if (!attr_set[dev].load(std::memory_order_acquire)) {
      const cudaError_t e = cudaFuncSetAttribute(
          paged_short_kernel<T, D, G>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
      if (e != cudaSuccess) return e;
      attr_set[dev].store(true, std::memory_order_release);
    }
    PagedDecParams q = p;
    q.places = ctas;
    return launch_pdl(paged_short_kernel<T, D, G>, dim3(p.g.B * p.g.Hkv * ctas), kShortThreads, q,
                      st, ShortSmem<T, D, G>::bytes(ctas), ctas);
  }
  const cudaError_t e = launch_pdl(paged_decode_kernel<T, D, G>, dim3(p.n_runs), 32, p, st);
  if (e != cudaSuccess) return e;
  const int runs = (p.n_runs + kJoinRuns - 1) / kJoinRuns;
  return launch_pdl(paged_join_kernel<D>, dim3(runs, p.G), kJoinThreads, p, st);
}

// Heads of a group, padded: for the matrix instructions to 4, 8 or 16, on the CUDA
// cores to a power of two.
template <int D>
cudaError_t launch_d(const PagedDecParams &p, int dtype, int dev, cudaStream_t st) {
  if (dtype == RIPPLE_BF16) {
    if (p.G <= 4) return launch<__nv_bfloat16, D, 4>(p, dev, st);
    if (p.G <= 8) return launch<__nv_bfloat16, D, 8>(p, dev, st);
    return launch<__nv_bfloat16, D, 16>(p, dev, st);
  }
  if (p.G == 1) return launch<float, D, 1>(p, dev, st);
  if (p.G == 2) return launch<float, D, 2>(p, dev, st);
  if (p.G <= 4) return launch<float, D, 4>(p, dev, st);
  if (p.G <= 8) return launch<float, D, 8>(p, dev, st);
  return launch<float, D, 16>(p, dev, st);
}

}  // namespace
}  // namespace ripple

using namespace ripple;

extern "C" ripple_status ripple_paged_decode_workspace_bytes(const ripple_paged_desc *desc,
                                                             int32_t n_q_heads,
                                                             size_t *bytes_host) {
  PagedDecParams p;
  if (!decode_args(desc, n_q_heads, &p) || bytes_host == nullptr) return RIPPLE_EINVAL;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) dev = 0;
  *bytes_host = plan(&p, desc->dtype, sm_count(dev), nullptr);
  return RIPPLE_OK;
}

extern "C" ripple_status ripple_paged_decode_attn(
    const ripple_paged_desc *desc, int32_t n_q_heads, float scale, const void *q,
    const ripple_token_strides *q_strides, const void *k_pages, const void *v_pages,
    const int32_t *block_table, const int32_t *lens, float *out, float *lse, void *workspace,
    size_t workspace_bytes, int32_t *dev_status, void *stream) {
  PagedDecParams p;
  if (!decode_args(desc, n_q_heads, &p)) return RIPPLE_EINVAL;
  if (!(scale >= 0.f) || scale > kMaxScale) return RIPPLE_EINVAL;
  if (!q || !k_pages || !v_pages || !block_table || !lens || !out || !workspace ||
      ((uintptr_t)workspace & 255u))
    return RIPPLE_EINVAL;
  if (!aligned16_host(q) || !aligned16_host(k_pages) || !aligned16_host(v_pages) ||
      !aligned16_host(out) || !aligned4_host({block_table, lens, lse, dev_status}))
    return RIPPLE_EINVAL;
  const int vec = vec_elems(desc->dtype);
  p.q_head = desc->head_dim;
  p.q_seq = (long long)n_q_heads * desc->head_dim;
  if (q_strides != nullptr) {
    p.q_seq = q_strides->seq_stride;
    p.q_head = q_strides->head_stride;
    if (p.q_seq < 0 || p.q_head < 0 || p.q_seq > (1LL << 40) || p.q_head > (1LL << 40) ||
        p.q_seq % vec != 0 || p.q_head % vec != 0)
      return RIPPLE_EINVAL;
  }
  int dev = 0;
  const cudaError_t got = cudaGetDevice(&dev);
  if (got != cudaSuccess || dev < 0 || dev >= kMaxDevices) dev = 0;
  if (workspace_bytes < plan(&p, desc->dtype, sm_count(dev), workspace)) return RIPPLE_EWORKSPACE;
  if (got != cudaSuccess) return RIPPLE_ECUDA;
  p.scale2 = (scale > 0.f ? scale : 1.0f / sqrtf((float)desc->head_dim)) * kLog2e;
  p.q = q;
  p.k_pages = k_pages;
  p.v_pages = v_pages;
  p.table = block_table;
  p.lens = lens;
  p.out = out;
  p.lse = lse;
  p.status = dev_status;
  cudaStream_t st = (cudaStream_t)stream;
  RIPPLE_CUDA_TRY(desc->head_dim == 128 ? launch_d<128>(p, desc->dtype, dev, st)
                                        : launch_d<64>(p, desc->dtype, dev, st));
  return RIPPLE_OK;
}
