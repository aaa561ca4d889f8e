// ripple_token_logprobs: log probabilities of given tokens, entropies and the most
// likely alternatives, from logits over the vocabulary, read from HBM once.
//
// With m the row's largest logit, d = x - m, w = exp(scale d), S' the sum of w over the
// row without one largest logit (whose w is 1) and T the sum of w d:
//   log P(x) = scale d - log1p(S'),   entropy = log1p(S') - scale T / (1 + S').
// Leaving the 1 out of the sum keeps the relative precision of log probabilities near 0.
// With y = scale d log2 e, w |y| is at most 0.54, so T stays below 0.54 V / (scale log2 e):
// in fp32 down to scales of kScaleOfD. Below, and for fp32 logits at every scale, T is the
// sum of w y and its factor ln 2. (For bf16 that costs 3%: 2048 rows of 128256 82.6 us, 85.2.)
//
// Work: one CTA of eight warps per row (of two for many short rows, launch_width), or with few
// rows one per slice of a row, the slices of a row being a cluster (slices_of). Every thread
// copies its 16-byte vectors of the row into places of its own in shared memory, kStages
// chunks ahead (asynchronous copies, waited for by the thread alone), so that the loads in
// flight cost no registers and no barrier. A warp keeps a maximum, which begins as the
// largest logit of the CTA's first chunk and so rarely moves (a vote per chunk), and sums
// per lane. The warps are merged through shared memory, the slices through the shared
// memory of the cluster's first CTA.
//
// Alternatives: keys order logits descending, equal ones by index. The n-th largest of the
// largest logits of kGroups groups of lanes bounds the slice's n-th largest key from below
// (64 groups and not 32: with 32 alternatives, the least of 32 groups' largest leaves three
// times as many candidates; 138 and 109 us for 2048 rows of 128256).
// The largest logit of every lane and segment of the slice (a few chunks) has been kept,
// so only the segments that reach the bound are read once more (from the ring if they are
// its last chunks, from L2 mostly if not), and the candidates, a few more than n, are
// ranked by counting. Where there are more than fit (many ties, sorted rows), the n-th
// largest of those found is a higher bound, and the reading is repeated with it; every turn
// drops some.
//
// Bound: 2048 rows of 128256, bf16: HBM (77 us of 84 without alternatives, 92 with one), and
// the issue slots close behind (two thirds taken; the exponentials take a third of their
// units' time). Many short rows: the instructions that a row costs once (about as many as 14000
// tokens by eight warps). Few rows: the chain of loads, joins and a cluster's barriers.
#include <float.h>
#include <math.h>

#include <atomic>

#include "common.cuh"
#include "kernels.cuh"

namespace ripple {
namespace {

constexpr int kWarpsPerSm = 24;
constexpr int kWide = 8, kNarrow = 2;  // warps of a CTA
constexpr int kPlaces = 152 * kWarpsPerSm / kWide;
constexpr int kMaxSlices = 8;
constexpr int kVecs = 4;               // 16-byte vectors of a thread in a chunk
constexpr int kStages = 3;
constexpr int kSegments = 8;
constexpr int kGroups = 64;            // of lanes, whose largest logits bound the alternatives
constexpr float kScaleOfD = 1e-29f;    // of the scale in base 2 (2^30 * 0.54 / 1e-29 < 2^127)
constexpr unsigned kAll = 0xffffffffu;
constexpr int kMaxDevices = 64;
typedef unsigned long long Key;

struct Scale {
  float two;    // scale * log2 e
  float of_t;   // factor of T: scale where it sums w d, ln 2 where w y
  bool sums_y;
};

struct LogprobParams {
  const void *logits;
  long long row_stride;
  int n_rows, vocab, n_top, slices;
  float scale;
  Scale by;
  const int32_t *tokens;
  float *logprob, *entropy, *lse;
  int32_t *top_idx;
  float *top_logprob;
  int32_t *status;
};

// Descending logits, then ascending indices, as one descending key; -0 ties with 0, and
// what is no number comes first.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return x != x ? 0xffffffffu : u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ Key key_of(float x, int i) { return (Key)order_of(x) << 32 | (uint32_t)~i; }

// Part of a row: a logit m at least as large as all of its logits, the sum of the terms
// relative to it, 1 for one logit m if it is in the part (one) and s for all others, and T.
struct Sums {
  float m, s, t, one;
};
// A sum n of terms relative to m_from, and its t, to a larger m.
__device__ __forceinline__ void rebase(float n, float &t, float &s, float m_from, float m,
                                       const Scale &by) {
  const float d = m_from == -INFINITY ? 0.f : fmaxf(m_from - m, -FLT_MAX), y = d * by.two;
  const float e = fast_exp2(y);
  t = e > 0.f ? e * (t + n * (by.sums_y ? y : d)) : 0.f;
  s = n * e;
}
__device__ __forceinline__ Sums merge(const Sums &a, const Sums &b, const Scale &by) {
  const bool first = a.m > b.m || (a.m == b.m && a.one >= b.one);
  const Sums &hi = first ? a : b, &lo = first ? b : a;
  float s, t = lo.t;
  rebase(lo.one + lo.s, t, s, lo.m, hi.m, by);
  return Sums{hi.m, hi.s + s, hi.t + t, hi.one};
}

// The largest of the warp's values (the others if some are no numbers).
__device__ __forceinline__ float warp_max(float v) {
  float r;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}

// The logits of a 16-byte vector: as floats, their largest, and with the first that equals
// `v` made -infinity (true if there is one).
__device__ __forceinline__ void unpack16(const uint4 &u, const float *, float *x) {
  x[0] = __uint_as_float(u.x);
  x[1] = __uint_as_float(u.y);
  x[2] = __uint_as_float(u.z);
  x[3] = __uint_as_float(u.w);
}
__device__ __forceinline__ void unpack16(const uint4 &u, const __nv_bfloat16 *, float *x) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ float max16(const uint4 &u) {  // of four floats
  return fmaxf(fmaxf(__uint_as_float(u.x), __uint_as_float(u.y)),
               fmaxf(__uint_as_float(u.z), __uint_as_float(u.w)));
}
__device__ __forceinline__ uint32_t max_pairs(uint32_t a, uint32_t b) {  // of two bf16 each
  uint32_t r;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ float larger(uint32_t pair) {
  return fmaxf(__uint_as_float(pair << 16), __uint_as_float(pair & 0xffff0000u));
}
// Infinite masks as the lowest bf16, NaN left.
__device__ __forceinline__ uint32_t finite(uint32_t pair) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(pair), "r"(0xff7fff7fu));
  return r;
}
__device__ __forceinline__ bool take(uint32_t &w, float v, const float *) {
  const bool is = __uint_as_float(w) == v;
  if (is) w = 0xff800000u;
  return is;
}
__device__ __forceinline__ bool take(uint32_t &w, float v, const __nv_bfloat16 *) {
  const bool low = __uint_as_float(w << 16) == v;
  const bool high = !low && __uint_as_float(w & 0xffff0000u) == v;
  if (low) w = (w & 0xffff0000u) | 0xff80u;
  if (high) w = (w & 0xffffu) | 0xff800000u;
  return low || high;
}
template <typename T>
__device__ __forceinline__ bool take16(uint4 &u, float v, const T *type) {
  return take(u.x, v, type) || take(u.y, v, type) || take(u.z, v, type) || take(u.w, v, type);
}
__device__ __forceinline__ uint4 none16(const float *) {  // a vector of -infinity
  return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u);
}
__device__ __forceinline__ uint4 none16(const __nv_bfloat16 *) {
  return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u);
}

// A row as vectors of 16 bytes: vector v holds elements v * E - lead .. , of which only
// those in [0, vocab) are the row's (the first and the last vector may be partial).
template <typename T>
struct Row {
  static constexpr int E = 16 / (int)sizeof(T);
  const T *x;
  int lead, vocab, n_vec;
  __device__ __forceinline__ Row(const LogprobParams &p, int row) {
    x = (const T *)p.logits + row * p.row_stride;
    lead = (int)(((uintptr_t)x & 15u) / sizeof(T));
    vocab = p.vocab;
    n_vec = (int)(((long long)vocab + lead + E - 1) / E);
  }
  __device__ __forceinline__ int first(int v) const { return v * E - lead; }
  __device__ __forceinline__ bool whole(int v) const {
    return first(v) >= 0 && first(v) + E <= vocab;
  }
  __device__ __forceinline__ uint4 load(int v) const {
    return __ldcg(reinterpret_cast<const uint4 *>(x + first(v)));
  }
  // A partial vector as it would lie there, -infinity where the row has no element.
  __device__ __forceinline__ uint4 get_raw(int v) const {
    return make_uint4(word(v, 0), word(v, 1), word(v, 2), word(v, 3));
  }
  __device__ __forceinline__ uint32_t word(int v, int w) const {
    uint32_t r = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
#pragma unroll
    for (int e = 0; e < E / 4; ++e) {
      const int i = first(v) + w * (E / 4) + e;
      if (i < 0 || i >= vocab) continue;
      if (sizeof(T) == 4)
        r = reinterpret_cast<const uint32_t *>(x)[i];
      else
        r = e == 0 ? (r & 0xffff0000u) | reinterpret_cast<const uint16_t *>(x)[i]
                   : (r & 0xffffu) | (uint32_t)reinterpret_cast<const uint16_t *>(x)[i] << 16;
    }
    return r;
  }
  // Elements of any vector; -infinity where the row has none.
  __device__ __forceinline__ void get(int v, float (&y)[E]) const {
    if (whole(v)) {
      unpack16(load(v), x, y);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int i = first(v) + e;
        y[e] = i >= 0 && i < vocab ? to_f32(x[i]) : -INFINITY;
      }
    }
  }
};

// A lane's part of the warp's running sums. m is the same on every lane; the lane that
// `owns` a logit m has left it out of its s. m begins as the largest logit of the CTA's
// first chunk, so that it rarely moves.
template <typename T>
struct Lane {
  float m, top = -INFINITY;  // of the warp, and this lane's own largest
  float2 s = make_float2(0.f, 0.f), t = make_float2(0.f, 0.f);
  bool owns = false;

  template <int N>
  static __device__ __forceinline__ float largest(const uint4 (&u)[N]) {
    if (sizeof(T) == 2) {
      uint32_t g = max_pairs(max_pairs(u[0].x, u[0].y), max_pairs(u[0].z, u[0].w));
#pragma unroll
      for (int i = 1; i < N; ++i)
        g = max_pairs(g, max_pairs(max_pairs(u[i].x, u[i].y), max_pairs(u[i].z, u[i].w)));
      return larger(g);
    }
    float g = max16(u[0]);
#pragma unroll
    for (int i = 1; i < N; ++i) g = fmaxf(g, max16(u[i]));
    return g;
  }
  // The first lane that has a logit m takes it out of u, its largest being g.
  template <int N>
  __device__ __forceinline__ void own(uint4 (&u)[N], float g, int lane) {
    owns = lane == __ffs(__ballot_sync(kAll, g == m)) - 1;
    if (owns) {
      const T *type = nullptr;
      bool taken = false;
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (!taken) taken = take16(u[i], m, type);
    }
  }
  // N vectors of every lane, this lane's largest being g.
  template <int N>
  __device__ __forceinline__ void add(uint4 (&u)[N], float g, const Scale &by, int lane) {
    if (__any_sync(kAll, g > m)) {
      const float mn = warp_max(g);
      float ss, tt = t.x + t.y;
      rebase(s.x + s.y + (owns ? 1.f : 0.f), tt, ss, m, mn, by);
      s = make_float2(ss, 0.f);
      t = make_float2(tt, 0.f);
      m = mn;
      own(u, g, lane);
    }
    // bf16 is made finite two at a time, where the lowest bf16 relative to m is finite and has no
    // weight (2048 rows of 128256: 83.6 us, 85.1 logit by logit); else, and fp32, d logit by logit
    if (sizeof(T) == 2 && fabsf(m) <= 1e36f && !by.sums_y)
      terms<true>(u, by);
    else
      terms<false>(u, by);
  }
  template <bool kFinite, int N>
  __device__ __forceinline__ void terms(const uint4 (&u)[N], const Scale &by) {
    constexpr int E = 16 / (int)sizeof(T);
    const T *type = nullptr;
    const float m0 = fmaxf(m, -FLT_MAX);  // nothing but -infinity so far: w = 0
    const float2 minus = make_float2(-m0, -m0), c = make_float2(by.two, by.two);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float x[E];
      unpack16(kFinite ? make_uint4(finite(u[i].x), finite(u[i].y), finite(u[i].z), finite(u[i].w))
                       : u[i],
               type, x);
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        float2 d = __fadd2_rn(make_float2(x[e], x[e + 1]), minus);
        const float2 y = __fmul2_rn(d, c);
        const float2 w = make_float2(fast_exp2(y.x), fast_exp2(y.y));
        s = __fadd2_rn(s, w);
        if (!kFinite) {
          if (sizeof(T) == 4 || by.sums_y) d = y;
          d.x = fmaxf(d.x, -FLT_MAX);  // 0 times -infinity is no term
          d.y = fmaxf(d.y, -FLT_MAX);
        }
        t = __ffma2_rn(w, d, t);
      }
    }
  }
};

template <int W>
struct Smem {
  static constexpr int kThreads = W * 32;
  static constexpr int kCands = W * 64;  // candidates ranked at a time
  uint4 ring[kStages][kVecs][kThreads];
  float seg[kSegments][kThreads];  // largest logit of a segment's lane
  Key cand[kCands];
  // n_top of every slice, in the cluster's first CTA
  Key best[(W == kWide ? kMaxSlices : 1) * RIPPLE_MAX_TOP];
  Sums sums[kMaxSlices], warp[W];
  float first[W];
  alignas(16) uint32_t group[kGroups];  // largest logits, as order_of
  float2 done;                          // of the row: its largest logit, log1p(S')
  uint16_t hot[W][kSegments * 32];   // segment * 32 + lane
  Key kth;
  int n_cand;
};

__device__ __forceinline__ void copy16(void *dst, const void *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src)
               : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Ranks `n` keys by counting: f(rank, key) for each; equal keys (0: none) share a rank.
template <int W, typename F>
__device__ __forceinline__ void rank_keys(const Key *keys, int n, F f) {
  for (int i = threadIdx.x; i < n; i += W * 32) {
    const Key k = keys[i];
    int rank = 0;
#pragma unroll 4
    for (int j = 0; j < n; ++j) rank += keys[j] > k;
    f(rank, k);
  }
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_arrive() {
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}
// `p` of this CTA's shared memory, in the cluster's first CTA.
__device__ __forceinline__ uint32_t in_first(const void *p) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(smem_u32(p)));
  return r;
}
__device__ __forceinline__ void st_cluster(uint32_t at, Key v) {
  asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(at), "l"(v) : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t at, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(v) : "memory");
}

// A CTA's slice of a row: vectors [v0, v1), of which [w0, w1) are whole and come through
// the ring, chunk by chunk.
template <typename T>
struct Slice {
  int v0, v1, w0, w1;
  __device__ __forceinline__ Slice(const Row<T> &row, int slice, int slices) {
    const int each = row.n_vec >> (__ffs(slices) - 1);  // (a power of two) the last has the rest
    v0 = each * slice;
    v1 = slice + 1 < slices ? v0 + each : row.n_vec;
    w0 = v0 + (v0 < v1 && !row.whole(v0) ? 1 : 0);
    w1 = max(w0, v1 - (v0 < v1 && !row.whole(v1 - 1) ? 1 : 0));
  }
  __device__ __forceinline__ int chunks(int vecs) const { return (w1 - w0 + vecs - 1) / vecs; }
  // The partial vectors: the first, the last, or -1.
  __device__ __forceinline__ int partial(int which) const {
    return which == 0 ? (w0 > v0 ? v0 : -1) : (v1 > w1 ? v1 - 1 : -1);
  }
};

// The Sums of lanes 0 .. n - 1, n <= 8, merged in a fixed order; on every lane.
__device__ __forceinline__ Sums merge_lanes(Sums a, int n, int lane, const Scale &by) {
  if (lane >= n) a = Sums{-INFINITY, 0.f, 0.f, 0.f};
#pragma unroll
  for (int o = 1; o < 8; o *= 2) {
    const Sums b{__shfl_xor_sync(kAll, a.m, o), __shfl_xor_sync(kAll, a.s, o),
                 __shfl_xor_sync(kAll, a.t, o), __shfl_xor_sync(kAll, a.one, o)};
    a = lane & o ? merge(b, a, by) : merge(a, b, by);
  }
  return Sums{__shfl_sync(kAll, a.m, 0), __shfl_sync(kAll, a.s, 0), __shfl_sync(kAll, a.t, 0),
              __shfl_sync(kAll, a.one, 0)};
}

template <typename T, int W>
__global__ void __launch_bounds__(W * 32, kWarpsPerSm / W)
    logprob_kernel(const __grid_constant__ LogprobParams p) {
  extern __shared__ __align__(128) uint8_t smem_raw[];
  Smem<W> &s = *reinterpret_cast<Smem<W> *>(smem_raw);
  constexpr int kThreads = W * 32, kChunkVecs = kThreads * kVecs, kCands = Smem<W>::kCands;
  constexpr int kGroup = kThreads / kGroups;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const bool many = W == kWide && p.slices > 1;
  const int slice = many ? (int)cluster_rank() : 0, r = blockIdx.x / p.slices;
  const int n_top = p.n_top;
  pdl_wait();
  if (many) cluster_arrive();  // waited for before the first CTA's memory is written

  const Row<T> row(p, r);
  const Slice<T> part(row, slice, p.slices);
  const int chunks = part.chunks(kChunkVecs);
  auto fetch = [&](int c, int stage) {  // chunk c; the thread's vectors behind w1 are none
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int v = part.w0 + c * kChunkVecs + i * kThreads + tid;
      if (v < part.w1)
        copy16(&s.ring[stage][i][tid],
               row.x + row.first((int)guard(v, 1, row.n_vec, p.status)));
    }
  };
#pragma unroll
  for (int c = 0; c < kStages - 1; ++c) {
    if (c < chunks) fetch(c, c);
    copy_commit();
  }
  // the given token's logit, on its way while the row is read (the warp that writes it)
  float given = 0.f;
  int token = -1;
  if (slice == 0 && warp == W - 1 && p.tokens != nullptr) {
    token = p.tokens[r];
    if (token >= 0 && token < p.vocab) given = to_f32(row.x[token]);
  }
  if (tid == 0) s.n_cand = 0;

  Lane<T> sum;
  sum.m = -INFINITY;
  float largest = -INFINITY;                                 // of this lane
  const int per_seg = (chunks + kSegments - 1) / kSegments;  // chunks of a segment
  int seg = 0, in_seg = 0, stage = 0;
  for (int c = 0; c < chunks; ++c) {
    copy_wait<kStages - 2>();
    uint4 u[kVecs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) u[i] = s.ring[stage][i][tid];
    if (part.w1 - part.w0 - c * kChunkVecs < kChunkVecs) {  // the last chunk
#pragma unroll
      for (int i = 0; i < kVecs; ++i)
        if (part.w0 + c * kChunkVecs + i * kThreads + tid >= part.w1) u[i] = none16(row.x);
    }
    // (into the stage read in the turn before, by this thread alone)
    if (c + kStages - 1 < chunks) fetch(c + kStages - 1, stage > 0 ? stage - 1 : kStages - 1);
    copy_commit();
    stage = stage + 1 < kStages ? stage + 1 : 0;
    const float g = Lane<T>::largest(u);
    sum.top = fmaxf(sum.top, g);
    if (c == 0) {
      const float mine = warp_max(g);
      if (lane == 0) s.first[warp] = mine;
      __syncthreads();
      const float of = lane < W ? s.first[lane] : -INFINITY;
      sum.m = warp_max(of);
      // the first warp that has it owns a logit
      const int owner = __ffs(__ballot_sync(kAll, lane < W && of == sum.m)) - 1;
      if (sum.m > -INFINITY && warp == owner) sum.own(u, g, lane);
    }
    sum.add(u, g, p.by, lane);
    if (++in_seg == per_seg || c == chunks - 1) {  // the segment's end
      s.seg[seg++][tid] = sum.top;
      largest = fmaxf(largest, sum.top);
      sum.top = -INFINITY;
      in_seg = 0;
    }
  }
  if (warp == 0 && (part.partial(0) >= 0 || part.partial(1) >= 0)) {
    uint4 x[1] = {none16(row.x)};
    if (lane < 2 && part.partial(lane) >= 0) x[0] = row.get_raw(part.partial(lane));
    const float g = Lane<T>::largest(x);
    largest = fmaxf(largest, g);  // (looked at apart from the segments)
    sum.add(x, g, p.by, lane);
  }

  // the warp, the slice
  {
    float ss = sum.s.x + sum.s.y, tt = sum.t.x + sum.t.y;
    const bool one = __any_sync(kAll, sum.owns);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      ss += __shfl_xor_sync(kAll, ss, o);
      tt += __shfl_xor_sync(kAll, tt, o);
    }
    if (lane == 0) s.warp[warp] = Sums{sum.m, ss, tt, one ? 1.f : 0.f};
  }
  float g = largest;
#pragma unroll
  for (int o = kGroup / 2; o > 0; o >>= 1) g = fmaxf(g, __shfl_xor_sync(kAll, g, o));
  if (lane % kGroup == 0) s.group[tid / kGroup] = order_of(g);
  __syncthreads();

  // Writes a row's outputs but the alternatives (a warp); its largest logit and log1p(S').
  auto write = [&](Sums all) {
    if (all.m == INFINITY) all.s = NAN;
    all.s -= 1.f - all.one;  // S' (no logit but -infinity: -1)
    const float ls = log1pf(all.s);
    if (lane == 0) {
      if (p.lse != nullptr)
        p.lse[r] = all.m == -INFINITY ? all.m + 0.f * all.s : p.scale * all.m + ls;
      if (p.entropy != nullptr) p.entropy[r] = ls - p.by.of_t * all.t / (1.f + all.s);
      if (p.logprob != nullptr) {
        float y = 0.f;
        if (token >= p.vocab) {
          report(p.status, RIPPLE_EBOUNDS);
          y = NAN;
        } else if (token >= 0) {
          y = p.scale * (given - all.m) - ls;
        }
        p.logprob[r] = y;
      }
      s.done = make_float2(all.m, ls);
    }
  };
  if (warp == W - 1) {
    const Sums all = merge_lanes(s.warp[lane % W], W, lane, p.by);
    if (!many)
      write(all);
    else if (lane == 0)
      s.sums[slice] = all;
  }

  if (n_top > 0) {
    // the n-th largest of the groups' largest logits, a group's threads a part of them each
    {
      constexpr int kOthers = kGroups / kGroup / 4;
      const uint32_t o = s.group[tid / kGroup];
      int above = 0, same = 0;
#pragma unroll
      for (int i = 0; i < kOthers; ++i) {
        const uint4 x = reinterpret_cast<const uint4 *>(s.group)[tid % kGroup * kOthers + i];
        above += (x.x > o) + (x.y > o) + (x.z > o) + (x.w > o);
        same += (x.x == o) + (x.y == o) + (x.z == o) + (x.w == o);
      }
#pragma unroll
      for (int i = 1; i < kGroup; i *= 2) {
        above += __shfl_xor_sync(kAll, above, i);
        same += __shfl_xor_sync(kAll, same, i);
      }
      // (groups with the same value all write it)
      if (above < n_top && above + same >= n_top) s.kth = (Key)o << 32;
    }
    __syncthreads();
    Key bound = s.kth;
    // the warp's lanes' segments with candidates
    int n_hot = 0;
    if (__any_sync(kAll, (Key)order_of(largest) << 32 >= bound))
      for (int i = 0; i < seg; ++i) {
        const bool is = (Key)order_of(s.seg[i][tid]) << 32 >= bound;
        const unsigned all = __ballot_sync(kAll, is);
        if (is) s.hot[warp][n_hot + __popc(all & ((1u << lane) - 1))] = (uint16_t)(i * 32 + lane);
        n_hot += __popc(all);
      }
    __syncwarp();
    const int per = per_seg * kVecs;  // vectors of one, at most
    for (;;) {
      auto look = [&](int v, const float (&x)[Row<T>::E]) {
#pragma unroll
        for (int e = 0; e < Row<T>::E; ++e) {
          const int idx = row.first(v) + e;
          const Key k = key_of(x[e], idx);
          if (k >= bound && idx >= 0 && idx < p.vocab) {
            const int at = atomicAdd(&s.n_cand, 1);
            if (at < kCands) s.cand[at] = k;
          }
        }
      };
      for (int i = lane; i < n_hot * per; i += 32) {
        const int hot = s.hot[warp][i / per];
        const int at = hot / 32 * per + i % per, of = warp * 32 + hot % 32;
        const int v = part.w0 + at * kThreads + of;
        if (v >= part.w1) continue;
        float x[Row<T>::E];
        const int back = chunks - at / kVecs;
        if (back <= kStages)  // still in the ring
          unpack16(s.ring[(stage + kStages - back) % kStages][at % kVecs][of], row.x, x);
        else
          unpack16(row.load((int)guard(v, 1, row.n_vec, p.status)), row.x, x);
        look(v, x);
      }
      if (tid < 2 && part.partial(tid) >= 0) {
        float x[Row<T>::E];
        row.get(part.partial(tid), x);
        look(part.partial(tid), x);
      }
      __syncthreads();
      if (s.n_cand <= kCands) break;
      // too many: a higher bound from those found
      rank_keys<W>(s.cand, kCands, [&](int rank, Key k) {
        if (rank == n_top - 1) s.kth = k;
      });
      __syncthreads();
      bound = s.kth;
      if (tid == 0) s.n_cand = 0;
      __syncthreads();
    }
  }
  const Key *keys = s.cand;
  int n_keys = n_top > 0 ? s.n_cand : 0;
  if (many) {
    cluster_wait();  // the first CTA runs
    if (n_top > 0) {
      const uint32_t to = in_first(s.best + slice * n_top);
      rank_keys<W>(keys, n_keys, [&](int rank, Key k) {
        if (rank < n_top) st_cluster(to + rank * 8, k);
      });
      if (tid >= n_keys && tid < n_top) st_cluster(to + tid * 8, (Key)0);
    }
    if (warp == W - 1 && lane == 0 && slice > 0) {
      const Sums all = s.sums[slice];
      const uint32_t to = in_first(&s.sums[slice]);
      st_cluster(to, all.m);
      st_cluster(to + 4, all.s);
      st_cluster(to + 8, all.t);
      st_cluster(to + 12, all.one);
    }
    cluster_arrive();
    cluster_wait();
    if (slice != 0) return;
    if (warp == W - 1) write(merge_lanes(s.sums[lane % kMaxSlices], p.slices, lane, p.by));
    keys = s.best;
    n_keys = p.slices * n_top;
    __syncthreads();
  }
  rank_keys<W>(keys, n_keys, [&](int rank, Key k) {
    if (rank >= n_top) return;
    const long long to =
        guard((long long)r * n_top + rank, 1, (long long)p.n_rows * n_top, p.status);
    p.top_idx[to] = (int)~(uint32_t)k;
    if (p.top_logprob != nullptr)
      p.top_logprob[to] = p.scale * (value_of((uint32_t)(k >> 32)) - s.done.x) - s.done.y;
  });
}

// Slices of a row: as many CTAs as find a place at once, of a chunk at least. More would come to
// a second turn: 333 rows of 32003, fp32, in halves 14.6 us, whole 10.6. Rows of four chunks at
// most stay whole, since a cluster costs more than it saves (a row of 36 KB 3.7 us, in halves
// 4.4; of 72 KB, bf16, 5.1, in quarters 4.6).
int slices_of(int n_rows, long long row_bytes) {
  constexpr long long kChunk = kWide * 32 * kVecs * 16;
  int c = 1;
  if (row_bytes <= 4 * kChunk) return c;
  while (c < kMaxSlices && (long long)n_rows * 2 * c <= kPlaces && row_bytes >= 2 * c * kChunk)
    c *= 2;
  return c;
}

template <typename T, int W>
cudaError_t launch(const LogprobParams &p, int dev, cudaStream_t st) {
  static std::atomic<bool> attr_set[kMaxDevices];
  static_assert(kWarpsPerSm / W * (sizeof(Smem<W>) + 1024) <= 228 * 1024,
                "shared memory per SM");
  if (!attr_set[dev].load(std::memory_order_acquire)) {
    const cudaError_t e = cudaFuncSetAttribute(
        logprob_kernel<T, W>, cudaFuncAttributeMaxDynamicSharedMemorySize,
        (int)sizeof(Smem<W>));
    if (e != cudaSuccess) return e;
    attr_set[dev].store(true, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.n_rows * p.slices);
  cfg.blockDim = dim3(W * 32);
  cfg.dynamicSmemBytes = sizeof(Smem<W>);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = p.slices;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.slices > 1 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, logprob_kernel<T, W>, p);
  count_launches(1);
  return e;
}

// Two warps a row where there are more rows than wide CTAs find a place and rows are short: what
// a CTA does once per row (sums joined, alternatives) costs eight warps four times as much,
// but as many two find too little to read ahead of long rows, and leave SMs idle at the end.
// Measured (no alternatives, us, two and eight warps): bf16, 14562 tokens: 460 rows 7.7 and 8.0,
// 2874 rows 23.8 and 33.9; 60000 tokens: 460 rows 17.5 and 16.4, 2874 rows 62 and 67; 128256
// tokens: 1000 rows 48.7 and 46.5, 2000 rows 98 and 84; fp32, 4000 tokens: 2000 rows 9.5 and 13.9,
// 45864 tokens: 2000 rows 77.5 and 62.6.
template <typename T>
cudaError_t launch_width(const LogprobParams &p, long long row_bytes, int dev, cudaStream_t st) {
  return p.n_rows > kPlaces && row_bytes <= 128 * 1024 ? launch<T, kNarrow>(p, dev, st)
                                                       : launch<T, kWide>(p, dev, st);
}

}  // namespace
}  // namespace ripple

using namespace ripple;

extern "C" ripple_status ripple_token_logprobs(
    int32_t n_rows, int32_t vocab, int64_t row_stride, int32_t dtype, float scale, int32_t n_top,
    const void *logits, const int32_t *tokens, float *logprob_out, float *entropy_out,
    float *lse_out, int32_t *top_idx_out, float *top_logprob_out, int32_t *dev_status,
    void *stream) {
  if (n_rows < 0 || n_rows > (1 << 27) || vocab < 1 || vocab > (1 << 30) || row_stride < 0 ||
      row_stride > (1LL << 40))
    return RIPPLE_EINVAL;
  if (dtype != RIPPLE_F32 && dtype != RIPPLE_BF16) return RIPPLE_EINVAL;
  if (!(scale >= 0.f) || scale > kMaxScale) return RIPPLE_EINVAL;
  if (n_top < 0 || n_top > RIPPLE_MAX_TOP || n_top > vocab) return RIPPLE_EINVAL;
  if ((tokens == nullptr) != (logprob_out == nullptr)) return RIPPLE_EINVAL;
  if (n_rows == 0) return RIPPLE_OK;
  if (logits == nullptr || (n_top > 0) != (top_idx_out != nullptr) ||
      (n_top == 0 && top_logprob_out != nullptr))
    return RIPPLE_EINVAL;
  if (((uintptr_t)logits & (dtype == RIPPLE_F32 ? 3u : 1u)) != 0) return RIPPLE_EINVAL;
  for (const void *o : {(const void *)tokens, (const void *)logprob_out, (const void *)entropy_out,
                        (const void *)lse_out, (const void *)top_idx_out,
                        (const void *)top_logprob_out, (const void *)dev_status})
    if ((uintptr_t)o & 3u) return RIPPLE_EINVAL;
  const float sc = scale > 0.f ? scale : 1.f;
  const long long row_bytes = (long long)vocab * (dtype == RIPPLE_F32 ? 4 : 2);
  const int slices = slices_of(n_rows, row_bytes);
  const float two = sc * kLog2e;
  const bool sums_y = dtype == RIPPLE_F32 || two < kScaleOfD;
  const Scale by{two, sums_y ? 0.6931471805599453f : sc, sums_y};
  const LogprobParams p{logits, row_stride, n_rows, vocab, n_top, slices, sc, by, tokens,
                        logprob_out, entropy_out, lse_out, top_idx_out, top_logprob_out,
                        dev_status};
  cudaStream_t st = (cudaStream_t)stream;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return RIPPLE_ECUDA;
  RIPPLE_CUDA_TRY(dtype == RIPPLE_BF16 ? launch_width<__nv_bfloat16>(p, row_bytes, dev, st)
                                       : launch_width<float>(p, row_bytes, dev, st));
  return RIPPLE_OK;
}
