// ripple_token_logprobs: log probabilities of given tokens, entropies and the most
// likely alternatives, from logits over the vocabulary, read from HBM once.
//
// With m the row's largest logit, d = x - m, w = exp(scale d), S' the sum of w over the
// row without one largest logit (whose w is 1) and T the sum of w d:
//   log P(x) = scale d - log1p(S'),   entropy = log1p(S') - scale T / (1 + S').
// Leaving the 1 out of the sum keeps the relative precision of log probabilities near 0.
//
// Work: a row is cut into C slices, one CTA each, the C CTAs of a row being a cluster
// (slices_of). A warp streams its share of the slice with 16-byte loads, several in
// flight, and keeps a running maximum for the warp (a vote per 8 logits of a lane, moved
// and rescaled when one is larger, which soon gets rare), sums per lane, and each lane's
// largest logit. The warps are merged through shared memory, the slices through the
// shared memory of the cluster's first CTA.
//
// Alternatives: keys order logits descending, equal ones by index. The n-th largest of the
// 32 largest logits of 8 lanes each bounds the slice's n-th largest key from below, so
// only lanes whose largest logit reaches it hold candidates; their logits are read once
// more (L2), and the candidates, a few more than n, are ranked by counting. Where there
// are more than fit (many ties, sorted rows), the n-th largest of those found is a
// higher bound, and the reading is repeated with it; every turn drops some.
#include <float.h>
#include <math.h>

#include "common.cuh"
#include "kernels.cuh"

namespace ripple {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kCtasPerSm = 4;
constexpr int kMaxSlices = 8;
constexpr int kVecs = 4;      // 16-byte loads a thread has in flight
constexpr int kCands = 512;   // candidates ranked at a time
constexpr unsigned kAll = 0xffffffffu;
typedef unsigned long long Key;

struct LogprobParams {
  const void *logits;
  long long row_stride;
  int n_rows, vocab, n_top, slices;
  float scale, scale2;
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

// Part of a row: its largest logit m, S' (the sum without that logit, so -1 for a part
// with nothing but -infinity) and T, relative to m.
struct Sums {
  float m, s, t;
};
// A sum n of terms relative to m_from, and its t, to a larger m.
__device__ __forceinline__ void rebase(float n, float &t, float &s, float m_from, float m,
                                       float scale2) {
  const float d = m_from == -INFINITY ? 0.f : fmaxf(m_from - m, -FLT_MAX);
  const float e = fast_exp2(d * scale2);
  t = e > 0.f ? e * (t + n * d) : 0.f;
  s = n * e;
}
__device__ __forceinline__ Sums merge(const Sums &a, const Sums &b, float scale2) {
  const bool first = a.m >= b.m;
  const Sums &hi = first ? a : b, &lo = first ? b : a;
  float s, t = lo.t;
  rebase(1.f + lo.s, t, s, lo.m, hi.m, scale2);
  return Sums{hi.m, hi.s + s, hi.t + t};
}

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

// A lane's part of the warp's running sums. The warp's m is the same on every lane; the
// lane that `owns` the logit m has left it out of its s.
struct Lane {
  float m = -INFINITY, top = -INFINITY;  // the warp's largest, this lane's own
  float2 s = make_float2(0.f, 0.f), t = make_float2(0.f, 0.f);
  bool owns = false;

  // N logits of every lane (-infinity for none).
  template <int N>
  __device__ __forceinline__ void add(const float (&x)[N], float scale2, int lane) {
    float g = x[0];
#pragma unroll
    for (int e = 1; e < N; ++e) g = fmaxf(g, x[e]);
    top = fmaxf(top, g);
    int skip = -1;
    if (__any_sync(kAll, g > m)) {
      float mn = g;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) mn = fmaxf(mn, __shfl_xor_sync(kAll, mn, o));
      const float n = s.x + s.y + (owns ? 1.f : 0.f);
      float ss, tt = t.x + t.y;
      rebase(n, tt, ss, m, mn, scale2);
      s = make_float2(ss, 0.f);
      t = make_float2(tt, 0.f);
      m = mn;
      owns = lane == __ffs(__ballot_sync(kAll, g == mn)) - 1;
      if (owns) {
#pragma unroll
        for (int e = N - 1; e >= 0; --e)
          if (x[e] == mn) skip = e;
      }
    }
    const float m0 = fmaxf(m, -FLT_MAX);  // a warp with nothing but -infinity so far: w = 0
    const float2 minus = make_float2(-m0, -m0), c = make_float2(scale2, scale2);
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      float2 d = __fadd2_rn(make_float2(x[e], x[e + 1]), minus);
      const float2 y = __fmul2_rn(d, c);
      float2 w = make_float2(fast_exp2(y.x), fast_exp2(y.y));
      if (skip >= 0) {
        if (skip == e) w.x = 0.f;
        if (skip == e + 1) w.y = 0.f;
      }
      s = __fadd2_rn(s, w);
      d.x = fmaxf(d.x, -FLT_MAX);  // 0 times -infinity is no term
      d.y = fmaxf(d.y, -FLT_MAX);
      t = __ffma2_rn(w, d, t);
    }
  }
};

struct Smem {
  Key cand[kCands];
  Key best[kMaxSlices][RIPPLE_MAX_TOP];  // of the slices, in the cluster's first CTA
  Sums sums[kMaxSlices];
  Sums warp[kWarps];
  float group[32];
  Key bound, kth;
  int n_hot, n_cand;
  uint16_t hot[kThreads];
};

// Ranks `n` keys by counting: f(rank, key) for each; equal keys (0: none) share a rank.
template <typename F>
__device__ __forceinline__ void rank_keys(const Key *keys, int n, F f) {
  for (int i = threadIdx.x; i < n; i += kThreads) {
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

template <typename T>
__global__ void __launch_bounds__(kThreads, kCtasPerSm)
    logprob_kernel(const __grid_constant__ LogprobParams p) {
  __shared__ Smem s;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int row_i = blockIdx.x / p.slices;
  const int slice = p.slices > 1 ? (int)cluster_rank() : 0;
  pdl_launch_dependents();
  pdl_wait();
  if (p.slices > 1) cluster_arrive();  // waited for before the first CTA's memory is written

  const Row<T> row(p, row_i);
  constexpr int E = Row<T>::E;
  const int v0 = (int)((long long)row.n_vec * slice / p.slices);
  const int v1 = (int)((long long)row.n_vec * (slice + 1) / p.slices);

  // the given token's logit, on its way while the row is read
  float given = 0.f;
  int token = -1;
  if (slice == 0 && tid == 0 && p.tokens != nullptr) {
    token = p.tokens[row_i];
    if (token >= 0 && token < p.vocab) given = to_f32(row.x[token]);
  }

  // Thread t has vectors v0 + t, v0 + t + kThreads, ..
  Lane sum;
  auto some = [&](int at) {  // one vector of every lane, partial ones and none among them
    float x[E];
    if (at < v1) {
      row.get(at, x);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = -INFINITY;
    }
    sum.add(x, p.scale2, lane);
  };
  int at = v0 + warp * 32;  // the warp's next
  if (v0 == 0 && row.lead != 0 && at < v1) {  // the row's first vector is partial
    some(at + lane);
    at += kThreads;
  }
  const int end = v1 - (v1 == row.n_vec && !row.whole(v1 - 1) ? 1 : 0);  // of whole vectors
  for (; at + 31 + (kVecs - 1) * kThreads < end; at += kVecs * kThreads) {
    uint4 u[kVecs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) u[i] = row.load(at + lane + i * kThreads);
#pragma unroll
    for (int i = 0; i < kVecs; i += 8 / E) {
      float x[8];
#pragma unroll
      for (int k = 0; k < 8 / E; ++k) unpack16(u[i + k], row.x, x + k * E);
      sum.add(x, p.scale2, lane);
    }
  }
  for (; at < v1; at += kThreads) some(at + lane);

  // the warp, the slice
  {
    float ss = sum.s.x + sum.s.y, tt = sum.t.x + sum.t.y;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      ss += __shfl_xor_sync(kAll, ss, o);
      tt += __shfl_xor_sync(kAll, tt, o);
    }
    if (lane == 0) s.warp[warp] = Sums{sum.m, sum.m == -INFINITY ? ss - 1.f : ss, tt};
  }
  float g = sum.top;
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) g = fmaxf(g, __shfl_xor_sync(kAll, g, o));
  if ((lane & 7) == 0) s.group[tid >> 3] = g;
  if (tid == 0) s.n_hot = s.n_cand = 0;
  __syncthreads();

  const int n_top = p.n_top;
  if (n_top > 0) {
    // the n-th largest of the 32 groups' largest logits
    if (warp == 0) {
      const uint32_t o = order_of(s.group[lane]);
      int above = 0;  // groups before this one, by value and then by lane
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const uint32_t other = __shfl_sync(kAll, o, i);
        above += other > o || (other == o && i < lane);
      }
      if (above == n_top - 1) s.bound = (Key)o << 32;
    }
    __syncthreads();
    Key bound = s.bound;
    // threads with candidates
    const bool has = v0 + tid < v1;
    if (has && (Key)order_of(sum.top) << 32 >= bound) s.hot[atomicAdd(&s.n_hot, 1)] = tid;
    __syncthreads();
    const int n_hot = s.n_hot;
    for (;;) {
      for (int i = warp; i < n_hot; i += kWarps)
        for (int u = v0 + s.hot[i] + lane * kThreads; u < v1; u += 32 * kThreads) {
          float x[E];
          row.get(u, x);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const int idx = row.first(u) + e;
            const Key k = key_of(x[e], idx);
            if (k >= bound && idx >= 0 && idx < p.vocab) {
              const int n = atomicAdd(&s.n_cand, 1);
              if (n < kCands) s.cand[n] = k;
            }
          }
        }
      __syncthreads();
      const int n = s.n_cand;
      if (n <= kCands) break;
      // too many: a higher bound from those found
      rank_keys(s.cand, kCands, [&](int rank, Key k) {
        if (rank == n_top - 1) s.kth = k;
      });
      __syncthreads();
      bound = s.kth;
      if (tid == 0) s.n_cand = 0;
      __syncthreads();
    }
  }
  Key *best = s.best[0];  // the slice's n_top largest, descending (0: none)
  if (p.slices > 1) cluster_wait();  // the first CTA runs
  if (n_top > 0) {
    const int n = s.n_cand;
    const uint32_t to = p.slices > 1 ? in_first(s.best[slice]) : 0;
    auto store = [&](int rank, Key k) {
      if (rank >= n_top) return;
      if (p.slices > 1)
        st_cluster(to + rank * 8, k);
      else
        best[rank] = k;
    };
    rank_keys(s.cand, n, store);
    if (tid >= n && tid < n_top) store(tid, 0);
  }
  Sums all = s.warp[0];
  if (tid == 0) {
#pragma unroll
    for (int w = 1; w < kWarps; ++w) all = merge(all, s.warp[w], p.scale2);
    if (p.slices > 1) {
      const uint32_t to = in_first(&s.sums[slice]);
      st_cluster(to, all.m);
      st_cluster(to + 4, all.s);
      st_cluster(to + 8, all.t);
    }
  }
  if (p.slices > 1) {
    cluster_arrive();
    cluster_wait();
    if (slice != 0) return;
    if (tid == 0) {
      all = s.sums[0];
      for (int i = 1; i < p.slices; ++i) all = merge(all, s.sums[i], p.scale2);
    }
    // the slices' alternatives, packed, and ranked again
    if (n_top > 0) {
      for (int i = tid; i < p.slices * n_top; i += kThreads)
        s.cand[i] = s.best[i / n_top][i % n_top];
      __syncthreads();
      rank_keys(s.cand, p.slices * n_top, [&](int rank, Key k) {
        if (rank < n_top) best[rank] = k;
      });
    }
  }
  if (tid == 0) {
    if (all.m == INFINITY) all.s = NAN;
    const float ls = log1pf(all.s);
    if (p.lse != nullptr) p.lse[row_i] = all.m == -INFINITY ? all.m + 0.f * all.s : p.scale * all.m + ls;
    if (p.entropy != nullptr) p.entropy[row_i] = ls - p.scale * all.t / (1.f + all.s);
    if (p.logprob != nullptr) {
      float y = 0.f;
      if (token >= p.vocab) {
        report(p.status, RIPPLE_EBOUNDS);
        y = NAN;
      } else if (token >= 0) {
        y = p.scale * (given - all.m) - ls;
      }
      p.logprob[row_i] = y;
    }
    s.sums[0] = Sums{all.m, ls, 0.f};
  }
  __syncthreads();
  if (tid < n_top) {
    const long long to = (long long)row_i * n_top + tid;
    const Key k = best[tid];
    p.top_idx[to] = (int)~(uint32_t)k;
    if (p.top_logprob != nullptr)
      p.top_logprob[to] = p.scale * (value_of((uint32_t)(k >> 32)) - s.sums[0].m) - s.sums[0].s;
  }
}

// Slices of a row: enough CTAs for every place on the GPU, of at least kVecs vectors a
// thread.
int slices_of(int n_rows, long long row_bytes) {
  constexpr int kPlaces = 152 * kCtasPerSm;
  int c = 1;
  while (c < kMaxSlices && (long long)n_rows * c < kPlaces &&
         row_bytes >= 2LL * c * kThreads * 16 * kVecs)
    c *= 2;
  return c;
}

template <typename T>
cudaError_t launch(const LogprobParams &p, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.n_rows * p.slices);
  cfg.blockDim = dim3(kThreads);
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
  const cudaError_t e = cudaLaunchKernelEx(&cfg, logprob_kernel<T>, p);
  count_launches(1);
  return e;
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
  if (!(scale >= 0.f) || isinf(scale)) return RIPPLE_EINVAL;
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
  const int slices = slices_of(n_rows, (long long)vocab * (dtype == RIPPLE_F32 ? 4 : 2));
  const LogprobParams p{logits, row_stride, n_rows, vocab, n_top, slices, sc, sc * kLog2e, tokens,
                        logprob_out, entropy_out, lse_out, top_idx_out, top_logprob_out,
                        dev_status};
  cudaStream_t st = (cudaStream_t)stream;
  RIPPLE_CUDA_TRY(dtype == RIPPLE_BF16 ? launch<__nv_bfloat16>(p, st) : launch<float>(p, st));
  return RIPPLE_OK;
}
