// ripple_token_logprobs: log probabilities of given tokens, entropies and the most
// likely alternatives, from logits over the vocabulary.
//
// With m the row's largest logit, d = x - m, w = exp(scale d), S' the sum of w over the
// row without the first largest logit (whose w is 1) and T the sum of w d:
//   log P(x) = scale d - log1p(S'),   entropy = log1p(S') - scale T / (1 + S').
// Leaving the 1 out of the sum keeps the relative precision of log probabilities near 0.
//
// One CTA per row: a pass for the largest logit, one for the sums, and one per
// alternative for the largest (logit, lowest index) below the one before.
#include <float.h>
#include <math.h>

#include "common.cuh"
#include "kernels.cuh"

namespace ripple {
namespace {

constexpr int kThreads = 256;

struct LogprobParams {
  const void *logits;
  long long row_stride;
  int n_rows, vocab, n_top;
  float scale;
  const int32_t *tokens;
  float *logprob, *entropy, *lse;
  int32_t *top_idx;
  float *top_logprob;
  int32_t *status;
};

// Descending logits, then ascending indices, as one descending 64-bit key; -0 ties with 0.
__device__ __forceinline__ unsigned long long key_of(float x, int i) {
  uint32_t u = __float_as_uint(x + 0.f);
  u = u & 0x80000000u ? ~u : u | 0x80000000u;
  return (unsigned long long)u << 32 | (uint32_t)~i;
}

template <typename V, typename F>
__device__ __forceinline__ V block_reduce(V v, F f) {
  __shared__ V part[kThreads / 32];
  for (int o = 16; o > 0; o >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  v = part[0];
  for (int w = 1; w < kThreads / 32; ++w) v = f(v, part[w]);
  return v;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) logprob_kernel(const LogprobParams p) {
  const int row = blockIdx.x, tid = threadIdx.x;
  const T *x = (const T *)p.logits + row * p.row_stride;
  auto most = [](unsigned long long a, unsigned long long b) { return a > b ? a : b; };
  auto sum = [](float a, float b) { return a + b; };
  unsigned long long best = 0;
  for (int i = tid; i < p.vocab; i += kThreads) best = most(best, key_of(to_f32(x[i]), i));
  best = block_reduce(best, most);
  const int at = (int)~(uint32_t)best;
  const float m = to_f32(x[at]);
  float s = 0.f, t = 0.f;
  for (int i = tid; i < p.vocab; i += kThreads) {
    const float d = to_f32(x[i]) - m;
    const float w = i == at ? (d == 0.f ? 0.f : d) : expf(p.scale * d);
    s += w;
    t += w > 0.f ? w * d : 0.f;
  }
  s = block_reduce(s, sum);
  t = block_reduce(t, sum);
  const float ls = log1pf(s);
  if (tid == 0) {
    if (p.lse != nullptr) p.lse[row] = m == -INFINITY ? m : p.scale * m + ls;
    if (p.entropy != nullptr) p.entropy[row] = ls - p.scale * t / (1.f + s);
    if (p.logprob != nullptr) {
      const int tok = p.tokens[row];
      float y = 0.f;
      if (tok >= p.vocab) {
        report(p.status, RIPPLE_EBOUNDS);
        y = NAN;
      } else if (tok >= 0) {
        y = p.scale * (to_f32(x[tok]) - m) - ls;
      }
      p.logprob[row] = y;
    }
  }
  for (int j = 0; j < p.n_top; ++j) {
    if (j > 0) {
      const unsigned long long before = best;
      best = 0;
      for (int i = tid; i < p.vocab; i += kThreads) {
        const unsigned long long key = key_of(to_f32(x[i]), i);
        if (key < before) best = most(best, key);
      }
      best = block_reduce(best, most);
    }
    if (tid == 0) {
      const int i = (int)~(uint32_t)best;
      p.top_idx[(long long)row * p.n_top + j] = i;
      if (p.top_logprob != nullptr)
        p.top_logprob[(long long)row * p.n_top + j] = p.scale * (to_f32(x[i]) - m) - ls;
    }
  }
}

}  // namespace
}  // namespace ripple

using namespace ripple;

extern "C" ripple_status ripple_token_logprobs(
    int32_t n_rows, int32_t vocab, int64_t row_stride, int32_t dtype, float scale, int32_t n_top,
    const void *logits, const int32_t *tokens, float *logprob_out, float *entropy_out,
    float *lse_out, int32_t *top_idx_out, float *top_logprob_out, int32_t *dev_status,
    void *stream) {
  if (n_rows < 0 || vocab < 1 || vocab > (1 << 30) || row_stride < 0 || row_stride > (1LL << 40))
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
  const LogprobParams p{logits, row_stride, n_rows, vocab, n_top, scale > 0.f ? scale : 1.f,
                        tokens, logprob_out, entropy_out, lse_out, top_idx_out, top_logprob_out,
                        dev_status};
  cudaStream_t st = (cudaStream_t)stream;
  if (dtype == RIPPLE_BF16)
    logprob_kernel<__nv_bfloat16><<<n_rows, kThreads, 0, st>>>(p);
  else
    logprob_kernel<float><<<n_rows, kThreads, 0, st>>>(p);
  count_launches(1);
  RIPPLE_CUDA_TRY(cudaGetLastError());
  return RIPPLE_OK;
}
