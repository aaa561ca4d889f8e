// ripple_paged_decode_attn: attention of one new token per sequence over a paged cache.
//
// One CTA per (sequence, KV head): its warps take the cache rows in turn, a lane holds
// d / 32 dims of the row and of every query head's output, and each warp keeps its own
// running maximum and sum per head (online softmax in log2 units); the warps are merged
// through shared memory.
#include <math.h>

#include "common.cuh"
#include "kernels.cuh"
#include "paged.cuh"

namespace ripple {
namespace {

constexpr int kMaxGroup = 16;
constexpr int kWarps = 4;

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
};

template <typename T, int D>
__global__ void __launch_bounds__(kWarps * 32)
    paged_decode_kernel(const __grid_constant__ PagedDecParams p) {
  constexpr int kDims = D / 32;
  __shared__ float red_o[kWarps][kMaxGroup][D];
  __shared__ float red_m[kWarps][kMaxGroup], red_l[kWarps][kMaxGroup];
  __shared__ float qs[kMaxGroup][D];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int b = blockIdx.x / p.g.Hkv, h = blockIdx.x % p.g.Hkv;
  int len = p.lens[b];
  const long long room = (long long)p.g.max_pages << p.g.shift;
  if (len > room) {
    if (tid == 0) report(p.status, RIPPLE_EFULL);
    len = (int)room;
  }
  for (int e = tid; e < p.G * D; e += kWarps * 32)
    qs[e / D][e % D] =
        to_f32(((const T *)p.q)[b * p.q_seq + (h * p.G + e / D) * p.q_head + e % D]) * p.scale2;
  __syncthreads();
  float acc[kMaxGroup][kDims], m[kMaxGroup], l[kMaxGroup];
#pragma unroll
  for (int g = 0; g < kMaxGroup; ++g) {
    m[g] = -INFINITY;
    l[g] = 0.f;
#pragma unroll
    for (int e = 0; e < kDims; ++e) acc[g][e] = 0.f;
  }
  for (int r = warp; r < len; r += kWarps) {
    const int page = p.table[(long long)b * p.g.max_pages + (r >> p.g.shift)];
    if ((unsigned)page >= (unsigned)p.g.n_pages) {
      if (lane == 0) report(p.status, RIPPLE_EBOUNDS);
      continue;
    }
    const long long at = page * p.g.page_stride + h * p.g.head_stride +
                         (r & ((1 << p.g.shift) - 1)) * p.g.row_stride;
    float k[kDims], v[kDims];
#pragma unroll
    for (int e = 0; e < kDims; ++e) {
      k[e] = to_f32(((const T *)p.k_pages)[at + e * 32 + lane]);
      v[e] = to_f32(((const T *)p.v_pages)[at + e * 32 + lane]);
    }
#pragma unroll
    for (int g = 0; g < kMaxGroup; ++g) {
      if (g >= p.G) break;
      float x = 0.f;
#pragma unroll
      for (int e = 0; e < kDims; ++e) x += qs[g][e * 32 + lane] * k[e];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
      const float mn = fmaxf(m[g], x);
      const float sub = mn == -INFINITY ? 0.f : mn;  // scores of -infinity alone
      const float a = fast_exp2(m[g] - sub), w = fast_exp2(x - sub);
      m[g] = mn;
      l[g] = l[g] * a + w;
#pragma unroll
      for (int e = 0; e < kDims; ++e) acc[g][e] = acc[g][e] * a + w * v[e];
    }
  }
#pragma unroll
  for (int g = 0; g < kMaxGroup; ++g) {
    if (g >= p.G) break;
#pragma unroll
    for (int e = 0; e < kDims; ++e) red_o[warp][g][e * 32 + lane] = acc[g][e];
    if (lane == 0) {
      red_m[warp][g] = m[g];
      red_l[warp][g] = l[g];
    }
  }
  __syncthreads();
  for (int e = tid; e < p.G * D; e += kWarps * 32) {
    const int g = e / D;
    float M = -INFINITY, num = 0.f, den = 0.f;
    for (int w = 0; w < kWarps; ++w) M = fmaxf(M, red_m[w][g]);
    const float sub = M == -INFINITY ? 0.f : M;
    for (int w = 0; w < kWarps; ++w) {
      const float a = fast_exp2(red_m[w][g] - sub);
      num += a * red_o[w][g][e % D];
      den += a * red_l[w][g];
    }
    const long long row = (long long)b * p.Hq + h * p.G + g;
    p.out[row * D + e % D] = den != 0.f ? num / den : 0.f;  // 0: no row counts
    if (p.lse != nullptr && e % D == 0) p.lse[row] = (M + log2f(den)) / kLog2e;
  }
}

bool decode_args(const ripple_paged_desc *d, int n_q_heads, PagedDecParams *p) {
  if (!paged_geom(d, &p->g)) return false;
  if (n_q_heads < 1 || n_q_heads % d->n_kv_heads != 0) return false;
  p->Hq = n_q_heads;
  p->G = n_q_heads / d->n_kv_heads;
  return p->G <= kMaxGroup;
}

template <typename T, int D>
cudaError_t launch(const PagedDecParams &p, cudaStream_t st) {
  paged_decode_kernel<T, D><<<p.g.B * p.g.Hkv, kWarps * 32, 0, st>>>(p);
  count_launches(1);
  return cudaGetLastError();
}

}  // namespace
}  // namespace ripple

using namespace ripple;

extern "C" ripple_status ripple_paged_decode_workspace_bytes(const ripple_paged_desc *desc,
                                                             int32_t n_q_heads,
                                                             size_t *bytes_host) {
  PagedDecParams p;
  if (!decode_args(desc, n_q_heads, &p) || bytes_host == nullptr) return RIPPLE_EINVAL;
  *bytes_host = 256;
  return RIPPLE_OK;
}

extern "C" ripple_status ripple_paged_decode_attn(
    const ripple_paged_desc *desc, int32_t n_q_heads, float scale, const void *q,
    const ripple_token_strides *q_strides, const void *k_pages, const void *v_pages,
    const int32_t *block_table, const int32_t *lens, float *out, float *lse, void *workspace,
    size_t workspace_bytes, int32_t *dev_status, void *stream) {
  PagedDecParams p;
  if (!decode_args(desc, n_q_heads, &p)) return RIPPLE_EINVAL;
  if (!(scale >= 0.f) || isinf(scale)) return RIPPLE_EINVAL;
  if (!q || !k_pages || !v_pages || !block_table || !lens || !out || !workspace ||
      ((uintptr_t)workspace & 255u))
    return RIPPLE_EINVAL;
  if (!aligned16_host(q) || !aligned16_host(k_pages) || !aligned16_host(v_pages) ||
      !aligned16_host(out))
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
  if (workspace_bytes < 256) return RIPPLE_EWORKSPACE;
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
  cudaError_t e;
  if (desc->dtype == RIPPLE_BF16)
    e = desc->head_dim == 128 ? launch<__nv_bfloat16, 128>(p, st) : launch<__nv_bfloat16, 64>(p, st);
  else
    e = desc->head_dim == 128 ? launch<float, 128>(p, st) : launch<float, 64>(p, st);
  RIPPLE_CUDA_TRY(e);
  return RIPPLE_OK;
}
