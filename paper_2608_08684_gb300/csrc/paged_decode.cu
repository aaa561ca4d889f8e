// ripple_paged_decode_attn: attention of one new token per sequence over a paged cache of
// bf16 or fp32 rows (kernels in paged_decode.cuh).
#include "paged_decode.cuh"

namespace ripple {
namespace {

int block_rows(const ripple_paged_desc *d) {
  return 4096 / (d->head_dim * (d->dtype == RIPPLE_BF16 ? 2 : 4));
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
  *bytes_host = plan(&p, block_rows(desc), kWarpsPerSm, true, sm_count(dev), nullptr);
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
  if (!query_strides(desc, n_q_heads, q_strides, &p)) return RIPPLE_EINVAL;
  int dev = 0;
  const cudaError_t got = cudaGetDevice(&dev);
  if (got != cudaSuccess || dev < 0 || dev >= kMaxDevices) dev = 0;
  if (workspace_bytes < plan(&p, block_rows(desc), kWarpsPerSm, true, sm_count(dev), workspace)) return RIPPLE_EWORKSPACE;
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
