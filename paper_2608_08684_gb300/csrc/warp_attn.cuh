// Warp-level pieces of attention for a few query rows: matrix instructions with
// probabilities kept to 24 bits, and sums over the lanes of a row group.
#pragma once

#include <stdint.h>

#include "common.cuh"

namespace ripple {

__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
// C (16 x 8, fp32) += A (16 x 16) . B (16 x 8), bf16.
__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                         uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// A pair of fp32 values >= 0 in three bf16 parts, h + m + l, 24 bits of each value, so
// that their products with bf16 values lose nothing against fp32. Every part is cut off
// (not rounded, which could leave a rest of the other sign) and m and l are at least
// 2^-133, the smallest bf16 value: a positive probability has no part that is 0, which
// an infinite value would turn into a NaN. A finite value v comes out at most
// 2^-131 |v| too large.
__device__ __forceinline__ uint32_t upper_halves(float x0, float x1) {
  return __byte_perm(__float_as_uint(x0), __float_as_uint(x1), 0x7632);
}
__device__ __forceinline__ float rest_of(float x, float least) {
  return fmaxf(x - __uint_as_float(__float_as_uint(x) & 0xffff0000u), least);
}
struct Parts {
  uint32_t h, m, l;
};
// kHalves: l is half of the low part (for operands that hold it twice).
template <bool kHalves>
__device__ __forceinline__ Parts three_parts(float x0, float x1) {
  Parts p;
  p.h = upper_halves(x0, x1);
  const float r0 = rest_of(x0, 0x1p-133f), r1 = rest_of(x1, 0x1p-133f);
  p.m = upper_halves(r0, r1);
  if (kHalves)
    p.l = upper_halves(0.5f * rest_of(r0, 0x1p-132f), 0.5f * rest_of(r1, 0x1p-132f));
  else
    p.l = upper_halves(rest_of(r0, 0x1p-133f), rest_of(r1, 0x1p-133f));
  return p;
}

// Per-head values of a lane in the order j ^ hq, hq the lane's own head
// (lane % S) / (S / G): every step of the sums and of their return over the S lanes of a
// row group is then a plain shuffle. reduce_heads: v[0] becomes the full sum of head hq.
template <int S, int G>
__device__ __forceinline__ void reduce_heads(float (&v)[G]) {
#pragma unroll
  for (int o = S / 2, n = G; o >= 1; o >>= 1) {
    if (n > 1) {
#pragma unroll
      for (int i = 0; i < G / 2; ++i)
        if (i < n / 2) v[i] += __shfl_xor_sync(0xffffffffu, v[i + n / 2], o);
      n /= 2;
    } else {
      v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
    }
  }
}
// The value x of head hq to every lane: o[j] of head j ^ hq.
template <int S, int G>
__device__ __forceinline__ void spread_heads(float x, float (&o)[G]) {
  o[0] = x;
#pragma unroll
  for (int lev = 0; (1 << lev) < G; ++lev)
#pragma unroll
    for (int i = 0; i < (1 << lev); ++i)
      o[(1 << lev) + i] = __shfl_xor_sync(0xffffffffu, o[i], (S / G) << lev);
}

}  // namespace ripple
