// ripple_paged_decode_attn_q8: attention of one new token per sequence over a paged cache of
// 8-bit codes (e4m3) with a power-of-two scale a row and head (runs, rings and joins in
// paged_decode.cuh).
//
// A step is bound by the cache's bytes, half of a bf16 cache's, so that a warp has half the
// time for a row. The scales stay out of the matrix products: a key's multiplies its scores,
// a value's its probabilities, and the codes become fp16 by one conversion for two of them,
// exactly. fp16 has too few exponents for queries and probabilities as they are:
//  - a head's query is multiplied by the power of two that brings its largest element to
//    [2^14, 2^15) (undone on the scores). An element is then off by at most 2^-25 of
//    2^14; fp32 queries are two fp16 parts, 22 bits.
//  - probability and value scale together, 2^(x_r + e_r), are taken relative to their own
//    running maximum, not the scores', times 2^14, in two fp16 parts: 22 bits, and at most
//    2^-39 of the largest lost where they are tiny.
// The sum of the probabilities has the scores' maximum, in fp32, and the products' reference is
// relative to that: there is none before the first score.
// Measured, D 128, 8 KV heads, 4 heads each: 64 sequences of 64 to 32768 rows (622 MB) 105 us,
// 5.9 TB/s (87% of the copy rate; bf16 pages 151); one of 470 rows 5.5 us. fp32 queries, 7 on each
// of 4 KV heads of 64, 9 sequences of up to 60000 rows 33 us, the chain of a block's two products
// and softmax.
#include <cuda_fp16.h>

#include "paged_decode.cuh"

namespace ripple {
namespace {

// Two codes (the low 16 bits) as fp16 values.
__device__ __forceinline__ uint32_t codes_f16x2(uint32_t codes) {
  uint32_t r;
  asm("{\n .reg .b16 c, d;\n mov.b32 {c, d}, %1;\n cvt.rn.f16x2.e4m3x2 %0, c;\n}\n"
      : "=r"(r)
      : "r"(codes));
  return r;
}
__device__ __forceinline__ uint32_t codes_f16x2_high(uint32_t codes) {
  uint32_t r;
  asm("{\n .reg .b16 c, d;\n mov.b32 {c, d}, %1;\n cvt.rn.f16x2.e4m3x2 %0, d;\n}\n"
      : "=r"(r)
      : "r"(codes));
  return r;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&h);
}
// What the fp16 pair leaves of lo and hi, as another.
__device__ __forceinline__ uint32_t rest_f16x2(float lo, float hi, uint32_t pair) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&pair));
  return pack_f16x2(lo - f.x, hi - f.y);
}
// C (16 x 8, fp32) += A (16 x 16) . B (16 x 8), fp16.
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                        uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// The transpose of an 8 x 8 matrix of 16-bit elements, two of a row in each lane.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ float pow2(int e) {  // -126 <= e <= 127
  return __int_as_float((e + 127) << 23);
}

// Keys and dims are the matrix products' rows, heads their columns: S^T[key][head] = K . Q^T
// and O^T[dim][head] += V^T . P^T, so that a product of 16 x 16 x 8 has no empty rows and
// up to 8 heads one set of columns. Which dims make up a step of the first product's sum is
// free (the same of K and of Q): a lane's 16 bytes of a key are four steps' operands as they
// lie. For the second, ldmatrix brings two keys' pairs of dims to a lane, and rows of the
// product are a pair's first dims (0-7) and second ones (8-15). The probabilities' parts: up
// to 4 heads repeat in columns 4-7, which take the second part; more heads take a product a
// part.
// A lane (g, t): keys g and g + 8 of 16, the heads of columns 2t and 2t + 1.
template <typename Q, int D, int G>
struct Rows<Codes8<Q>, D, G> {
  using C = Cfg<Codes8<Q>, D, G>;
  static constexpr int NT = G > 8 ? 2 : 1;         // sets of 8 columns
  static constexpr bool kTwice = G <= 4;           // heads repeat
  static constexpr int QP = sizeof(Q) == 4 ? 2 : 1;  // parts of a query
  static constexpr int KS = D / 16, PC = D / 16;   // steps of a score, pieces of a row
  // The probabilities' reference may lag by so much (log2), and is 2^14 times.
  static constexpr float kSlackW = 1.f;
  static constexpr int kTop = 14;
  uint32_t qb[QP][NT][KS][2];
  float qs[NT][2];  // the heads' scale: logit scale, over the query's power of two
  float m[NT][2], l[NT][2];
  int ew[NT][2];    // the outputs' reference is m + ew
  float acc[PC][NT][4];

  __device__ __forceinline__ void start(const PagedDecParams &p, const Walk<C::RB, C::COST> &w, int lane) {
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int head = (kTwice ? g & 3 : g) + 8 * nt;
      const Q *q = (const Q *)p.q + w.b * p.q_seq + (w.h * p.G + min(head, p.G - 1)) * p.q_head;
      // (as it lies: the loads of a lane are in flight together)
      constexpr int kRaw = 2 * sizeof(Q);  // 16-byte pieces of 16 elements
      uint4 raw[D / 64][kRaw];
#pragma unroll
      for (int i = 0; i < D / 64; ++i)
#pragma unroll
        for (int j = 0; j < kRaw; ++j)
          raw[i][j] = *(reinterpret_cast<const uint4 *>(q + 16 * (t + 4 * i)) + j);
      auto element = [&](int i, int e) {  // of the 16 of piece i
        const uint4 &u = raw[i][e * sizeof(Q) / 16];
        const int word = e * sizeof(Q) % 16 / 4;
        const uint32_t w = word == 0 ? u.x : word == 1 ? u.y : word == 2 ? u.z : u.w;
        return __uint_as_float(sizeof(Q) == 4 ? w : e & 1 ? w & 0xffff0000u : w << 16);
      };
      float most = 0.f;
#pragma unroll
      for (int i = 0; i < D / 64; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) most = fmaxf(most, fabsf(element(i, e)));
      most = fmaxf(most, __shfl_xor_sync(kAll, most, 1));
      most = fmaxf(most, __shfl_xor_sync(kAll, most, 2));
      // (infinities keep the others finite; what is below 2^-86 may be lost)
      const int up = most == 0.f ? 0 : min(kTop - ((__float_as_int(most) >> 23) - 127), 100);
      const float f = head < p.G ? pow2(up) : 0.f;
#pragma unroll
      for (int i = 0; i < D / 64; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {  // step 4 i + e / 2
          const float lo = head < p.G ? element(i, 2 * e) * f : 0.f;
          const float hi = head < p.G ? element(i, 2 * e + 1) * f : 0.f;
          const uint32_t h = pack_f16x2(lo, hi);
          qb[0][nt][4 * i + e / 2][e & 1] = h;
          if constexpr (QP == 2) qb[1][nt][4 * i + e / 2][e & 1] = rest_f16x2(lo, hi, h);
        }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        qs[nt][e] = p.scale2 * pow2(-__shfl_sync(kAll, up, (2 * t + e) * 4));
        m[nt][e] = -INFINITY;
        l[nt][e] = 0.f;
        ew[nt][e] = 0;
      }
#pragma unroll
      for (int i = 0; i < PC; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][nt][e] = 0.f;
    }
  }

  // 16 rows from row0 of the stage on; kMask: some are not there.
  template <bool kMask>
  __device__ __forceinline__ void step(const Stage<Codes8<Q>, D, G> &stage, uint32_t ks, uint32_t vs,
                                       int row0, uint32_t live, int lane) {
    const int g = lane >> 2, t = lane & 3;
    const int swz = C::swizzle(g);  // (of rows g and g + 8)
    float sc[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) sc[nt][e] = 0.f;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const uint32_t at = ks + (row0 + g) * C::ROW_BYTES + (((t + 4 * i) ^ swz) << 4);
      uint32_t w0[4], w1[4];
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(w0[0]), "=r"(w0[1]), "=r"(w0[2]), "=r"(w0[3])
                   : "r"(at)
                   : "memory");
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(w1[0]), "=r"(w1[1]), "=r"(w1[2]), "=r"(w1[3])
                   : "r"(at + 8 * C::ROW_BYTES)
                   : "memory");
#pragma unroll
      for (int s2 = 0; s2 < 4; s2 += 2) {  // two steps: matrix instructions cut their sums off
        uint32_t a[2][4];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          a[s][0] = codes_f16x2(w0[s2 + s]);
          a[s][1] = codes_f16x2(w1[s2 + s]);
          a[s][2] = codes_f16x2_high(w0[s2 + s]);
          a[s][3] = codes_f16x2_high(w1[s2 + s]);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int qp = QP - 1; qp >= 0; --qp)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
              const uint32_t(&b)[2] = qb[qp][nt][4 * i + s2 + s];
              mma_f16(part, a[s], b[0], b[1]);
            }
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[nt][e] += part[e];
        }
      }
    }
    const float4 s0 = stage.scale[row0 + g], s1 = stage.scale[row0 + g + 8];
    const bool on0 = !kMask || (live >> g & 1), on1 = !kMask || (live >> (g + 8) & 1);
    uint32_t ph[NT][2], pl[NT][2];  // the operand's keys 0-7 and 8-15, high and low parts
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float w[2][2];  // [key][column]
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        // scores are a product of a (exact) and b; the fused multiply-add leaves out its rounding
        const float a0 = sc[nt][e] * s0.x, b0 = s0.y * qs[nt][e];
        const float a1 = sc[nt][2 + e] * s1.x, b1 = s1.y * qs[nt][e];
        const float x0 = on0 ? a0 * b0 : -INFINITY, x1 = on1 ? a1 * b1 : -INFINITY;
        const float mb = fmaxf(x0, x1);
        float sub = m[nt][e] == -INFINITY ? 0.f : m[nt][e];
        auto top_weight = [&] {  // of the lane's two, log2, over the scores' maximum
          return fmaxf(on0 ? (x0 - sub) + s0.z : -INFINITY, on1 ? (x1 - sub) + s1.z : -INFINITY);
        };
        if (__any_sync(kAll, mb > m[nt][e] + kSlack || top_weight() > (float)ew[nt][e] + kSlackW)) {
          // (both references move together where one has to; the outputs' never falls, and is none
          // before the first score)
          float mr = mb;
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) mr = fmaxf(mr, __shfl_xor_sync(kAll, mr, o));
          float was = m[nt][e] == -INFINITY ? -INFINITY : (float)ew[nt][e];
          if (mr > m[nt][e]) {
            const float fall = m[nt][e] - mr;
            l[nt][e] *= fast_exp2(fall);
            was += fall;
            m[nt][e] = mr;
            sub = mr;
          }
          float yr = top_weight();
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) yr = fmaxf(yr, __shfl_xor_sync(kAll, yr, o));
          ew[nt][e] = (int)fminf(fmaxf(ceilf(fmaxf(was, yr)), -400.f), 400.f);
          const float a = fast_exp2(was - (float)ew[nt][e]);
#pragma unroll
          for (int i = 0; i < PC; ++i) {
            acc[i][nt][e] *= a;
            acc[i][nt][2 + e] *= a;
          }
          __syncwarp();
        }
        const bool rounded = fabsf(sub) >= 65536.f;
        const float d0 = rounded ? x0 - sub : fmaf(a0, b0, -sub);
        const float d1 = rounded ? x1 - sub : fmaf(a1, b1, -sub);
        const float top = (float)(kTop - ew[nt][e]);
        const float p0 = on0 ? fast_exp2(d0) : 0.f, p1 = on1 ? fast_exp2(d1) : 0.f;
        l[nt][e] += p0 + p1;
        w[0][e] = on0 ? fast_exp2(d0 + (s0.z + top)) : 0.f;
        w[1][e] = on1 ? fast_exp2(d1 + (s1.z + top)) : 0.f;
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t hi = pack_f16x2(w[k][0], w[k][1]);
        const uint32_t lo = rest_f16x2(w[k][0], w[k][1], hi);
        if constexpr (kTwice) {
          ph[nt][k] = transpose8(t < 2 ? hi : lo);
        } else {
          ph[nt][k] = transpose8(hi);
          pl[nt][k] = transpose8(lo);
        }
      }
    }
    const int row = row0 + (lane & 15);  // keys 0-7, 8-15 of a piece, then of the next one
    const uint32_t va = vs + row * C::ROW_BYTES;
    const int vz = C::swizzle(lane & 7), vp = lane >> 4;
#pragma unroll
    for (int i = 0; i < PC; i += 2) {
      uint32_t r[4];
      ldmatrix4_trans(va + (((i + vp) ^ vz) << 4), r);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        // two keys' pairs of dims: to two keys' first and second ones
        const uint32_t lo = __byte_perm(r[2 * j], 0, 0x3120), hi = __byte_perm(r[2 * j + 1], 0, 0x3120);
        const uint32_t a[4] = {codes_f16x2(lo), codes_f16x2_high(lo), codes_f16x2(hi),
                               codes_f16x2_high(hi)};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float part[4] = {0.f, 0.f, 0.f, 0.f};
          if constexpr (!kTwice) mma_f16(part, a, pl[nt][0], pl[nt][1]);
          mma_f16(part, a, ph[nt][0], ph[nt][1]);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i + j][nt][e] += part[e];
        }
      }
    }
  }

  __device__ __forceinline__ void block(const PagedDecParams &, const Stage<Codes8<Q>, D, G> &stage,
                                        uint32_t live, int lane) {
    const uint32_t ks = smem_u32(stage.kv[0]), vs = smem_u32(stage.kv[1]);
#pragma unroll 1
    for (int i = 0; i < C::RB / 16; ++i) {
      const uint32_t part = live >> (16 * i) & 0xffffu;
      if (part == 0xffffu)
        step<false>(stage, ks, vs, 16 * i, part, lane);
      else if (part != 0)
        step<true>(stage, ks, vs, 16 * i, part, lane);
    }
  }

  // The warp's rows done: full sums, outputs relative to the scores' maximum.
  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) l[nt][e] += __shfl_xor_sync(kAll, l[nt][e], o);
        const int up = ew[nt][e] - kTop, half = up / 2;  // two factors: 2^up may be no fp32 value
        const float f = fast_exp2((float)half), f2 = fast_exp2((float)(up - half));
#pragma unroll
        for (int i = 0; i < PC; ++i)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float &a = acc[i][nt][2 * k + e];
            if (kTwice) a += __shfl_xor_sync(kAll, a, 2);
            a = a * f * f2;
          }
      }
  }
  __device__ __forceinline__ void normalise() {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float inv = l[nt][e] != 0.f ? 1.f / l[nt][e] : 0.f;  // 0: no row counts
#pragma unroll
        for (int i = 0; i < PC; ++i) {
          acc[i][nt][e] *= inv;
          acc[i][nt][2 + e] *= inv;
        }
      }
  }
  template <typename F>
  __device__ __forceinline__ void stats(int lane, F f) {
    const int t = lane & 3;
    if (lane >= 4 || (kTwice && t >= 2)) return;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) f(8 * nt + 2 * t + e, m[nt][e], l[nt][e]);
  }
  template <typename F>
  __device__ __forceinline__ void outputs(int lane, F f) {
    const int g = lane >> 2, t = lane & 3;
    if (kTwice && t >= 2) return;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int i = 0; i < PC; ++i)
          f(8 * nt + 2 * t + e, 16 * i + 2 * g, make_float2(acc[i][nt][e], acc[i][nt][2 + e]));
  }
};

// Heads of a group, padded to 4, 8 or 16.
template <typename Q, int D>
cudaError_t launch_q8(const PagedDecParams &p, int dev, cudaStream_t st) {
  if (p.G <= 4) return launch<Codes8<Q>, D, 4>(p, dev, st);
  if (p.G <= 8) return launch<Codes8<Q>, D, 8>(p, dev, st);
  return launch<Codes8<Q>, D, 16>(p, dev, st);
}

constexpr int kBlockRows = 32;
// One phase of runs: a warp's time for a row is its own more than HBM's, so that SMs differ little
// (64 sequences of 64 to 32768 rows 105.8 us, in three phases 117.9).
constexpr bool kPhased = false;
// Bytes of a call's workspace; those of the most warps that any group size has, so that more
// query heads never need fewer.
size_t workspace_need(PagedDecParams p, int sms) {
  return plan(&p, kBlockRows, codes_warps(p.g.D, 1), kPhased, sms, nullptr);
}

}  // namespace
}  // namespace ripple

using namespace ripple;

extern "C" ripple_status ripple_paged_decode_q8_workspace_bytes(const ripple_paged_desc *desc,
                                                                int32_t n_q_heads,
                                                                size_t *bytes_host) {
  PagedDecParams p;
  if (!decode_args(desc, n_q_heads, &p, true) || bytes_host == nullptr) return RIPPLE_EINVAL;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) dev = 0;
  *bytes_host = workspace_need(p, sm_count(dev));
  return RIPPLE_OK;
}

extern "C" ripple_status ripple_paged_decode_attn_q8(
    const ripple_paged_desc *desc, const ripple_paged_scales *scales, int32_t n_q_heads,
    float scale, const void *q, const ripple_token_strides *q_strides, const void *k_pages,
    const void *v_pages, const int32_t *block_table, const int32_t *lens, float *out, float *lse,
    void *workspace, size_t workspace_bytes, int32_t *dev_status, void *stream) {
  PagedDecParams p;
  if (!decode_args(desc, n_q_heads, &p, true)) return RIPPLE_EINVAL;
  ScaleGeom s;
  if (!scale_geom(desc, scales, &s)) return RIPPLE_EINVAL;
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
  if (workspace_bytes < workspace_need(p, sm_count(dev))) return RIPPLE_EWORKSPACE;
  plan(&p, kBlockRows, codes_warps(p.g.D, p.G), kPhased, sm_count(dev), workspace);
  if (got != cudaSuccess) return RIPPLE_ECUDA;
  p.scale2 = (scale > 0.f ? scale : 1.0f / sqrtf((float)desc->head_dim)) * kLog2e;
  p.q = q;
  p.k_pages = k_pages;
  p.v_pages = v_pages;
  p.k_scales = s.k;
  p.v_scales = s.v;
  p.scale_page = s.page_stride;
  p.scale_head = s.head_stride;
  p.scale_row = s.row_stride;
  p.table = block_table;
  p.lens = lens;
  p.out = out;
  p.lse = lse;
  p.status = dev_status;
  cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e;
  if (desc->dtype == RIPPLE_BF16)
    e = desc->head_dim == 128 ? launch_q8<__nv_bfloat16, 128>(p, dev, st)
                              : launch_q8<__nv_bfloat16, 64>(p, dev, st);
  else
    e = desc->head_dim == 128 ? launch_q8<float, 128>(p, dev, st)
                              : launch_q8<float, 64>(p, dev, st);
  RIPPLE_CUDA_TRY(e);
  return RIPPLE_OK;
}
