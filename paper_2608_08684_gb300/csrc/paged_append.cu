// ripple_paged_append and ripple_paged_append_q8: new tokens' keys and values into a paged
// cache, keys and queries rotated to their positions on the way, one pass over q, k and v.
//
// Rotation: the angle pos * inv_freq is only needed modulo a turn. The host gives
// f_j = inv_freq_j / (2 pi) as a 64-bit fraction of a turn (modulo one turn, to
// nearest); pos * f_j in wrapping 64-bit integers is then the angle modulo a turn, off
// by at most 2^31 * 2^-65 turns at the farthest int32 position, where a product in
// fp32 would be off by whole turns. Its upper 32 bits are split into the nearest
// quarter turn and a rest of at most an eighth, exact in 30 bits, so that the fp32
// sine and cosine see an argument rounded by 2^-25 of 1/4 at most.
//
// Work: a head's d elements are spread over d / 16 lanes, each with the two 16-byte
// (fp32: 32-byte) pieces that hold eight pairs, so that the eight sines and cosines
// of a lane serve every head of the token that its warp takes (the lanes that need the
// same eight compute them together). A token's Hq + 2 Hkv head rows are cut into groups
// of 32 / (d / 16) rows, one per warp step; with few tokens every warp takes one group,
// with many a warp takes several, the loads of kAhead of them in flight at a time.
// 8-bit pages: the lanes of a head row, which all have it in registers as fp32, find its
// largest magnitude by shuffles (as integers, so that NaNs count as the largest), and each
// writes 16 codes. The scale is a power of two, so that scaling rounds nothing.
#include <cuda_fp8.h>
#include <math.h>

#include "common.cuh"
#include "kernels.cuh"
#include "paged.cuh"

namespace ripple {
namespace {

constexpr int kAppendWarps = 4;  // per CTA (8: 142 us for 33.6k tokens of 48 head rows; 4: 131)
constexpr int kMaxPairs = 64;

struct TokenRows {
  const void *data;
  long long seq, token, head;  // strides, elements
};

struct AppendParams {
  PagedGeom g;
  int Hq, n_tokens, per_seq;   // per_seq: tokens of every sequence, 0 with seq_starts
  int rot;                     // 0: no rotation
  int groups, per_warp, warps; // groups of head rows a token, of a warp, warps a token
  TokenRows q, k, v, q_out;
  const int32_t *starts, *positions, *table, *lens;
  void *k_pages, *v_pages;
  ScaleGeom sc;                // 8-bit pages
  int32_t *status;
  unsigned long long freq[kMaxPairs];  // turns per position, times 2^64
};

// 8 elements as they lie in memory.
template <typename T>
struct Raw8 {
  uint4 u[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ Raw8<T> load_raw(const T *p) {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.u[i] = reinterpret_cast<const uint4 *>(p)[i];
  return r;
}
template <typename T>
__device__ __forceinline__ void store_raw(T *p, const Raw8<T> &r) {
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4 *>(p)[i] = r.u[i];
}
__device__ __forceinline__ void unpack(const Raw8<float> &r, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    x[4 * i] = __uint_as_float(r.u[i].x);
    x[4 * i + 1] = __uint_as_float(r.u[i].y);
    x[4 * i + 2] = __uint_as_float(r.u[i].z);
    x[4 * i + 3] = __uint_as_float(r.u[i].w);
  }
}
__device__ __forceinline__ void unpack(const Raw8<__nv_bfloat16> &r, float (&x)[8]) {
  const uint32_t w[4] = {r.u[0].x, r.u[0].y, r.u[0].z, r.u[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void pack(const float (&x)[8], Raw8<float> &r) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
    r.u[i] = make_uint4(__float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]),
                        __float_as_uint(x[4 * i + 2]), __float_as_uint(x[4 * i + 3]));
}
// the one rounding of a stored value: to nearest even in the cache's type
__device__ __forceinline__ void pack(const float (&x)[8], Raw8<__nv_bfloat16> &r) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t *>(&h);
  }
  r.u[0] = make_uint4(w[0], w[1], w[2], w[3]);
}

// The scale byte of a row whose largest magnitude has these bits: the least e >= -120 with
// it <= 448 2^e = 1.75 2^(e + 8), plus 127; 255 for an infinity or a NaN.
__device__ __forceinline__ int scale_byte(uint32_t most) {
  if (most >= 0x7f800000u) return 255;
  const int e = (int)(most >> 23) - 127 - 8 + ((most & 0x7fffffu) > 0x600000u);
  return max(e, -120) + 127;
}
// Eight values over the scale, to nearest even in e4m3. (247: 256 2^120 would be infinite.)
__device__ __forceinline__ uint2 codes_of(const float (&x)[8], int byte) {
  if (byte == 255) return make_uint2(0, 0);
  const float f = __int_as_float((254 - byte) << 23);
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float lo = x[2 * i] * f, hi = x[2 * i + 1] * f;
    if (byte == 247) {
      lo = fminf(fmaxf(lo, -240.f), 240.f);
      hi = fminf(fmaxf(hi, -240.f), 240.f);
    }
    const uint32_t c = __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
    w[i / 2] |= c << (16 * (i & 1));
  }
  return make_uint2(w[0], w[1]);
}

// Cosine and sine of `turns` / 2^64 turns.
__device__ __forceinline__ void cos_sin(unsigned long long turns, float &c, float &s) {
  const uint32_t x = (uint32_t)(turns >> 32);
  const uint32_t quarter = (x + 0x20000000u) >> 30;
  const int rest = (int)(x - (quarter << 30));  // in [-2^29, 2^29): an eighth of a turn at most
  float sr, cr;
  sincospif((float)rest * 0x1p-31f, &sr, &cr);  // half turns
  const float a = quarter & 1 ? sr : cr, b = quarter & 1 ? cr : sr;
  c = (quarter + 1) & 2 ? -a : a;
  s = quarter & 2 ? -b : b;
}

// The last sequence b < B with starts[b] <= t, or -1, by one warp: every step compares 32
// entries, equally spaced in what is left.
__device__ __forceinline__ int find_seq(const int32_t *starts, int B, int t, int lane) {
  int lo = 0, n = B;  // the answer lies in [lo, lo + n)
  for (;;) {
    const int step = (n + 31) / 32;
    const bool le = lane * step < n && starts[lo + lane * step] <= t;
    const int k = __popc(__ballot_sync(0xffffffffu, le));
    if (k == 0) return -1;
    const int at = (k - 1) * step;
    if (step == 1) return lo + at;
    lo += at;
    n = min(step, n - at);
  }
}

// kAhead: groups whose loads are in flight at a time. kCodes: 8-bit pages.
template <typename T, int D, bool kInter, int kAhead, bool kCodes>
__global__ void __launch_bounds__(kAppendWarps * 32, kCodes && sizeof(T) == 2 ? 8 : 0)
    append_kernel(const __grid_constant__ AppendParams p) {
  constexpr int kLanes = D / 16;       // lanes per head row
  constexpr int kRows = 32 / kLanes;   // head rows per warp step
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const unsigned w = blockIdx.x * (unsigned)kAppendWarps + (threadIdx.x >> 5);
  const int t = (int)(w / (unsigned)p.warps), part = (int)(w % (unsigned)p.warps);
  if (t >= p.n_tokens) return;
  const int l = lane % kLanes, sub = lane / kLanes;
  const bool turns = l < p.rot / 16;
  const int o0 = turns && !kInter ? 8 * l : 16 * l;
  const int o1 = turns && !kInter ? p.rot / 2 + 8 * l : 16 * l + 8;
  const int n_rows = p.Hq + 2 * p.g.Hkv;
  int b = 0, i = t;  // of seq_starts: found below
  if (p.per_seq > 0) {
    b = t / p.per_seq;
    i = t - b * p.per_seq;
  }

  // The rows of kAhead groups from g on, as they are.
  const int g_end = min(p.groups, (part + 1) * p.per_warp);
  Raw8<T> x[kAhead], y[kAhead];
  auto load = [&](int g, int b, int i) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int r = (g + u) * kRows + sub;
      if (g + u >= g_end || r >= n_rows) continue;
      const bool is_q = r < p.Hq, is_v = r >= p.Hq + p.g.Hkv;
      const TokenRows &src = is_q ? p.q : is_v ? p.v : p.k;
      const int h = is_q ? r : is_v ? r - p.Hq - p.g.Hkv : r - p.Hq;
      const T *from = (const T *)src.data + b * src.seq + i * src.token + h * src.head;
      x[u] = load_raw(from + o0);
      y[u] = load_raw(from + o1);
    }
  };
  // where a token lies does not depend on its sequence with seq_starts (strides by t alone)
  const int src_b = b, src_i = i;
  int g = part * p.per_warp;
  load(g, src_b, src_i);

  // the token's sequence, cache row and position
  int n_b = p.per_seq;
  if (p.per_seq == 0) {
    b = find_seq(p.starts, p.g.B, t, lane);
    if (b < 0) return;
    const int s0 = p.starts[b], s1 = p.starts[b + 1];
    if (t >= s1) return;  // behind the last token
    i = t - s0;
    n_b = s1 - s0;
  }
  const int len = p.lens[b];
  const long long row = (long long)len - n_b + i;
  const long long pos = p.positions != nullptr ? (long long)p.positions[t] : row;
  int32_t bad = 0;
  long long place = -1;  // element offset of the row, head 0
  long long scale_at = 0;
  if (len > 0) {
    const long long pg = row >> p.g.shift;
    if (row < 0) {
      bad = RIPPLE_EBOUNDS;
    } else if (pg >= p.g.max_pages) {
      bad = RIPPLE_EFULL;
    } else {
      const int page = p.table[guard((long long)b * p.g.max_pages + pg, 1,
                                     (long long)p.g.B * p.g.max_pages, p.status)];
      if ((unsigned)page >= (unsigned)p.g.n_pages)
        bad = RIPPLE_EBOUNDS;
      else {
        const long long slot = row & ((1 << p.g.shift) - 1);
        place = guard(page, 1, p.g.n_pages, p.status) * p.g.page_stride + slot * p.g.row_stride;
        if (kCodes)
          scale_at = guard(page, 1, p.g.n_pages, p.status) * p.sc.page_stride +
                     slot * p.sc.row_stride;
      }
    }
  }
  if (bad != 0 && part == 0 && lane == 0) report(p.status, bad);

  // Eight sines and cosines for every lane of the same l: each of the kRows lanes of that
  // l computes its share.
  float c[8], s[8];
  {
    constexpr int kShare = 8 / kRows;  // 2 (d = 128) or 1 (d = 64)
    float cs[kShare], sn[kShare];
#pragma unroll
    for (int j = 0; j < kShare; ++j) {
      cs[j] = 1.f;
      sn[j] = 0.f;
      if (turns) cos_sin((unsigned long long)pos * p.freq[8 * l + sub * kShare + j], cs[j], sn[j]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      c[j] = __shfl_sync(0xffffffffu, cs[j % kShare], j / kShare * kLanes + l);
      s[j] = __shfl_sync(0xffffffffu, sn[j % kShare], j / kShare * kLanes + l);
    }
  }

  auto turn = [&](float (&a)[8], float (&d)[8]) {
    if (kInter) {  // pairs (0, 1), (2, 3), .. of the 16 elements a, d
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float a0 = a[2 * j], a1 = a[2 * j + 1], d0 = d[2 * j], d1 = d[2 * j + 1];
        a[2 * j] = a0 * c[j] - a1 * s[j];
        a[2 * j + 1] = a1 * c[j] + a0 * s[j];
        d[2 * j] = d0 * c[4 + j] - d1 * s[4 + j];
        d[2 * j + 1] = d1 * c[4 + j] + d0 * s[4 + j];
      }
    } else {  // pairs (a_j, d_j)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float a0 = a[j], d0 = d[j];
        a[j] = a0 * c[j] - d0 * s[j];
        d[j] = d0 * c[j] + a0 * s[j];
      }
    }
  };
  for (;;) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int r = (g + u) * kRows + sub;
      if (g + u >= g_end || r >= n_rows) continue;
      const bool is_q = r < p.Hq, is_v = r >= p.Hq + p.g.Hkv;
      if (!is_q && place < 0) continue;
      const int h = is_q ? r : is_v ? r - p.Hq - p.g.Hkv : r - p.Hq;
      if constexpr (kCodes) {
        if (!is_q) {
          float a[8], d[8];
          unpack(x[u], a);
          unpack(y[u], d);
          if (turns && !is_v) turn(a, d);
          uint32_t most = 0;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            most = max(most, max(__float_as_uint(a[j]) & 0x7fffffffu, __float_as_uint(d[j]) & 0x7fffffffu));
          const uint32_t row_lanes = ((1u << kLanes) - 1) << (sub * kLanes);
#pragma unroll
          for (int o = 1; o < kLanes; o <<= 1) most = max(most, __shfl_xor_sync(row_lanes, most, o));
          const int byte = scale_byte(most);
          uint8_t *to = (uint8_t *)(is_v ? p.v_pages : p.k_pages) + place + h * p.g.head_stride;
          *reinterpret_cast<uint2 *>(to + o0) = codes_of(a, byte);
          *reinterpret_cast<uint2 *>(to + o1) = codes_of(d, byte);
          if (l == 0) (is_v ? p.sc.v : p.sc.k)[scale_at + h * p.sc.head_stride] = (uint8_t)byte;
          continue;
        }
      }
      T *to = is_q ? (T *)p.q_out.data + src_b * p.q_out.seq + src_i * p.q_out.token +
                         h * p.q_out.head
                   : (T *)(is_v ? p.v_pages : p.k_pages) + place + h * p.g.head_stride;
      if (turns && !is_v) {
        float a[8], d[8];
        unpack(x[u], a);
        unpack(y[u], d);
        turn(a, d);
        pack(a, x[u]);
        pack(d, y[u]);
      }
      store_raw(to + o0, x[u]);
      store_raw(to + o1, y[u]);
    }
    g += kAhead;
    if (g >= g_end) break;
    load(g, src_b, src_i);
  }
}

// inv_freq / (2 pi) turns modulo one, times 2^64, to nearest. |inv_freq| <= 1024.
unsigned long long to_turns(double inv_freq) {
  int e;
  const double m = frexp(fabs(inv_freq), &e);  // inv_freq = m 2^e, m in [1/2, 1)
  const unsigned long long mant = (unsigned long long)ldexp(m, 53);  // inv_freq = mant 2^(e - 53)
  // 1 / (2 pi) to 128 bits, from the digits of pi
  const unsigned long long hi = 0x28be60db9391054aULL, lo = 0x7f09d5f47d4d3770ULL;
  // mant / (2 pi) * 2^64, to 117 bits
  const unsigned __int128 prod =
      (unsigned __int128)mant * hi + (unsigned __int128)(((unsigned __int128)mant * lo) >> 64);
  const int down = 53 - e;  // >= 42, as e <= 11
  if (down > 126) return 0;
  const unsigned __int128 r = (prod >> down) + ((prod >> (down - 1)) & 1);
  const unsigned long long turns = (unsigned long long)r;
  return inv_freq < 0 ? 0ULL - turns : turns;
}

// A programmatic dependent of the kernel before it, as that one ends: without a trigger in
// it, since CTAs that wait in its SMs cost more (a batch of 108 tokens 5.2 us from a graph,
// 3.7 without) than an earlier start gains (one token 2.9, 3.0).
template <typename T, int D, bool kInter, int kAhead, bool kCodes>
cudaError_t launch_as(const AppendParams &p, int grid, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kAppendWarps * 32);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, append_kernel<T, D, kInter, kAhead, kCodes>, p);
  count_launches(1);
  return e;
}

template <typename T, int D, bool kCodes>
cudaError_t launch(const AppendParams &p, bool inter, int grid, cudaStream_t st) {
  // 4 to 8 loads of a lane in flight. Over 8-bit pages more warps with fewer loads each do better
  // (65.6k tokens of 48 head rows: one group at 64 registers 246 us, 86% of the copy rate, at 72 255; two
  // at 64 252, at 72 267).
  constexpr int kMany = kCodes ? 1 : sizeof(T) == 2 && D == 64 ? 4 : 2;
  if (kMany == 1 || p.per_warp == 1)
    return inter ? launch_as<T, D, true, 1, kCodes>(p, grid, st)
                 : launch_as<T, D, false, 1, kCodes>(p, grid, st);
  return inter ? launch_as<T, D, true, kMany, kCodes>(p, grid, st)
               : launch_as<T, D, false, kMany, kCodes>(p, grid, st);
}

template <bool kCodes>
cudaError_t launch_any(const AppendParams &p, int dtype, bool inter, int grid, cudaStream_t st) {
  if (dtype == RIPPLE_BF16)
    return p.g.D == 128 ? launch<__nv_bfloat16, 128, kCodes>(p, inter, grid, st)
                        : launch<__nv_bfloat16, 64, kCodes>(p, inter, grid, st);
  return p.g.D == 128 ? launch<float, 128, kCodes>(p, inter, grid, st)
                      : launch<float, 64, kCodes>(p, inter, grid, st);
}

// A tensor of tokens: pointer and strides in place.
bool token_rows(const void *data, const ripple_token_strides *s, int vec, TokenRows *out) {
  if (data == nullptr || s == nullptr || !aligned16_host(data)) return false;
  for (const int64_t x : {s->seq_stride, s->token_stride, s->head_stride})
    if (x < 0 || x > (1LL << 40) || x % vec != 0) return false;
  *out = TokenRows{data, s->seq_stride, s->token_stride, s->head_stride};
  return true;
}

// The rows of a tensor of tokens with `heads` heads; spans beyond 2^48 elements, which no
// tensor has, are refused.
bool row_set(const TokenRows &t, const AppendParams &p, int heads, int elem, RowSet *out) {
  *out = RowSet{(long long)((uintptr_t)t.data / elem),
                {t.seq, t.token, t.head},
                {p.per_seq > 0 ? p.g.B : 1, p.per_seq > 0 ? p.per_seq : p.n_tokens, heads}};
  for (int i = 0; i < 3; ++i)
    if (out->count[i] > 1 && out->stride[i] > (1LL << 48) / out->count[i]) return false;
  return true;
}

// scales: NULL for pages in desc->dtype.
ripple_status append(
    const ripple_paged_desc *desc, const ripple_paged_scales *scales, const ripple_rope *rope,
    int32_t n_tokens,
    const int32_t *seq_starts, int32_t n_q_heads, const void *q,
    const ripple_token_strides *q_strides, void *q_out, const ripple_token_strides *q_out_strides,
    const void *k, const ripple_token_strides *k_strides, const void *v,
    const ripple_token_strides *v_strides, const int32_t *positions, void *k_pages, void *v_pages,
    const int32_t *block_table, const int32_t *lens, int32_t *dev_status, void *stream) {
  AppendParams p;
  const bool codes = scales != nullptr;
  p.sc = ScaleGeom{};
  if (!paged_geom(desc, &p.g, codes) || (codes && !scale_geom(desc, scales, &p.sc)) || n_tokens < 0)
    return RIPPLE_EINVAL;
  if (seq_starts == nullptr && n_tokens % desc->batch != 0) return RIPPLE_EINVAL;
  if ((q == nullptr) != (q_out == nullptr)) return RIPPLE_EINVAL;
  p.rot = 0;
  bool inter = false;
  if (rope != nullptr) {
    if (rope->rot_dim < 16 || rope->rot_dim > desc->head_dim || rope->rot_dim % 16 != 0 ||
        (rope->interleaved != 0 && rope->interleaved != 1) || rope->inv_freq_host == nullptr)
      return RIPPLE_EINVAL;
    for (int j = 0; j < rope->rot_dim / 2; ++j) {
      if (!(fabs(rope->inv_freq_host[j]) <= 1024.0)) return RIPPLE_EINVAL;
      p.freq[j] = to_turns(rope->inv_freq_host[j]);
    }
    p.rot = rope->rot_dim;
    inter = rope->interleaved != 0;
  }
  if (n_tokens == 0) return RIPPLE_OK;
  if (!k_pages || !v_pages || !block_table || !lens || !aligned16_host(k_pages) ||
      !aligned16_host(v_pages))
    return RIPPLE_EINVAL;
  if (!aligned4_host({seq_starts, positions, block_table, lens, dev_status})) return RIPPLE_EINVAL;
  const int vec = vec_elems(desc->dtype);
  if (!token_rows(k, k_strides, vec, &p.k) || !token_rows(v, v_strides, vec, &p.v))
    return RIPPLE_EINVAL;
  p.Hq = 0;
  p.q = p.q_out = TokenRows{};
  p.n_tokens = n_tokens;
  p.per_seq = seq_starts == nullptr ? n_tokens / desc->batch : 0;
  // What one warp reads no other may write: the queries' places lie apart from each other's, the
  // keys' and the values', and the pools from each other.
  const int elem = 16 / vec;
  RowSet in[3], to;  // q, k, v; q_out
  if (!row_set(p.k, p, p.g.Hkv, elem, &in[1]) || !row_set(p.v, p, p.g.Hkv, elem, &in[2]))
    return RIPPLE_EINVAL;
  if (q != nullptr) {
    if (n_q_heads < 1 || n_q_heads > (1 << 16)) return RIPPLE_EINVAL;
    if (!token_rows(q, q_strides, vec, &p.q) || !token_rows(q_out, q_out_strides, vec, &p.q_out))
      return RIPPLE_EINVAL;
    if (q == q_out && (p.q.seq != p.q_out.seq || p.q.token != p.q_out.token ||
                       p.q.head != p.q_out.head))
      return RIPPLE_EINVAL;
    if (!row_set(p.q, p, n_q_heads, elem, &in[0]) ||
        !row_set(p.q_out, p, n_q_heads, elem, &to) ||
        !disjoint(3, to.stride, to.count, desc->head_dim))
      return RIPPLE_EINVAL;
    for (int i = q == q_out ? 1 : 0; i < 3; ++i)
      if (overlap(in[i], to, desc->head_dim)) return RIPPLE_EINVAL;
    p.Hq = n_q_heads;
  }
  const int page_elem = codes ? 1 : elem;
  const RowSet pool[2] = {p.g.rows(k_pages, page_elem), p.g.rows(v_pages, page_elem)};
  if (overlap(pool[0], pool[1], desc->head_dim)) return RIPPLE_EINVAL;
  if (codes) {
    const RowSet sc[2] = {p.sc.rows(p.sc.k, p.g), p.sc.rows(p.sc.v, p.g)};
    if (overlap(sc[0], sc[1], 1)) return RIPPLE_EINVAL;
    for (int i = 0; i < 4; ++i)
      if (overlap(pool[i / 2], sc[i % 2], desc->head_dim, 1)) return RIPPLE_EINVAL;
  }
  p.starts = seq_starts;
  p.positions = positions;
  p.table = block_table;
  p.lens = lens;
  p.k_pages = k_pages;
  p.v_pages = v_pages;
  p.status = dev_status;
  const int rows = 32 / (desc->head_dim / 16);
  p.groups = (p.Hq + 2 * p.g.Hkv + rows - 1) / rows;
  // one group a warp while all warps find a place at once, then more
  constexpr int kPlaces = 152 * 32;
  const long long steps = (long long)n_tokens * p.groups;
  p.warps = (int)std::max<long long>(1, std::min<long long>(p.groups, kPlaces * (long long)p.groups / steps));
  p.per_warp = (p.groups + p.warps - 1) / p.warps;
  p.warps = (p.groups + p.per_warp - 1) / p.per_warp;
  const long long ctas = ((long long)n_tokens * p.warps + kAppendWarps - 1) / kAppendWarps;
  if (ctas > 0x7fffffffLL / kAppendWarps) return RIPPLE_EINVAL;
  cudaStream_t st = (cudaStream_t)stream;
  RIPPLE_CUDA_TRY(codes ? launch_any<true>(p, desc->dtype, inter, (int)ctas, st)
                        : launch_any<false>(p, desc->dtype, inter, (int)ctas, st));
  return RIPPLE_OK;
}

}  // namespace
}  // namespace ripple

using namespace ripple;

extern "C" ripple_status ripple_paged_append(
    const ripple_paged_desc *desc, const ripple_rope *rope, int32_t n_tokens,
    const int32_t *seq_starts, int32_t n_q_heads, const void *q,
    const ripple_token_strides *q_strides, void *q_out, const ripple_token_strides *q_out_strides,
    const void *k, const ripple_token_strides *k_strides, const void *v,
    const ripple_token_strides *v_strides, const int32_t *positions, void *k_pages, void *v_pages,
    const int32_t *block_table, const int32_t *lens, int32_t *dev_status, void *stream) {
  return append(desc, nullptr, rope, n_tokens, seq_starts, n_q_heads, q, q_strides, q_out,
                q_out_strides, k, k_strides, v, v_strides, positions, k_pages, v_pages, block_table,
                lens, dev_status, stream);
}

extern "C" ripple_status ripple_paged_append_q8(
    const ripple_paged_desc *desc, const ripple_paged_scales *scales, const ripple_rope *rope,
    int32_t n_tokens,
    const int32_t *seq_starts, int32_t n_q_heads, const void *q,
    const ripple_token_strides *q_strides, void *q_out, const ripple_token_strides *q_out_strides,
    const void *k, const ripple_token_strides *k_strides, const void *v,
    const ripple_token_strides *v_strides, const int32_t *positions, void *k_pages, void *v_pages,
    const int32_t *block_table, const int32_t *lens, int32_t *dev_status, void *stream) {
  if (scales == nullptr) return RIPPLE_EINVAL;
  return append(desc, scales, rope, n_tokens, seq_starts, n_q_heads, q, q_strides, q_out,
                q_out_strides, k, k_strides, v, v_strides, positions, k_pages, v_pages, block_table,
                lens, dev_status, stream);
}
