// ripple_paged_decode_attn: attention of one new token per sequence over a paged cache.
//
// Work: the cache rows of every (sequence, KV head) group are cut into tiles of kTileRows
// rows, and the tiles of all groups, in order, into one run of equal length per CTA (one
// CTA per SM): whatever the lengths, every SM streams the same number of rows, and no
// counter hands out work. Lengths are read on the device (graphs are replayed with new
// ones); each CTA finds its run by a sum over the sequences.
//
// A CTA's eight warps take the 4 KB blocks (K and V each) of a group's part in turn.
// Every warp is on its own: it fetches its blocks with asynchronous 16-byte copies into a
// ring of its own, two blocks ahead, whatever the page size and layout (a lane looks up
// the page of one row of the block, one block before it is fetched), and keeps its own
// running maximum and sum. Copies of 16 bytes and not bulk copies, because a block's rows
// need a layout that ldmatrix reads without bank conflicts, and pages may be one row.
// Rows behind a length and rows whose page is none are filled with zeros and left out by
// their place, so that what lies there never counts.
//
// bf16: warp-level matrix instructions (mma.sync: a step is bound by its bytes, and its few
// rows would leave tcgen05's 128-row tiles empty), probabilities in three bf16 parts so
// that nothing is lost against fp32, short chains in the accumulators because matrix
// instructions cut their sums off. fp32: the CUDA cores.
//
// At the end of a group's part the warps are merged through shared memory. A group that
// lies in one CTA is written; otherwise each CTA leaves its partial in the workspace and
// raises a flag, and the CTA with the group's last tiles joins them in order once it has
// finished its own run. It waits for CTAs of lower index only, which have been given
// their SMs before it, and the waits are bounded (RIPPLE_ETIMEOUT). A flag is the call's
// 64-bit tag; the reader lowers it, so that a replay of the same launch starts from
// lowered flags, and no workspace needs initialising.
#include <math.h>

#include <atomic>
#include <chrono>

#include "common.cuh"
#include "kernels.cuh"
#include "paged.cuh"
#include "warp_attn.cuh"

namespace ripple {
namespace {

constexpr int kMaxGroup = 16;
constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kBlockBytes = 4096;  // of K (and of V) a block
constexpr int kStages = 3;         // blocks in a warp's ring
constexpr int kTileRows = 64;
// A running maximum (log2 units) moves only when a score exceeds it by more than this.
constexpr float kSlack = 8.f;
constexpr unsigned kAll = 0xffffffffu;
constexpr int kMaxDevices = 64;

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
  unsigned long long *flags;  // [2 * CTAs] partials finished (the call's tag)
  float *ws_o;                // [2 * CTAs][G][D] partial outputs
  float2 *ws_ml;              // [2 * CTAs][G] their maximum and sum
  unsigned long long tag;
  long long wait_cycles;
  int n_ctas;
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
  // merge buffers of the warps; with many heads the warps share four
  static constexpr int RED = G * D > 512 ? kWarps / 2 : kWarps;
  static constexpr int PITCH = D + 8;     // floats per head in a merge buffer
  // where a piece of a row lies in the block: rows are multiples of 128 bytes, so eight rows
  // of ldmatrix, or the rows of a quarter warp, must differ in the piece
  static __device__ __forceinline__ int swizzle(int row) {
    return kMma ? row & 7 : (row * S) & 7;
  }
  static_assert(kMma || (S <= 32 && STEPS >= 1 && STEPS * R == RB && PPL >= 1), "lane layout");
};

template <typename T, int D, int G>
struct Smem {
  using C = Cfg<T, D, G>;
  alignas(128) uint8_t ring[kWarps][kStages][2][kBlockBytes];  // [stage][K, V]
  alignas(16) float red_o[C::RED][G][C::PITCH];
  float red_m[C::RED][G], red_l[C::RED][G];
  long long part[kWarps];
  long long total, rest;
  int first_seq;
  int gave_up;
};

__device__ __forceinline__ int clamp_len(const PagedDecParams &p, int b) {
  const long long room = (long long)p.g.max_pages << p.g.shift;
  const int n = p.lens[b];
  return n <= 0 ? 0 : (int)(n < room ? n : room);
}
__device__ __forceinline__ int tiles_of(int len) {
  return len / kTileRows + (len % kTileRows != 0);
}

// The first tile of CTA c's run, of `total` tiles over n CTAs; the CTA that has tile t.
__device__ __forceinline__ long long run_start(int c, long long total, int n) {
  return (long long)((unsigned long long)c * (unsigned long long)total / (unsigned)n);
}
__device__ __forceinline__ int cta_of(long long t, long long total, int n) {
  return (int)((((unsigned long long)t + 1) * (unsigned)n - 1) / (unsigned long long)total);
}

// A walk over the parts of groups in a CTA's run.
struct Walk {
  int b, h;
  int tiles, tile;     // of the group, and the part's first
  int begin, end;      // the part's rows
  long long left;      // tiles of the run, the part's included
  __device__ __forceinline__ void set(int len) {
    const long long n = min((long long)(tiles - tile), left);
    begin = tile * kTileRows;
    end = (int)min((long long)len, (tile + n) * kTileRows);
  }
  __device__ __forceinline__ int count() const {
    return (int)min((long long)(tiles - tile), left);
  }
  // To the next part; false at the end of the run.
  __device__ __forceinline__ bool next(const PagedDecParams &p) {
    left -= count();
    if (left <= 0) return false;
    tile = 0;
    if (++h < p.g.Hkv) {
      set_len(p);
      return true;
    }
    h = 0;
    do {
      ++b;
      tiles = tiles_of(clamp_len(p, b));
    } while (tiles == 0);  // left > 0: there are more
    set_len(p);
    return true;
  }
  __device__ __forceinline__ void set_len(const PagedDecParams &p) { set(clamp_len(p, b)); }
};

__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src),
               "r"(there ? 16 : 0)
               : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ unsigned long long ld_acquire64(const unsigned long long *p) {
  unsigned long long v;
  asm volatile("ld.acquire.gpu.global.b64 %0, [%1];" : "=l"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void st_release64(unsigned long long *p, unsigned long long v) {
  asm volatile("st.release.gpu.global.b64 [%0], %1;" ::"l"(p), "l"(v) : "memory");
}

// A warp's fetching side: the walk, the next block of this warp in its part, and the page
// of the lane's row in that block.
template <typename T, int D, int G>
struct Fetch {
  using C = Cfg<T, D, G>;
  Walk w;
  int blk;     // block of the part
  bool live;   // there is a next block
  int entry;   // block-table entry of row begin + blk * RB + lane % RB
  __device__ __forceinline__ void look_up(const PagedDecParams &p, int lane) {
    const int row = w.begin + blk * C::RB + lane % C::RB;
    entry = -1;
    if (row < w.end)
      entry = p.table[guard((long long)w.b * p.g.max_pages + (row >> p.g.shift), 1,
                            (long long)p.g.B * p.g.max_pages, p.status)];
  }
  // To a block of this warp at or after blk.
  __device__ __forceinline__ void settle(const PagedDecParams &p, int warp, int lane) {
    while (live && w.begin + blk * C::RB >= w.end) {
      live = w.next(p);
      blk = warp;
    }
    if (live) look_up(p, lane);
  }
  // Copies the block into `stage` and goes on; returns its live rows as bits.
  __device__ __forceinline__ uint32_t issue(const PagedDecParams &p, uint8_t (*stage)[kBlockBytes],
                                            int warp, int lane) {
    uint32_t rows = 0;
    if (live) {
      const int row = w.begin + blk * C::RB + lane % C::RB;
      const bool there = row < w.end, ok = there && (unsigned)entry < (unsigned)p.g.n_pages;
      if (there && !ok) report(p.status, RIPPLE_EBOUNDS);
      rows = __ballot_sync(kAll, ok) & (uint32_t)((1ull << C::RB) - 1);
      const long long off = ok ? entry * p.g.page_stride +
                                     (row & ((1 << p.g.shift) - 1)) * p.g.row_stride +
                                     w.h * p.g.head_stride
                               : 0;
      const uint32_t ks = smem_u32(stage[0]), vs = smem_u32(stage[1]);
#pragma unroll
      for (int j = 0; j < kBlockBytes / 512; ++j) {
        const int r = (j * 32 + lane) / C::PIECES, pc = (j * 32 + lane) % C::PIECES;
        const long long o = __shfl_sync(kAll, off, r) + pc * (16 / (int)sizeof(T));
        const uint32_t dst = r * C::ROW_BYTES + (pc ^ C::swizzle(r)) * 16;
        const bool has = rows >> r & 1;
        copy16(ks + dst, (const T *)p.k_pages + o, has);
        copy16(vs + dst, (const T *)p.v_pages + o, has);
      }
      blk += kWarps;
      settle(p, warp, lane);
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

  __device__ __forceinline__ void start(const PagedDecParams &p, const Walk &w, int lane) {
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

  __device__ __forceinline__ void start(const PagedDecParams &p, const Walk &w, int lane) {
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

// Writes a head's output element, or with lse its log of the sum.
__device__ __forceinline__ void put(const PagedDecParams &p, long long row, int D, int d, float num,
                                    float den, float M) {
  p.out[guard(row * D + d, 1, (long long)p.g.B * p.Hq * D, p.status)] =
      den != 0.f ? num / den : 0.f;  // no row counts: 0
  // den >= 2^-kSlack of the largest score's 1
  if (p.lse != nullptr && d == 0)
    p.lse[guard(row, 1, (long long)p.g.B * p.Hq, p.status)] = (M + log2f(den)) * 0.6931471805599453f;
}

template <typename T, int D, int G>
__global__ void __launch_bounds__(kThreads, 1)
    paged_decode_kernel(const __grid_constant__ PagedDecParams p) {
  using C = Cfg<T, D, G>;
  extern __shared__ __align__(128) uint8_t smem_raw[];
  Smem<T, D, G> &s = *reinterpret_cast<Smem<T, D, G> *>(smem_raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int cta = blockIdx.x;
  pdl_launch_dependents();
  pdl_wait();

  // The run of this CTA: tiles of all groups, thread by thread over the sequences.
  const int per = (p.g.B + kThreads - 1) / kThreads;
  const int b0 = min(tid * per, p.g.B), b1 = min(b0 + per, p.g.B);
  long long mine = 0;
  for (int b = b0; b < b1; ++b) {
    mine += (long long)tiles_of(clamp_len(p, b)) * p.g.Hkv;
    if (cta == 0 && (long long)p.lens[b] > (long long)p.g.max_pages << p.g.shift)
      report(p.status, RIPPLE_EFULL);
  }
  long long incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(kAll, incl, o);
    if (lane >= o) incl += y;
  }
  if (lane == 31) s.part[warp] = incl;
  __syncthreads();
  long long total = 0, before = incl - mine;
#pragma unroll
  for (int i = 0; i < kWarps; ++i) {
    if (i < warp) before += s.part[i];
    total += s.part[i];
  }
  const int n = (int)min((long long)p.n_ctas, total);
  const bool busy = cta < n;
  const long long t0 = busy ? run_start(cta, total, n) : 0;
  const long long t1 = busy ? run_start(cta + 1, total, n) : 0;
  if (busy && before <= t0 && t0 < before + mine) {
    long long rest = t0 - before;
    for (int b = b0;; ++b) {
      const long long k = (long long)tiles_of(clamp_len(p, b)) * p.g.Hkv;
      if (rest < k) {
        s.first_seq = b;
        s.rest = rest;
        break;
      }
      rest -= k;
    }
  }
  if (tid == 0) s.gave_up = 0;
  __syncthreads();

  Fetch<T, D, G> fetch = {};
  fetch.live = busy;
  if (busy) {
    Walk &w = fetch.w;
    w.b = s.first_seq;
    const int len = clamp_len(p, w.b);
    w.tiles = tiles_of(len);
    w.h = (int)(s.rest / w.tiles);
    w.tile = (int)(s.rest % w.tiles);
    w.left = t1 - t0;
    w.set(len);
  }
  Walk at = fetch.w;
  const int first_tile = at.tile;  // of the run's first part
  fetch.blk = warp;
  fetch.settle(p, warp, lane);
  uint64_t coming = 0;  // live rows of the blocks on their way, 32 bits each
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i)
    coming |= (uint64_t)fetch.issue(p, s.ring[warp][i], warp, lane) << (32 * i);
  static_assert(kStages == 3, "two blocks on their way");

  // sequences without rows
  for (int b = cta; b < p.g.B; b += gridDim.x) {
    if (clamp_len(p, b) > 0) continue;
    for (int e = tid; e < p.Hq * D; e += kThreads)
      p.out[guard((long long)b * p.Hq * D + e, 1, (long long)p.g.B * p.Hq * D, p.status)] = 0.f;
    for (int e = tid; p.lse != nullptr && e < p.Hq; e += kThreads)
      p.lse[guard((long long)b * p.Hq + e, 1, (long long)p.g.B * p.Hq, p.status)] = -INFINITY;
  }
  if (!busy) return;

  int stage = 0;
  bool joins = false;  // this CTA joins the partials of its first part's group
  Walk first = at;
  for (bool more = true; more;) {
    Rows<T, D, G> rows;
    rows.start(p, at, lane);
    for (int blk = warp; at.begin + blk * C::RB < at.end; blk += kWarps) {
      copy_wait<kStages - 2>();
      __syncwarp();  // the block has landed, and the stage before it has been read
      const uint32_t live = (uint32_t)coming;
      const int fill = stage + kStages - 1 < kStages ? stage + kStages - 1 : stage - 1;
      coming = coming >> 32 | (uint64_t)fetch.issue(p, s.ring[warp][fill], warp, lane) << 32;
      rows.block(p, s.ring[warp][stage], live, lane);
      stage = stage + 1 < kStages ? stage + 1 : 0;
    }
    rows.finish();

    // The warps of the part, through shared memory, as many at a time as there are buffers.
    constexpr int NE = (G * D + kThreads - 1) / kThreads;
    float M[NE], num[NE], den[NE];
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      M[i] = -INFINITY;
      num[i] = den[i] = 0.f;
    }
#pragma unroll
    for (int turn = 0; turn < kWarps / C::RED; ++turn) {
      named_bar_sync(1, kThreads);  // the buffers have been read
      if (warp / C::RED == turn) {
        const int buf = warp % C::RED;
        rows.stats(lane, [&](int head, float m, float l) {
          s.red_m[buf][head] = m;
          s.red_l[buf][head] = l;
        });
        rows.outputs(lane, [&](int head, int d, const float2 &o) {
          *reinterpret_cast<float2 *>(&s.red_o[buf][head][d]) = o;
        });
      }
      named_bar_sync(1, kThreads);
#pragma unroll
      for (int i = 0; i < NE; ++i) {
        const int e = tid + i * kThreads, head = e / D;
        if (e >= p.G * D) continue;
        float top = M[i];
#pragma unroll
        for (int w = 0; w < C::RED; ++w) top = fmaxf(top, s.red_m[w][head]);
        const float sub = top == -INFINITY ? 0.f : top;
        const float old = fast_exp2(M[i] - sub);
        num[i] *= old;
        den[i] *= old;
        M[i] = top;
#pragma unroll
        for (int w = 0; w < C::RED; ++w) {
          const float a = fast_exp2(s.red_m[w][head] - sub);
          num[i] += a * s.red_o[w][head][e % D];
          den[i] += a * s.red_l[w][head];
        }
      }
    }
    const bool whole = at.tile == 0 && at.count() == at.tiles;
    const int slot = 2 * cta + (at.tile == 0 ? 1 : 0);
    const long long row0 = (long long)at.b * p.Hq + at.h * p.G;
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      const int e = tid + i * kThreads, head = e / D, d = e % D;
      if (e >= p.G * D) continue;
      if (whole) {
        put(p, row0 + head, D, d, num[i], den[i], M[i]);
      } else {
        const long long at_slot =
            guard((long long)slot * p.G + head, 1, 2LL * p.n_ctas * p.G, p.status);
        p.ws_o[at_slot * D + d] = num[i];
        if (d == 0) p.ws_ml[at_slot] = make_float2(M[i], den[i]);
      }
    }
    if (!whole) {
      const bool last = at.tile + at.count() == at.tiles;
      if (last) {
        joins = true;
      } else {
        __threadfence();
        named_bar_sync(1, kThreads);
        if (tid == 0) st_release64(&p.flags[slot], p.tag);
      }
    }
    more = at.next(p);
  }
  copy_wait<0>();

  if (!joins) return;
  // The partials of the first part's group: of the CTA with its first tile (a part that
  // begins the group), of those between, and this CTA's own.
  const long long group_start = t0 - first_tile;
  const int c0 = cta_of(group_start, total, n);
  const int parts = cta - c0 + 1;
  for (int i = tid; i < parts - 1; i += kThreads) {
    unsigned long long *flag = &p.flags[2 * (c0 + i) + (i == 0 ? 1 : 0)];
    const long long from = clock64();
    bool up;
    while (!(up = ld_acquire64(flag) == p.tag) && clock64() - from <= p.wait_cycles) __nanosleep(20);
    if (up) {
      *flag = 0;  // a replay of this launch starts from lowered flags
    } else {
      report(p.status, RIPPLE_ETIMEOUT);
      s.gave_up = 1;
    }
  }
  __threadfence();
  __syncthreads();
  if (s.gave_up) return;
  const long long row0 = (long long)first.b * p.Hq + first.h * p.G;
  constexpr int kAt = 8;  // partials loaded at a time
  for (int e = tid; e < p.G * D; e += kThreads) {
    const int head = e / D, d = e % D;
    float M = -INFINITY, num = 0.f, den = 0.f;
    for (int i0 = 0; i0 < parts; i0 += kAt) {
      float2 ml[kAt];
      float o[kAt];
#pragma unroll
      for (int i = 0; i < kAt; ++i) {
        const int c = min(i0 + i, parts - 1);
        const long long slot = 2 * (c0 + c) + (c == 0 ? 1 : 0);
        ml[i] = __ldcg(&p.ws_ml[slot * p.G + head]);
        o[i] = __ldcg(&p.ws_o[(slot * p.G + head) * D + d]);
        if (i0 + i >= parts) {
          ml[i] = make_float2(-INFINITY, 0.f);
          o[i] = 0.f;
        }
      }
      float Mn = M;
#pragma unroll
      for (int i = 0; i < kAt; ++i) Mn = fmaxf(Mn, ml[i].x);
      const float sub = Mn == -INFINITY ? 0.f : Mn, a = fast_exp2(M - sub);
      num *= a;
      den *= a;
      M = Mn;
#pragma unroll
      for (int i = 0; i < kAt; ++i) {
        const float w = fast_exp2(ml[i].x - sub);
        den += w * ml[i].y;
        num += w * o[i];
      }
    }
    put(p, row0 + head, D, d, num, den, M);
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

// Tag of a call: a sequence, never 0, from a start taken from the clock, so that a flag
// left in reused memory by an earlier call or process does not match.
unsigned long long next_tag() {
  static std::atomic<unsigned long long> seq{
      (unsigned long long)std::chrono::steady_clock::now().time_since_epoch().count() *
      0x9e3779b97f4a7c15ULL};
  unsigned long long t;
  do t = seq.fetch_add(1, std::memory_order_relaxed) + 1;
  while (t == 0);
  return t;
}

size_t round_up(size_t x) { return (x + 255) & ~(size_t)255; }

bool decode_args(const ripple_paged_desc *d, int n_q_heads, PagedDecParams *p) {
  if (!paged_geom(d, &p->g)) return false;
  if (n_q_heads < 1 || n_q_heads % d->n_kv_heads != 0) return false;
  p->Hq = n_q_heads;
  p->G = n_q_heads / d->n_kv_heads;
  return p->G <= kMaxGroup;
}

// Workspace layout: flags, (max, sum), outputs, two partials per CTA at most (the first
// and the last part of its run). Returns the bytes; fills p's pointers if given a base.
size_t plan(PagedDecParams *p, int sms, void *ws) {
  const size_t slots = 2 * (size_t)sms;
  const size_t flags = round_up(slots * sizeof(unsigned long long));
  const size_t ml = round_up(slots * p->G * sizeof(float2));
  uint8_t *base = (uint8_t *)ws;
  p->n_ctas = sms;
  p->flags = (unsigned long long *)base;
  p->ws_ml = (float2 *)(base + flags);
  p->ws_o = (float *)(base + flags + ml);
  return flags + ml + round_up(slots * p->G * p->g.D * sizeof(float));
}

template <typename T, int D, int G>
cudaError_t launch(const PagedDecParams &p, int dev, cudaStream_t st) {
  static std::atomic<bool> attr_set[kMaxDevices];
  constexpr int smem = (int)sizeof(Smem<T, D, G>);
  static_assert(smem <= 227 * 1024, "shared memory per CTA");
  if (!attr_set[dev].load(std::memory_order_acquire)) {
    const cudaError_t e = cudaFuncSetAttribute(paged_decode_kernel<T, D, G>,
                                               cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    attr_set[dev].store(true, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.n_ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, paged_decode_kernel<T, D, G>, p);
  count_launches(1);
  return e;
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
  *bytes_host = plan(&p, sm_count(dev), nullptr);
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
  int dev = 0;
  const cudaError_t got = cudaGetDevice(&dev);
  if (got != cudaSuccess || dev < 0 || dev >= kMaxDevices) dev = 0;
  if (workspace_bytes < plan(&p, sm_count(dev), workspace)) return RIPPLE_EWORKSPACE;
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
  p.tag = next_tag();
  p.wait_cycles = wait_limit_cycles();
  cudaStream_t st = (cudaStream_t)stream;
  RIPPLE_CUDA_TRY(desc->head_dim == 128 ? launch_d<128>(p, desc->dtype, dev, st)
                                        : launch_d<64>(p, desc->dtype, dev, st));
  return RIPPLE_OK;
}
