// ripple_paged_tree_attn: attention of a tree of drafted tokens per sequence over a paged
// cache. Entry points, the kernel on the CUDA cores (fp32 queries) and the join.
//
// fp32: a CTA of four warps has 32 query rows and takes blocks of 32 keys. Scores: a thread
// has 4 rows x 2 keys, outputs: 4 rows x D / 16 dims, both from shared memory by 16 bytes; the
// next block's rows are loaded into registers meanwhile. A row's 16 threads are half a warp, so its
// maximum and sum are shuffles. The cache's bytes are 8 d a row and the FMAs 2 n G d: above a few rows
// a KV head the instructions bound it, about 1400 a warp and block of 64 dims, of which 512 are FMAs, two
// of them in each. Every row tile is a group of its own (sequences of few tokens have fewer tiles, and CTAs
// of all tiles would idle beside them). 7 sequences of up to 6000 rows, 1 to 9 tokens of 28 heads on 4,
// d 64: 40.5 us (four and five CTAs an SM at 128 and 96 registers: 41.2 and 45.4).
#include "paged_tree.cuh"

#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <atomic>

namespace ripple {
namespace {

constexpr int kMaxDevices = 64;
constexpr int kThreads = 128;
constexpr int R = kTreeSimtRows, KB = kTreeSimtKeys;
constexpr float kSlack = 8.f;
// Blocks that a group's queries and outputs take as long as (0, 1, 2, 4: 41.6, 40.2, 40.1, 40.4 us for the
// batch above, 29.4, 26.5, 29.7, 28.9 for 54 sequences of up to 148 rows and 43 tokens).
constexpr int kGroupCost = 1;

// 16 bytes of a page's row: 4 fp32 values, or 16 codes.
template <typename T>
struct Piece;
template <>
struct Piece<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void put(float *to, const uint4 &u, float) {
    *reinterpret_cast<uint4 *>(to) = u;
  }
};
template <>
struct Piece<uint8_t> {
  static constexpr int N = 16;
  static __device__ __forceinline__ void put(float *to, const uint4 &u, float scale) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float x[4];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const __half2_raw h =
            __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i] >> (16 * j)), __NV_E4M3);
        const float2 f = __half22float2(__half2(h));
        x[2 * j] = f.x * scale;
        x[2 * j + 1] = f.y * scale;
      }
      *reinterpret_cast<float4 *>(to + 4 * i) = make_float4(x[0], x[1], x[2], x[3]);
    }
  }
};

template <int D>
struct SimtSmem {
  static constexpr int LD = D + 4;  // rows of a quarter warp start in other banks
  float q[R][LD], k[KB][LD], v[KB][D];
  float p[KB][R + 4];   // probabilities; negative: the key is hidden from the row
  uint64_t mask[R];
};

__device__ __forceinline__ float scale_of_byte(int s) {
  return s == 255 ? __int_as_float(0x7fffffff) : __int_as_float(s << 23);  // (7..247)
}

// T: float, or uint8_t for codes. Queries and outputs fp32.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads, kTreeSimtCtas)
    tree_simt_kernel(const __grid_constant__ TreeParams p) {
  using P = Piece<T>;
  using W = TreeWalk<KB, kGroupCost, R>;
  constexpr int kPieces = D / P::N;                        // of a row
  constexpr int kMine = KB * kPieces / kThreads;           // of a block's keys, a thread
  constexpr bool kCodes = sizeof(T) == 1;
  constexpr int DT = D / 16;                               // output dims of a thread
  extern __shared__ __align__(16) uint8_t smem_raw[];
  SimtSmem<D> &s = *reinterpret_cast<SimtSmem<D> *>(smem_raw);
  static_assert(KB * kPieces % kThreads == 0, "");
  const int tid = threadIdx.x, lane = tid & 31;
  const int run = blockIdx.x;
  pdl_wait();
  if (blockIdx.x == 0)
    for (int b = tid; b < p.g.B; b += kThreads) TreeSeq::check(p, b);
  W w;
  int2 rec = make_int2(0, 0);
  for (bool more = w.start(p, run, lane); more; more = w.next(p)) {
    if (w.count == 0) continue;
    const TreeSeq seq(p, w.b);
    const int tile = w.tile;
    const bool here = w.block == 0, whole = w.whole();
    if (here && !whole)
      rec = make_int2((w.b * p.g.Hkv + w.h) * p.tiles + tile, w.runs_of_group(run));
    const int n_rows = min(seq.tokens * p.G - tile * R, R);
    // this tile's queries (scaled) and masks; row r is token r / G, head r % G
    for (int i = tid; i < R * (D / 4); i += kThreads) {
      const int r = i / (D / 4), c = i % (D / 4) * 4;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r < n_rows) {
        const int row = tile * R + r, tok = row / p.G, head = w.h * p.G + row % p.G;
        const float *q = (const float *)p.q + head * p.q_head +
                         (p.starts == nullptr ? w.b * p.q_seq + tok * p.q_token
                                              : (long long)(seq.first + tok) * p.q_token);
        x = *reinterpret_cast<const float4 *>(q + c);
        x = make_float4(x.x * p.scale2, x.y * p.scale2, x.z * p.scale2, x.w * p.scale2);
      }
      *reinterpret_cast<float4 *>(&s.q[r][c]) = x;
    }
    if (tid < R) {
      const int tok = (tile * R + tid) / p.G;
      uint64_t mask = 0;
      if (tid < n_rows)
        mask = p.masks == nullptr ? ~0ull >> (63 - tok) : p.masks[seq.first + tok];
      s.mask[tid] = mask;
    }
    float2 o[4][DT / 2];
    float m[4], l[4];  // of the thread's rows, the same in the 16 threads of a row
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int j = 0; j < DT / 2; ++j) o[i][j] = make_float2(0.f, 0.f);
    }
    const int rg = tid / 16 * 4, cg = tid % 16;  // rows rg.., keys cg and cg + 16, dims 4 cg + 64 j..

    uint4 kx[kMine], vx[kMine];
    uint32_t there = 0;  // the block's rows that are in the cache (this thread's pieces' rows)
    float ksc[kCodes ? kMine : 1], vsc[kCodes ? kMine : 1];
    auto load = [&](int row0) {
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int e = tid + i * kThreads, row = row0 + e / kPieces, pc = e % kPieces;
        kx[i] = vx[i] = make_uint4(0, 0, 0, 0);
        if (kCodes) ksc[i % (kCodes ? kMine : 1)] = vsc[i % (kCodes ? kMine : 1)] = 1.f;
        there &= ~(1u << i);
        if (row >= w.end) continue;
        const int page = p.table[guard((long long)w.b * p.g.max_pages + (row >> p.g.shift), 1,
                                       (long long)p.g.B * p.g.max_pages, p.status)];
        if ((unsigned)page >= (unsigned)p.g.n_pages) {
          report(p.status, RIPPLE_EBOUNDS);
          continue;
        }
        there |= 1u << i;
        const int slot = row & ((1 << p.g.shift) - 1);
        const long long at = page * p.g.page_stride + w.h * p.g.head_stride +
                             slot * p.g.row_stride + pc * P::N;
        kx[i] = *reinterpret_cast<const uint4 *>((const T *)p.k_pages + at);
        vx[i] = *reinterpret_cast<const uint4 *>((const T *)p.v_pages + at);
        if constexpr (kCodes) {
          const long long sc = page * p.scale_page + w.h * p.scale_head + slot * p.scale_row;
          ksc[i] = scale_of_byte(p.k_scales[sc]);
          vsc[i] = scale_of_byte(p.v_scales[sc]);
        }
      }
    };
    __shared__ uint32_t row_there;
    load(w.begin);
    for (int row0 = w.begin; row0 < w.end; row0 += KB) {
      __syncthreads();  // the block before has been read
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int e = tid + i * kThreads, r = e / kPieces, c = e % kPieces * P::N;
        P::put(&s.k[r][c], kx[i], kCodes ? ksc[i % (kCodes ? kMine : 1)] : 1.f);
        P::put(&s.v[r][c], vx[i], kCodes ? vsc[i % (kCodes ? kMine : 1)] : 1.f);
      }
      uint32_t present = 0xffffffffu;
      if (!__syncthreads_and(there == (1u << kMine) - 1)) {  // which rows are there
        if (tid == 0) row_there = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
          const int e = tid + i * kThreads;
          if (e % kPieces == 0 && (there >> i & 1)) atomicOr(&row_there, 1u << (e / kPieces));
        }
        __syncthreads();
        present = row_there;
      }
      if (row0 + KB < w.end) load(row0 + KB);
      // scores (warps of rows that are none have nothing to do)
      const bool busy = rg - rg % 8 < n_rows;
      float x[4][2];
      if (busy) {
        float2 d[4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i][0] = d[i][1] = make_float2(0.f, 0.f);
#pragma unroll 4
        for (int c = 0; c < D; c += 4) {
          float4 kk[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) kk[j] = *reinterpret_cast<const float4 *>(&s.k[cg + 16 * j][c]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 qq = *reinterpret_cast<const float4 *>(&s.q[rg + i][c]);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              d[i][j] = __ffma2_rn(make_float2(qq.x, qq.y), make_float2(kk[j].x, kk[j].y), d[i][j]);
              d[i][j] = __ffma2_rn(make_float2(qq.z, qq.w), make_float2(kk[j].z, kk[j].w), d[i][j]);
            }
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) x[i][j] = d[i][j].x + d[i][j].y;
      }
      // the 16 threads of a row are half a warp; the four rows' steps side by side
      if (busy) {
        bool on[4][2];
        float mb[4], sum[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint64_t mask = s.mask[rg + i];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int c = cg + 16 * j;
            const long long of_draft = row0 + c - seq.prefix;
            on[i][j] = (present >> c & 1) && (of_draft < 0 || (mask >> (of_draft & 63) & 1));
            if (!on[i][j]) x[i][j] = -INFINITY;
          }
          mb[i] = fmaxf(x[i][0], x[i][1]);
        }
#pragma unroll
        for (int k = 1; k < 16; k <<= 1)
#pragma unroll
          for (int i = 0; i < 4; ++i) mb[i] = fmaxf(mb[i], __shfl_xor_sync(0xffffffffu, mb[i], k));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (mb[i] > m[i] + kSlack) {
            const float a = fast_exp2(m[i] - mb[i]);
            m[i] = mb[i];
            l[i] *= a;
#pragma unroll
            for (int j = 0; j < DT / 2; ++j) o[i][j] = __fmul2_rn(o[i][j], make_float2(a, a));
          }
          const float sub = m[i] == -INFINITY ? 0.f : m[i];
          sum[i] = 0.f;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float e = on[i][j] ? fast_exp2(x[i][j] - sub) : 0.f;
            sum[i] += e;
            s.p[cg + 16 * j][rg + i] = on[i][j] ? e : -1.f;
          }
        }
#pragma unroll
        for (int k = 1; k < 16; k <<= 1)
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], k);
#pragma unroll
        for (int i = 0; i < 4; ++i) l[i] += sum[i];
      }
      __syncthreads();
      // outputs: a negative probability's key counts for nothing, whatever its value holds
      auto add = [&](bool hidden) {
#pragma unroll 4
        for (int c = 0; c < KB; ++c) {
          const float4 pr = *reinterpret_cast<const float4 *>(&s.p[c][rg]);
          const float pp[4] = {pr.x, pr.y, pr.z, pr.w};
#pragma unroll
          for (int j = 0; j < DT; j += 4) {
            const float4 vv = *reinterpret_cast<const float4 *>(&s.v[c][4 * cg + 16 * j]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (hidden && pp[i] < 0.f) continue;
              const float2 both = make_float2(pp[i], pp[i]);
              o[i][j / 2] = __ffma2_rn(both, make_float2(vv.x, vv.y), o[i][j / 2]);
              o[i][j / 2 + 1] = __ffma2_rn(both, make_float2(vv.z, vv.w), o[i][j / 2 + 1]);
            }
          }
        }
      };
      if (!busy)
        continue;
      else if (present != 0xffffffffu || row0 + KB > seq.prefix)
        add(true);
      else
        add(false);
    }
    __syncthreads();
    const long long slot = (2LL * run + (here ? 1 : 0)) * p.tile_rows;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = rg + i;
      if (r >= n_rows) continue;
      const int row = tile * R + r;
      const long long at = (long long)(seq.first + row / p.G) * p.Hq + w.h * p.G + row % p.G;
      const float inv = !whole ? 1.f : l[i] != 0.f ? 1.f / l[i] : 0.f;  // 0: no row counts
      float *to = whole ? (float *)p.out + at * D : p.ws_o + (slot + r) * D;
#pragma unroll
      for (int j = 0; j < DT; j += 4)
        put4(to + 4 * cg + 16 * j,
             make_float4(o[i][j / 2].x * inv, o[i][j / 2].y * inv, o[i][j / 2 + 1].x * inv,
                         o[i][j / 2 + 1].y * inv));
      if (cg == 0) {
        if (!whole)
          p.ws_ml[slot + r] = make_float2(m[i], l[i]);
        else if (p.lse != nullptr)
          p.lse[at] = tree_lse(m[i], l[i]);
      }
    }
    __syncthreads();
  }
  if (tid == 0) p.rec[run] = rec;
}

// Joins the partials of the group that begins in run blockIdx.x and goes on, kJoinRows of its
// query rows per blockIdx.y; and writes the outputs of idle sequences.
constexpr int kJoinThreads = 256;

// kTiles: every tile is a group of its own.
template <typename O, int D, bool kTiles>
__global__ void __launch_bounds__(kJoinThreads)
    tree_join_kernel(const __grid_constant__ TreeParams p) {
  constexpr int kCols = D / 4, kRows = kJoinThreads / kCols;
  constexpr int kAt = 8;  // partials loaded at a time
  const int tid = threadIdx.x, col = tid % kCols, sub = tid / kCols;
  pdl_wait();
  const int run = blockIdx.x;
  const int2 rec = __ldcg(&p.rec[run]);
  if (rec.y > 0) {
    const int group = kTiles ? rec.x / p.tiles : rec.x, b = group / p.g.Hkv, h = group % p.g.Hkv;
    const TreeSeq seq(p, b);
    const int in = blockIdx.y * kRows + sub;
    const int tile = kTiles ? rec.x % p.tiles : in / p.tile_rows, r = kTiles ? in : in % p.tile_rows;
    const int row = kTiles ? tile * p.tile_rows + in : in;
    if (row < seq.tokens * p.G && r < p.tile_rows) {
      float m = -INFINITY, den = 0.f;
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int k0 = 0; k0 < rec.y; k0 += kAt) {
        float2 ml[kAt];
        float4 o[kAt];
#pragma unroll
        for (int i = 0; i < kAt; ++i) {
          const int k = min(k0 + i, rec.y - 1);
          const long long part = 2LL * (run + k) + (k == 0 ? 1 : 0);
          const long long slot = (kTiles ? part : part * p.tiles + tile) * p.tile_rows + r;
          ml[i] = __ldcg(&p.ws_ml[slot]);
          o[i] = __ldcg(reinterpret_cast<const float4 *>(p.ws_o + slot * D) + col);
        }
        float mn = m;
#pragma unroll
        for (int i = 0; i < kAt; ++i) mn = fmaxf(mn, ml[i].x);  // (repeats change no maximum)
        const float subm = mn == -INFINITY ? 0.f : mn, a = fast_exp2(m - subm);
        sum = make_float4(sum.x * a, sum.y * a, sum.z * a, sum.w * a);
        den *= a;
        m = mn;
#pragma unroll
        for (int i = 0; i < kAt; ++i)
          if (k0 + i < rec.y) {
            const float f = fast_exp2(ml[i].x - subm);
            sum.x += f * o[i].x;
            sum.y += f * o[i].y;
            sum.z += f * o[i].z;
            sum.w += f * o[i].w;
            den += f * ml[i].y;
          }
      }
      const long long at = (long long)(seq.first + row / p.G) * p.Hq + h * p.G + row % p.G;
      const float inv = den != 0.f ? 1.f / den : 0.f;  // 0: no row counts
      put4((O *)p.out + at * D + 4 * col,
           make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv));
      if (p.lse != nullptr && col == 0) p.lse[at] = tree_lse(m, den);
    }
  }
  // idle sequences
  const int blocks = gridDim.x * gridDim.y, me = blockIdx.y * gridDim.x + blockIdx.x;
  for (int b = me; b < p.g.B; b += blocks) {
    const TreeSeq seq(p, b);
    if (seq.len > 0) continue;
    for (long long i = tid; i < (long long)seq.tokens * p.Hq * kCols; i += kJoinThreads) {
      put4((O *)p.out + (long long)seq.first * p.Hq * D + 4 * i, make_float4(0.f, 0.f, 0.f, 0.f));
      if (p.lse != nullptr && i % kCols == 0) p.lse[(long long)seq.first * p.Hq + i / kCols] = -INFINITY;
    }
  }
}

cudaError_t launch_pdl(void (*kernel)(TreeParams), dim3 grid, int threads, const TreeParams &p,
                       cudaStream_t st, int smem = 0) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, p);
  count_launches(1);
  return e;
}

template <typename T, int D>
cudaError_t launch_simt(const TreeParams &p, int dev, cudaStream_t st) {
  static std::atomic<bool> attr_set[kMaxDevices];
  constexpr int smem = (int)sizeof(SimtSmem<D>);
  if (!attr_set[dev].load(std::memory_order_acquire)) {
    const cudaError_t e = cudaFuncSetAttribute(tree_simt_kernel<T, D>,
                                               cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    attr_set[dev].store(true, std::memory_order_release);
  }
  return launch_pdl(tree_simt_kernel<T, D>, dim3(p.n_runs), kThreads, p, st, smem);
}

template <typename O, int D, bool kTiles>
cudaError_t launch_join(const TreeParams &p, cudaStream_t st) {
  const int rows = kJoinThreads / (D / 4), most = kTiles ? p.tile_rows : p.max_tokens * p.G;
  return launch_pdl(tree_join_kernel<O, D, kTiles>, dim3(p.n_runs, (most + rows - 1) / rows),
                    kJoinThreads, p, st);
}

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

bool tree_args(const ripple_paged_desc *d, const ripple_paged_scales *scales, int n_q_heads,
               int max_tokens, TreeParams *p, ScaleGeom *s) {
  *s = ScaleGeom{};
  if (!paged_geom(d, &p->g, scales != nullptr)) return false;
  if (scales != nullptr && !scale_geom(d, scales, s)) return false;
  if (n_q_heads < 1 || n_q_heads % d->n_kv_heads != 0) return false;
  if (max_tokens < 1 || max_tokens > RIPPLE_MAX_DRAFT) return false;
  p->Hq = n_q_heads;
  p->G = n_q_heads / d->n_kv_heads;
  p->max_tokens = max_tokens;
  return p->G <= 16;
}

// Tiles and runs of a call and the workspace: records, (max, sum), outputs of the partials. The
// runs are bounded by the blocks that the table has room for; everything grows with the call.
// together: the CTAs of a run's tiles go over the same rows (tensor cores: the reads are shared
// through L2), otherwise every tile is a group of its own (the CUDA cores: bound by the FMAs, and
// sequences of few tokens have fewer tiles). Returns the bytes; fills p's pointers if given a base.
size_t plan(TreeParams *p, int tile, int block, int places, bool together, void *ws) {
  const int rows = p->max_tokens * p->G;
  p->tiles = (rows + tile - 1) / tile;
  p->tile_rows = rows < tile ? rows : tile;
  const long long room = (((long long)p->g.max_pages << p->g.shift) + block - 1) / block *
                         p->g.B * p->g.Hkv;
  size_t parts, runs;  // partials' tiles over two, records
  if (together) {
    // (as many records and partials as the places allow, whether or not the tiles divide them, so
    // that the workspace of more tokens is no smaller)
    p->n_runs = (int)std::min<long long>(std::max(1, places / p->tiles), room);
    runs = (size_t)std::min<long long>(places, room);
    parts = std::max((size_t)p->n_runs * p->tiles,
                     (size_t)std::min<long long>(places, room * p->tiles));
  } else {
    p->n_runs = (int)std::min<long long>(places, room * p->tiles);
    parts = runs = (size_t)p->n_runs;
  }
  const size_t slots = 2 * parts * p->tile_rows;
  const size_t rec = round_up(runs * sizeof(int2));
  const size_t ml = round_up(slots * sizeof(float2));
  uint8_t *base = (uint8_t *)ws;
  p->rec = (int2 *)base;
  p->ws_ml = (float2 *)(base + rec);
  p->ws_o = (float *)(base + rec + ml);
  return rec + ml + round_up(slots * p->g.D * sizeof(float));
}
size_t plan(TreeParams *p, int dtype, int sms, void *ws) {
  if (dtype == RIPPLE_BF16)
    return plan(p, kTreeTcRows, kTreeTcKeys, kTreeTcTeams * sms, true, ws);
  return plan(p, kTreeSimtRows, kTreeSimtKeys, kTreeSimtCtas * sms, false, ws);
}

// Shares of a group on the tensor cores where the table's room is short, 0 where it is not: as
// many teams as find a place at once, at most one a block, with few blocks each; their partials
// fit where the runs' would. Shares and runs (us, D 128, 8 KV heads, 4 heads each, 4 tokens; runs
// have a second launch and sums over the sequences): 16 sequences of 100 to 1000 rows 19.4 and 19.3,
// 32 of 60 to 200 14.1 and 18.2, one of 900 14.4 and 14.3, of 4000 19.1 and 19.0, of 8000 24.5 and
// 23.0, 4 of 2000 17.6 and 20.1. 8-bit pages, 16 tokens: 16 of 100 to 1000 rows 28.0 and 27.8, 4 of
// 2000 22.4 and 26.9, 32 of 64 15.5 and 21.7, but one of 900 18.8 and 16.8, of 8000 32.0 and 27.5.
// (Shares gain with several sequences, up to a third; one long sequence alone loses by a tenth, most
// over 8-bit pages.)
constexpr int kMostTeams = 16;  // (a cluster of 8)
constexpr int kShortBlocks = 8;
int short_teams(const TreeParams &p, int sms) {
  if (p.tiles > 1) return 0;
  const long long groups = (long long)p.g.B * p.g.Hkv, places = (long long)kTreeTcTeams * sms;
  const long long blocks = (((long long)p.g.max_pages << p.g.shift) + kTreeTcKeys - 1) / kTreeTcKeys;
  if (groups > places) return 0;
  int teams = 1;
  while (teams < kMostTeams && 2 * teams <= blocks && groups * 2 * teams <= places) teams *= 2;
  return blocks <= (long long)teams * kShortBlocks ? teams : 0;
}

}  // namespace

}  // namespace ripple

using namespace ripple;

extern "C" ripple_status ripple_paged_tree_workspace_bytes(const ripple_paged_desc *desc,
                                                           const ripple_paged_scales *scales,
                                                           int32_t n_q_heads, int32_t max_tokens,
                                                           size_t *bytes_host) {
  TreeParams p;
  ScaleGeom s;
  if (!tree_args(desc, scales, n_q_heads, max_tokens, &p, &s) || bytes_host == nullptr)
    return RIPPLE_EINVAL;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) dev = 0;
  *bytes_host = plan(&p, desc->dtype, sm_count(dev), nullptr);
  return RIPPLE_OK;
}

extern "C" ripple_status ripple_paged_tree_attn(
    const ripple_paged_desc *desc, const ripple_paged_scales *scales, int32_t n_tokens,
    const int32_t *seq_starts, int32_t max_tokens, const uint64_t *masks, int32_t n_q_heads,
    float scale, const void *q, const ripple_token_strides *q_strides, const void *k_pages,
    const void *v_pages, const int32_t *block_table, const int32_t *lens, void *out, float *lse,
    void *workspace, size_t workspace_bytes, int32_t *dev_status, void *stream) {
  TreeParams p;
  ScaleGeom s;
  if (n_tokens < 0 || (seq_starts == nullptr && desc != nullptr && desc->batch > 0 &&
                       n_tokens % desc->batch != 0))
    return RIPPLE_EINVAL;
  if (!tree_args(desc, scales, n_q_heads, max_tokens, &p, &s)) return RIPPLE_EINVAL;
  p.per_seq = seq_starts == nullptr ? n_tokens / desc->batch : 0;
  if (p.per_seq > max_tokens) return RIPPLE_EINVAL;
  if (!(scale >= 0.f) || scale > kMaxScale) return RIPPLE_EINVAL;
  if (n_tokens == 0) return RIPPLE_OK;
  if (!q || !q_strides || !k_pages || !v_pages || !block_table || !lens || !out || !workspace ||
      ((uintptr_t)workspace & 255u))
    return RIPPLE_EINVAL;
  if (!aligned16_host(q) || !aligned16_host(k_pages) || !aligned16_host(v_pages) ||
      !aligned16_host(out) || !aligned4_host({block_table, lens, lse, seq_starts, dev_status}) ||
      ((uintptr_t)masks & 7u) != 0)
    return RIPPLE_EINVAL;
  for (const int64_t x : {q_strides->seq_stride, q_strides->token_stride, q_strides->head_stride})
    if (x < 0 || x > (1LL << 40) || x % vec_elems(desc->dtype) != 0) return RIPPLE_EINVAL;
  int dev = 0;
  const cudaError_t got = cudaGetDevice(&dev);
  if (got != cudaSuccess || dev < 0 || dev >= kMaxDevices) dev = 0;
  if (workspace_bytes < plan(&p, desc->dtype, sm_count(dev), workspace)) return RIPPLE_EWORKSPACE;
  if (got != cudaSuccess) return RIPPLE_ECUDA;
  p.scale2 = (scale > 0.f ? scale : 1.0f / sqrtf((float)desc->head_dim)) * kLog2e;
  p.q = q;
  p.q_seq = q_strides->seq_stride;
  p.q_token = q_strides->token_stride;
  p.q_head = q_strides->head_stride;
  p.k_pages = k_pages;
  p.v_pages = v_pages;
  p.k_scales = s.k;
  p.v_scales = s.v;
  p.scale_page = s.page_stride;
  p.scale_head = s.head_stride;
  p.scale_row = s.row_stride;
  p.table = block_table;
  p.lens = lens;
  p.starts = seq_starts;
  p.masks = masks;
  p.out = out;
  p.lse = lse;
  p.status = dev_status;
  p.n_tokens = n_tokens;
  p.wait_cycles = wait_limit_cycles();
  cudaStream_t st = (cudaStream_t)stream;
  const bool d128 = desc->head_dim == 128;
  if (desc->dtype == RIPPLE_BF16) {
    p.teams = short_teams(p, sm_count(dev));
    RIPPLE_CUDA_TRY(launch_tree_tc(p, scales != nullptr, dev, sm_count(dev), st));
    if (p.teams > 0) return RIPPLE_OK;
    RIPPLE_CUDA_TRY((d128 ? launch_join<__nv_bfloat16, 128, false>(p, st)
                          : launch_join<__nv_bfloat16, 64, false>(p, st)));
    return RIPPLE_OK;
  }
  RIPPLE_CUDA_TRY((scales != nullptr ? (d128 ? launch_simt<uint8_t, 128>(p, dev, st)
                                             : launch_simt<uint8_t, 64>(p, dev, st))
                                     : (d128 ? launch_simt<float, 128>(p, dev, st)
                                             : launch_simt<float, 64>(p, dev, st))));
  RIPPLE_CUDA_TRY((d128 ? launch_join<float, 128, true>(p, st) : launch_join<float, 64, true>(p, st)));
  return RIPPLE_OK;
}
