// What the kernels of ripple_paged_tree_attn share: parameters, the cut of the work into
// runs, and the join of a group's partials.
//
// Work: the cache rows of every (sequence, KV head) group are cut into blocks, and the
// blocks of all groups, in order, into equal runs. The queries of a group, n_b tokens times
// G heads, are rows of tiles; a CTA takes a run for one row tile, and the CTAs of a run's
// tiles are neighbours, so that they read the same rows from L2 at about the same time.
// Lengths are read on the device; every CTA finds its run by a sum over the sequences. A
// group that lies in one run is written there; of the others every run leaves a partial
// (a run has two at most: of the group it begins within and of the one it ends within),
// joined in order by a second launch. What a run covers does not depend on where it goes, so
// results do not either.
#pragma once

#include <math.h>

#include <algorithm>

#include "common.cuh"
#include "kernels.cuh"
#include "paged.cuh"

namespace ripple {

struct TreeParams {
  PagedGeom g;
  int Hq, G;
  float scale2;                          // logit scale * log2(e)
  const void *q;
  long long q_seq, q_token, q_head;      // strides, elements
  const void *k_pages, *v_pages;
  const uint8_t *k_scales, *v_scales;    // 8-bit pages: a byte a row and head
  long long scale_page, scale_head, scale_row;
  const int32_t *table, *lens, *starts;
  const uint64_t *masks;
  void *out;
  float *lse;
  int32_t *status;
  int n_tokens, per_seq, max_tokens;     // per_seq: tokens of every sequence, without starts
  int tiles, tile_rows;                  // row tiles of a group at most, rows of a partial
  int n_runs;
  long long wait_cycles;
  uint32_t suspend_ns;                   // of a poll of an mbarrier, at most
  bool tma;                              // whole blocks by TMA
  int2 *rec;      // [n_runs] the group that begins in the run and goes on, and its runs (0: none)
  float *ws_o;    // [2 * n_runs][tiles][tile_rows][D] partials: of the group begun before, begun here
  float2 *ws_ml;  // [2 * n_runs][tiles][tile_rows] their maximum (log2) and sum
};

// A sequence of the batch as a call sees it.
struct TreeSeq {
  int tokens, len;      // drafted tokens; rows to attend to (0: idle)
  int first;            // index of the first token
  long long prefix;     // rows before the draft (negative: a draft of more tokens than rows)
  __device__ __forceinline__ TreeSeq(const TreeParams &p, int b) {
    if (p.starts == nullptr) {
      tokens = p.per_seq;
      first = b * p.per_seq;
    } else {
      first = p.starts[b];
      tokens = min(max(p.starts[b + 1] - first, 0), p.max_tokens);
      if (first < 0 || first > p.n_tokens - tokens) tokens = 0;  // (reported by check)
    }
    const long long room = (long long)p.g.max_pages << p.g.shift;
    const int n = p.lens[b];
    prefix = (long long)n - tokens;
    len = n <= 0 ? 0 : (int)(n < room ? n : room);
  }
  // What the host cannot see of a sequence.
  static __device__ __forceinline__ void check(const TreeParams &p, int b) {
    const int n = p.lens[b];
    int tokens = p.per_seq;
    if (p.starts != nullptr) {
      const int first = p.starts[b];
      tokens = p.starts[b + 1] - first;
      if (tokens < 0 || tokens > p.max_tokens || first < 0 || first > p.n_tokens - tokens)
        report(p.status, RIPPLE_EBOUNDS);
    }
    if (n > 0 && n < tokens) report(p.status, RIPPLE_EBOUNDS);
    if ((long long)n > (long long)p.g.max_pages << p.g.shift) report(p.status, RIPPLE_EFULL);
  }
};

// Where a run of `total` blocks begins.
__device__ __forceinline__ long long run_start(long long total, int runs, int run) {
  return total * run / runs;
}
// The run that has block t.
__device__ __forceinline__ int run_of(long long total, int runs, long long t) {
  return (int)(((t + 1) * runs - 1) / total);
}

// A walk over the parts of groups in a run. KB: rows of a block.
template <int KB>
struct TreeWalk {
  int b, h, len;
  int block;           // the part's first in its group
  int begin, end;      // the part's rows
  long long left;      // blocks of the run, the part's included
  static __device__ __forceinline__ int blocks_of(const TreeSeq &s) {
    return s.tokens > 0 ? s.len / KB + (s.len % KB != 0) : 0;
  }
  __device__ __forceinline__ int blocks() const { return len / KB + (len % KB != 0); }
  __device__ __forceinline__ int count() const {
    return (int)min((long long)(blocks() - block), left);
  }
  __device__ __forceinline__ void set() {
    begin = block * KB;
    end = (int)min((long long)len, (long long)(block + count()) * KB);
  }
  // To the next part; false at the end of the run.
  __device__ __forceinline__ bool next(const TreeParams &p) {
    left -= count();
    if (left <= 0) return false;
    block = 0;
    if (++h >= p.g.Hkv) {
      h = 0;
      for (;;) {  // left > 0: there are more
        const TreeSeq s(p, ++b);
        len = s.len;
        if (blocks_of(s) > 0) break;
      }
    }
    set();
    return true;
  }
  // The run's first part, by one warp; returns the number of all blocks, 0 where the run is
  // empty (or nothing is to do).
  __device__ __forceinline__ long long start(const TreeParams &p, int run, int lane) {
    constexpr unsigned kAll = 0xffffffffu;
    const int per = (p.g.B + 31) / 32;
    const int b0 = min(lane * per, p.g.B), b1 = min(b0 + per, p.g.B);
    long long mine = 0;
    for (int i = b0; i < b1; ++i) mine += (long long)blocks_of(TreeSeq(p, i)) * p.g.Hkv;
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(kAll, incl, o);
      if (lane >= o) incl += y;
    }
    const long long total = __shfl_sync(kAll, incl, 31);
    const int runs = (int)min((long long)p.n_runs, total);
    if (run >= runs) return 0;
    const long long t0 = run_start(total, runs, run);
    left = run_start(total, runs, run + 1) - t0;
    const int owner = __ffs(__ballot_sync(kAll, incl > t0)) - 1;
    int seq = 0;
    long long rest = t0 - (incl - mine);
    if (lane == owner) {
      for (seq = b0;; ++seq) {
        const long long k = (long long)blocks_of(TreeSeq(p, seq)) * p.g.Hkv;
        if (rest < k) break;
        rest -= k;
      }
    }
    b = __shfl_sync(kAll, seq, owner);
    rest = __shfl_sync(kAll, rest, owner);
    len = TreeSeq(p, b).len;
    h = (int)(rest / blocks());
    block = (int)(rest % blocks());
    set();
    return total;
  }
};

__device__ __forceinline__ float tree_lse(float m, float l) {  // of log2 units; no row: -infinity
  return (m + log2f(l)) * 0.6931471805599453f;
}
__device__ __forceinline__ void put4(float *p, const float4 &x) {
  *reinterpret_cast<float4 *>(p) = x;
}
__device__ __forceinline__ void put4(__nv_bfloat16 *p, const float4 &x) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(x.x, x.y), b = __floats2bfloat162_rn(x.z, x.w);
  *reinterpret_cast<uint2 *>(p) = make_uint2(*reinterpret_cast<const uint32_t *>(&a),
                                             *reinterpret_cast<const uint32_t *>(&b));
}

// bf16 queries: on the tensor cores (paged_tree_tc.cu). Rows of a tile, keys of a block, CTAs
// of an SM.
constexpr int kTreeTcRows = 128, kTreeTcKeys = 64, kTreeTcCtas = 2;
cudaError_t launch_tree_tc(const TreeParams &p, bool codes, int dev, cudaStream_t st);
// fp32 queries: on the CUDA cores (paged_tree.cu).
constexpr int kTreeSimtRows = 32, kTreeSimtKeys = 32, kTreeSimtCtas = 3;

}  // namespace ripple
