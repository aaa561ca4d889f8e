// What the kernels of ripple_paged_tree_attn share: parameters, the cut of the work into
// runs, and the join of a group's partials.
//
// Work: the cache rows of every (sequence, KV head) group are cut into blocks, and the
// blocks of all groups, in order, into runs of equal cost: a group's first block costs kGroupCost
// more (its queries, its outputs), in units of a block that begin the group. The queries of a
// group, n_b tokens times G heads, are rows of tiles; a CTA takes a run for one row tile, and the
// CTAs of a run's tiles are neighbours, so that they read the same rows from L2 at about the same
// time.
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
  int teams;                             // on the tensor cores, short caches: shares of a group (0: runs)
  long long wait_cycles;
  uint32_t suspend_ns;                   // of a poll of an mbarrier, at most
  bool tma;                              // whole blocks by TMA
  int2 *rec;      // [n_runs] the group that begins in the run and goes on (with tiles of its own:
                  // times tiles, plus the tile), and its runs (0: none)
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

// Where a run of `total` units begins.
__device__ __forceinline__ long long run_start(long long total, int runs, int run) {
  return total * run / runs;
}
// The run that has unit t.
__device__ __forceinline__ int run_of(long long total, int runs, long long t) {
  return (int)(((t + 1) * runs - 1) / total);
}

// A walk over the parts of groups in a run. KB: rows of a block; COST: units of a group besides
// its blocks; TR: query rows of a tile where every tile is a group of its own (0: a tile each
// for other CTAs).
template <int KB, int COST, int TR>
struct TreeWalk {
  int b, h, len;
  int tiles, tile;     // of the sequence, with TR; the group's
  int block;           // the part's first in its group
  int count;           // blocks of the part
  int begin, end;      // the part's rows
  long long at, stop;  // the group's first unit, the run's end
  long long total;
  int runs;
  static __device__ __forceinline__ int blocks_of(const TreeSeq &s) {
    return s.tokens > 0 ? s.len / KB + (s.len % KB != 0) : 0;
  }
  static __device__ __forceinline__ int tiles_of(const TreeParams &p, const TreeSeq &s) {
    return TR > 0 ? (s.tokens * p.G + TR - 1) / (TR > 0 ? TR : 1) : 1;
  }
  // Units of a sequence's groups of one KV head.
  static __device__ __forceinline__ long long units_of(const TreeParams &p, const TreeSeq &s) {
    const int n = blocks_of(s);
    return n > 0 ? (long long)(n + COST) * tiles_of(p, s) : 0;
  }
  __device__ __forceinline__ int blocks() const { return len / KB + (len % KB != 0); }
  __device__ __forceinline__ void set(int first) {
    block = first;
    count = (int)min((long long)blocks(), max(stop - at - COST, (long long)first)) - first;
    begin = block * KB;
    end = (int)min((long long)len, (long long)(block + count) * KB);
  }
  // The part begins its group; the runs from this one on that have the group's blocks.
  __device__ __forceinline__ bool whole() const { return block == 0 && count == blocks(); }
  __device__ __forceinline__ int runs_of_group(int run) const {
    return run_of(total, runs, at + COST + blocks() - 1) - run + 1;
  }
  // To the next part; false at the end of the run. (A part may have no blocks: the units that
  // begin its group are all that the run has of it.)
  __device__ __forceinline__ bool next(const TreeParams &p) {
    at += blocks() + COST;
    if (at >= stop) return false;
    if (++tile < tiles) {
      set(0);
      return true;
    }
    tile = 0;
    if (++h >= p.g.Hkv) {
      h = 0;
      for (;;) {  // at < stop: there are more
        const TreeSeq s(p, ++b);
        len = s.len;
        tiles = tiles_of(p, s);
        if (blocks_of(s) > 0) break;
      }
    }
    set(0);
    return true;
  }
  // The share `of` in `shares` equal ones of a group, the only part; false where it has no blocks.
  __device__ __forceinline__ bool share(const TreeParams &p, int group, int of, int shares) {
    if (group >= p.g.B * p.g.Hkv) return false;
    b = group / p.g.Hkv;
    h = group % p.g.Hkv;
    const TreeSeq s(p, b);
    len = s.len;
    const unsigned n = blocks_of(s);  // (fewer than 2^25)
    block = (int)(n * of / shares);
    count = (int)(n * (of + 1) / shares) - block;
    begin = block * KB;
    end = (int)min((long long)len, (long long)(block + count) * KB);
    at = stop = total = 0;
    runs = tile = 0;
    tiles = 1;
    return count > 0;
  }
  // To the run's first part, by one warp; false where the run is empty.
  __device__ __forceinline__ bool start(const TreeParams &p, int run, int lane) {
    constexpr unsigned kAll = 0xffffffffu;
    const int per = (p.g.B + 31) / 32;
    const int b0 = min(lane * per, p.g.B), b1 = min(b0 + per, p.g.B);
    long long mine = 0;
    for (int i = b0; i < b1; ++i) mine += units_of(p, TreeSeq(p, i)) * p.g.Hkv;
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(kAll, incl, o);
      if (lane >= o) incl += y;
    }
    total = __shfl_sync(kAll, incl, 31);
    runs = (int)min((long long)p.n_runs, total);
    if (run >= runs) return false;
    const long long t0 = run_start(total, runs, run);
    stop = run_start(total, runs, run + 1);
    const int owner = __ffs(__ballot_sync(kAll, incl > t0)) - 1;
    int seq = 0;
    long long rest = t0 - (incl - mine);
    if (lane == owner) {
      for (seq = b0;; ++seq) {
        const long long k = units_of(p, TreeSeq(p, seq)) * p.g.Hkv;
        if (rest < k) break;
        rest -= k;
      }
    }
    b = __shfl_sync(kAll, seq, owner);
    rest = __shfl_sync(kAll, rest, owner);
    const TreeSeq s(p, b);
    len = s.len;
    tiles = tiles_of(p, s);
    const int units = blocks() + COST;
    const int group = (int)(rest / units), in = (int)(rest % units);
    h = group / tiles;
    tile = group % tiles;
    at = t0 - in;
    set(max(0, in - COST));
    return true;
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

// bf16 queries: on the tensor cores (paged_tree_tc.cu). Rows of a tile, keys of a block, teams
// (which take the place of CTAs) of an SM.
constexpr int kTreeTcRows = 128, kTreeTcKeys = 64, kTreeTcTeams = 2;
cudaError_t launch_tree_tc(const TreeParams &p, bool codes, int dev, int sms, cudaStream_t st);
// fp32 queries: on the CUDA cores (paged_tree.cu).
constexpr int kTreeSimtRows = 32, kTreeSimtKeys = 32, kTreeSimtCtas = 3;

}  // namespace ripple
