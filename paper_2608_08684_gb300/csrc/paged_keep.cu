// ripple_paged_keep_rows: the accepted drafted tokens' rows moved up behind the rows before
// the draft, in every layer's cache, and the lengths that leaves.
//
// A CTA takes a (sequence, layer): its rows' places by the lanes of its first warp, then each
// thread 16 bytes of one head's keys or values, over all the kept rows in ascending order.
// As the kept tokens ascend, no row is written before it is read (kept[j] >= j), and no
// thread touches another's bytes. What is moved is a few hundred KB, so the call is bound by
// the launch and by the chain lengths - tables - rows; the rows' loads of a thread are in
// flight together. 32 layers of one sequence, 4 rows of 8 heads of 128 kept: 3.3 us; of 64
// sequences in 8 bits (17 MB): 7.7 us.
#include "common.cuh"
#include "kernels.cuh"
#include "paged.cuh"

namespace ripple {
namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 8;  // rows of a thread on their way

struct KeepLayer {
  uint8_t *k, *v;
  const int32_t *table;
  uint8_t *k_scales, *v_scales;
};
struct KeepParams {
  PagedGeom g;  // strides in bytes here
  long long scale_page, scale_head, scale_row;
  int pieces;   // 16 bytes of a row
  bool codes;
  int per_seq, max_kept;
  const int32_t *starts, *kept, *lens;
  int32_t *lens_out, *status;
  KeepLayer layer[RIPPLE_MAX_LAYERS];
};
static_assert(sizeof(KeepParams) <= 32764, "kernel parameters");

struct Move {
  long long from, to;              // of the rows, bytes from the pool's start, head 0
  long long scale_from, scale_to;
};

__global__ void __launch_bounds__(kThreads) keep_kernel(const __grid_constant__ KeepParams p) {
  __shared__ Move moves[RIPPLE_MAX_DRAFT];
  __shared__ int n_moves;
  pdl_wait();
  const int b = blockIdx.x, tid = threadIdx.x;
  const KeepLayer &layer = p.layer[blockIdx.y];
  if (tid < 32) {
    const long long at = (long long)blockIdx.y * p.g.B + b;
    const int len = p.lens[at];
    const int n_b = p.per_seq > 0 || p.starts == nullptr ? p.per_seq : p.starts[b + 1] - p.starts[b];
    const long long first = (long long)len - n_b;
    const bool idle = len <= 0, short_of = !idle && (first < 0 || n_b < 0);  // no such draft
    // how many entries count: up to the first that is negative, no token or does not ascend
    int n = 0;
    bool bad = short_of;
    int entry[RIPPLE_MAX_DRAFT / 32];
    if (!idle && !short_of) {
      int before = -1;
      bool ended = false;
#pragma unroll
      for (int i = 0; i < RIPPLE_MAX_DRAFT / 32; ++i) {
        const int j = 32 * i + tid;
        const int e = j < p.max_kept ? p.kept[(long long)b * p.max_kept + j] : -1;
        entry[i] = e;
        int prev = __shfl_up_sync(0xffffffffu, e, 1);
        if (tid == 0) prev = before;
        before = __shfl_sync(0xffffffffu, e, 31);
        const bool wrong = e >= 0 && (e >= n_b || (j > 0 && e <= prev));
        const uint32_t stop = __ballot_sync(0xffffffffu, e < 0 || wrong);
        const uint32_t wrongs = __ballot_sync(0xffffffffu, wrong);
        if (!ended) {
          const int k = stop != 0 ? __ffs(stop) - 1 : 32;
          n += k;
          if (stop != 0) {
            ended = true;
            bad = wrongs >> k & 1;
          }
        }
      }
    }
    int count = 0;
#pragma unroll
    for (int i = 0; i < RIPPLE_MAX_DRAFT / 32; ++i) {
      const int j = 32 * i + tid;
      Move m{};
      bool moves_it = j < n && entry[i] != j;
      int wrong = 0;
      if (moves_it) {
        const long long rows[2] = {first + entry[i], first + j};
        long long place[2], scale[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const long long pg = rows[k] >> p.g.shift, slot = rows[k] & ((1 << p.g.shift) - 1);
          int page = -1;
          if (pg >= p.g.max_pages)
            wrong = wrong == 0 ? RIPPLE_EFULL : wrong;
          else
            page = layer.table[guard((long long)b * p.g.max_pages + pg, 1,
                                     (long long)p.g.B * p.g.max_pages, p.status)];
          if ((unsigned)page >= (unsigned)p.g.n_pages) {
            if (wrong == 0) wrong = RIPPLE_EBOUNDS;
            page = 0;
          }
          place[k] = page * p.g.page_stride + slot * p.g.row_stride;
          scale[k] = page * p.scale_page + slot * p.scale_row;
        }
        m = Move{place[0], place[1], scale[0], scale[1]};
        if (wrong != 0) report(p.status, wrong);
        moves_it = wrong == 0;
      }
      const uint32_t them = __ballot_sync(0xffffffffu, moves_it);
      if (moves_it) moves[count + __popc(them & ((1u << tid) - 1))] = m;
      count += __popc(them);
    }
    if (tid == 0) {
      if (bad) report(p.status, RIPPLE_EBOUNDS);
      n_moves = count;
      p.lens_out[at] = idle || short_of ? len : (int)(first + n);
    }
  }
  __syncthreads();
  const int n = n_moves, items = 2 * p.g.Hkv * p.pieces;
  if (n == 0) return;
  for (int i = tid; i < items; i += kThreads) {
    const int pc = i % p.pieces, h = i / p.pieces % p.g.Hkv;
    uint8_t *pool = (i < items / 2 ? layer.k : layer.v) + h * p.g.head_stride + 16 * pc;
    for (int j0 = 0; j0 < n; j0 += kAhead) {
      uint4 x[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (j0 + j < n) x[j] = *reinterpret_cast<const uint4 *>(pool + moves[j0 + j].from);
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (j0 + j < n) *reinterpret_cast<uint4 *>(pool + moves[j0 + j].to) = x[j];
    }
  }
  if (p.codes)
    for (int i = tid; i < 2 * p.g.Hkv; i += kThreads) {
      uint8_t *pool = (i < p.g.Hkv ? layer.k_scales : layer.v_scales) + i % p.g.Hkv * p.scale_head;
      for (int j = 0; j < n; ++j) pool[moves[j].scale_to] = pool[moves[j].scale_from];
    }
}

}  // namespace
}  // namespace ripple

using namespace ripple;

extern "C" ripple_status ripple_paged_keep_rows(
    const ripple_paged_desc *desc, const ripple_paged_scales *scales_host, int32_t n_layers,
    void *const *k_pages_host, void *const *v_pages_host, const int32_t *const *block_tables_host,
    int32_t n_tokens, const int32_t *seq_starts, int32_t max_kept, const int32_t *kept,
    const int32_t *lens, int32_t *lens_out, int32_t *dev_status, void *stream) {
  KeepParams p;
  const bool codes = scales_host != nullptr;
  if (!paged_geom(desc, &p.g, codes)) return RIPPLE_EINVAL;
  if (n_layers < 1 || n_layers > RIPPLE_MAX_LAYERS || !k_pages_host || !v_pages_host ||
      !block_tables_host || !lens || !lens_out)
    return RIPPLE_EINVAL;
  if (n_tokens < 0 || (seq_starts == nullptr && n_tokens % desc->batch != 0)) return RIPPLE_EINVAL;
  if (max_kept < 0 || max_kept > RIPPLE_MAX_DRAFT || (max_kept > 0 && kept == nullptr))
    return RIPPLE_EINVAL;
  if (!aligned4_host({seq_starts, kept, lens, lens_out, dev_status})) return RIPPLE_EINVAL;
  const int bytes = codes ? 1 : 16 / vec_elems(desc->dtype);
  p.scale_page = p.scale_head = p.scale_row = 0;
  for (int l = 0; l < n_layers; ++l) {
    KeepLayer &x = p.layer[l];
    x.k = (uint8_t *)k_pages_host[l];
    x.v = (uint8_t *)v_pages_host[l];
    x.table = block_tables_host[l];
    x.k_scales = x.v_scales = nullptr;
    if (!x.k || !x.v || !x.table || !aligned16_host(x.k) || !aligned16_host(x.v) ||
        !aligned4_host({x.table}))
      return RIPPLE_EINVAL;
    if (overlap(p.g.rows(x.k, bytes), p.g.rows(x.v, bytes), desc->head_dim)) return RIPPLE_EINVAL;
    if (codes) {
      ScaleGeom s;
      if (!scale_geom(desc, &scales_host[l], &s)) return RIPPLE_EINVAL;
      if (l > 0 && (s.page_stride != p.scale_page || s.head_stride != p.scale_head ||
                    s.row_stride != p.scale_row))
        return RIPPLE_EINVAL;
      // what one thread moves no other may: the scales lie apart from each other and from the rows
      const RowSet rows[2] = {p.g.rows(x.k, 1), p.g.rows(x.v, 1)};
      const RowSet places[2] = {s.rows(s.k, p.g), s.rows(s.v, p.g)};
      if (overlap(places[0], places[1], 1)) return RIPPLE_EINVAL;
      for (int i = 0; i < 4; ++i)
        if (overlap(rows[i / 2], places[i % 2], desc->head_dim, 1)) return RIPPLE_EINVAL;
      p.scale_page = s.page_stride;
      p.scale_head = s.head_stride;
      p.scale_row = s.row_stride;
      x.k_scales = s.k;
      x.v_scales = s.v;
    }
  }
  // what one thread block reads no other may write
  const long long entries = (long long)n_layers * desc->batch;
  const auto over_lens_out = [&](const int32_t *at, long long n) {
    return at != nullptr && (uintptr_t)at < (uintptr_t)(lens_out + entries) &&
           (uintptr_t)lens_out < (uintptr_t)(at + n);
  };
  if ((lens != lens_out && over_lens_out(lens, entries)) ||
      over_lens_out(kept, (long long)max_kept * desc->batch) ||
      over_lens_out(seq_starts, desc->batch + 1LL))
    return RIPPLE_EINVAL;
  p.g.page_stride *= bytes;
  p.g.head_stride *= bytes;
  p.g.row_stride *= bytes;
  p.pieces = desc->head_dim * bytes / 16;
  p.codes = codes;
  p.per_seq = seq_starts == nullptr ? n_tokens / desc->batch : 0;
  p.max_kept = max_kept;
  p.starts = seq_starts;
  p.kept = kept;
  p.lens = lens;
  p.lens_out = lens_out;
  p.status = dev_status;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(desc->batch, n_layers);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = (cudaStream_t)stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, keep_kernel, p);
  count_launches(1);
  RIPPLE_CUDA_TRY(e);
  return RIPPLE_OK;
}
