// The paged cache as the kernels see it (ripple_paged_desc with its pointers),
// and its host-side checks.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <initializer_list>

#include "ripple.h"

namespace ripple {

// Rows of `inner` elements at at + the sum of i_j stride_j, i_j < count_j (places in elements).
struct RowSet {
  long long at, stride[3], count[3];
};

struct PagedGeom {
  int B, Hkv, D, shift;        // page_size == 1 << shift
  int n_pages, max_pages;
  long long page_stride, head_stride, row_stride;  // elements
  RowSet rows(const void *pages, int elem) const {  // of a pool
    return RowSet{(long long)((uintptr_t)pages / elem),
                  {row_stride, head_stride, page_stride},
                  {1LL << shift, Hkv, n_pages}};
  }
};

// Whether the places i * stride (i < count) of the dimensions, each `inner` long
// elements at the innermost, are disjoint: sorted by stride, every stride reaches past
// the dimensions within it.
inline bool disjoint(int n, const long long *stride, const long long *count, long long inner) {
  int order[3] = {0, 1, 2};
  std::sort(order, order + n, [&](int a, int b) { return stride[a] < stride[b]; });
  long long extent = inner;
  for (int i = 0; i < n; ++i) {
    const int d = order[i];
    if (count[d] <= 1) continue;
    if (stride[d] < extent) return false;
    extent += stride[d] * (count[d] - 1);
  }
  return true;
}

// Whether an element lies in a row of `a` and in one of `b`. Dimensions that both have with
// the same stride are looked at row by row (by the difference of the indices), the others as
// the span that they reach over: what is said to be apart is, and two views of one buffer
// that interleave (heads side by side in a token's row) are told from ones that overlap.
inline bool overlap(const RowSet &a, const RowSet &b, long long inner) {
  long long span_a = inner, span_b = inner;
  long long stride[3], most[3], least[3];  // of the shared dimensions, and the index differences
  int n = 0;
  for (int i = 0; i < 3; ++i) {
    if (a.count[i] > 1 && b.count[i] > 1 && a.stride[i] != b.stride[i]) {
      span_a += a.stride[i] * (a.count[i] - 1);
      span_b += b.stride[i] * (b.count[i] - 1);
    } else if (a.count[i] > 1 || b.count[i] > 1) {
      int j = n++;  // by descending stride
      const long long s = a.count[i] > 1 ? a.stride[i] : b.stride[i];
      for (; j > 0 && stride[j - 1] < s; --j) {
        stride[j] = stride[j - 1];
        most[j] = most[j - 1];
        least[j] = least[j - 1];
      }
      stride[j] = s;
      most[j] = a.count[i] - 1;
      least[j] = 1 - b.count[i];
    }
  }
  // is a sum of difference_j stride_j in [lo, hi] ?
  struct Search {
    const long long *stride, *most, *least;
    int n;
    bool find(int j, long long lo, long long hi) const {
      long long up = 0, down = 0;  // what the dimensions from j on reach
      for (int i = j; i < n; ++i) {
        up += most[i] * stride[i];
        down += least[i] * stride[i];
      }
      if (lo > up || hi < down) return false;
      if (j == n) return true;
      const long long s = stride[j];
      if (s == 0) return find(j + 1, lo, hi);
      up -= most[j] * s;
      down -= least[j] * s;
      const auto floor_div = [](long long x, long long y) { return x / y - (x % y < 0 ? 1 : 0); };
      const long long first = std::max(least[j], -floor_div(up - lo, s));
      const long long last = std::min(most[j], floor_div(hi - down, s));
      if (last - first > 64) return true;  // (no layout of rows that lie apart)
      for (long long i = first; i <= last; ++i)
        if (find(j + 1, lo - i * s, hi - i * s)) return true;
      return false;
    }
  };
  const long long d = b.at - a.at;
  return Search{stride, most, least, n}.find(0, d - span_a + 1, d + span_b - 1);
}

inline bool aligned16_host(const void *p) { return ((uintptr_t)p & 15u) == 0; }
inline bool aligned4_host(std::initializer_list<const void *> pointers) {
  for (const void *p : pointers)
    if (((uintptr_t)p & 3u) != 0) return false;
  return true;
}

// Elements of 16 bytes, or 0 for an unknown type.
inline int vec_elems(int dtype) {
  return dtype == RIPPLE_BF16 ? 8 : dtype == RIPPLE_F32 ? 4 : 0;
}

inline bool paged_geom(const ripple_paged_desc *d, PagedGeom *g) {
  if (d == nullptr) return false;
  const int vec = vec_elems(d->dtype);
  if (vec == 0 || d->batch < 1 || d->n_kv_heads < 1 || d->n_pages < 1 || d->max_pages < 1)
    return false;
  if (d->head_dim != 64 && d->head_dim != 128) return false;
  if (d->page_size < 1 || d->page_size > 1024 || (d->page_size & (d->page_size - 1)) != 0)
    return false;
  // every CTA of the decode sums over the sequences
  if (d->batch > (1 << 16) || (int64_t)d->batch * d->n_kv_heads > (1 << 24)) return false;
  // row numbers are int32, a block's end behind the last one included
  if ((int64_t)d->max_pages * d->page_size > 0x7fffffffLL - 1024) return false;
  g->B = d->batch;
  g->Hkv = d->n_kv_heads;
  g->D = d->head_dim;
  g->shift = 0;
  while ((1 << g->shift) < d->page_size) ++g->shift;
  g->n_pages = d->n_pages;
  g->max_pages = d->max_pages;
  g->row_stride = d->row_stride;
  g->head_stride = d->head_stride;
  g->page_stride = d->page_stride;
  if (d->row_stride == 0 && d->head_stride == 0 && d->page_stride == 0) {
    g->row_stride = d->head_dim;
    g->head_stride = (long long)d->page_size * g->row_stride;
    g->page_stride = d->n_kv_heads * g->head_stride;
  }
  const long long stride[3] = {g->row_stride, g->head_stride, g->page_stride};
  const long long count[3] = {d->page_size, d->n_kv_heads, d->n_pages};
  for (int i = 0; i < 3; ++i)
    if (stride[i] < 0 || stride[i] > (1LL << 48) / count[i] || stride[i] % vec != 0) return false;
  return disjoint(3, stride, count, d->head_dim);
}

}  // namespace ripple
