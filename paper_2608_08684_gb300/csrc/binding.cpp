// Argument marshalling of the calls that a serving program makes per layer and token:
// checks of the tensors, their pointers and strides, the current stream, and the call of
// the library's entry point (whose address is given, so that the bounds-checked library is
// called the same way). A pass of ripple_paged_append through ctypes took 9.1 us of the
// host's time on a GB300's Grace, 2 of them the launch; through these functions 3.6.
#include <Python.h>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <memory>
#include <vector>

#include "paged.cuh"
#include "ripple.h"

namespace {

struct Cache {
  ripple_paged_desc desc;
  void *k, *v;
  const int32_t *table;
  int device;
  at::ScalarType type;            // of q, k and v
  ripple_paged_scales scales;     // of 8-bit pages, NULL pointers otherwise
  const ripple_paged_scales *codes() const { return scales.k_scales != nullptr ? &scales : nullptr; }
};

// A call's refusal; the message goes into a ValueError.
struct Refused {
  const char *why;
};
void need(bool ok, const char *why) {
  if (!ok) throw Refused{why};
}

const at::Tensor &tensor(PyObject *o) {
  need(THPVariable_Check(o), "expected a tensor");
  return THPVariable_Unpack(o);
}

const char *const kDevice = "expected CUDA tensors on one device, the current one";

// A dense tensor of `type` on `device`; its pointer, or NULL for None.
template <typename T>
T *dense(PyObject *o, int device, at::ScalarType type, const char *shape, int64_t numel = -1) {
  if (o == Py_None) return nullptr;
  const at::Tensor &t = tensor(o);
  need(t.scalar_type() == type && (numel < 0 || t.numel() == numel), shape);
  need(t.get_device() == device, kDevice);
  need(t.is_contiguous(), "expected a contiguous tensor");
  return static_cast<T *>(t.data_ptr());
}

// A tensor of tokens: [B][heads][d], [B][n][heads][d], or ragged [tokens][heads][d].
struct Tokens {
  void *data;
  ripple_token_strides strides;
  int64_t lead[2], heads;  // leading sizes, the second 1 where there is one
  int dim;
  Tokens(PyObject *o, const Cache &c, bool ragged) {
    const at::Tensor &t = tensor(o);
    dim = (int)t.dim();
    need(dim == 3 || (dim == 4 && !ragged),
         "tokens must be [B][heads][d] or [B][n][heads][d]; with seq_starts [tokens][heads][d]");
    need(t.size(dim - 1) == c.desc.head_dim && t.stride(dim - 1) == 1 && t.scalar_type() == c.type,
         "tokens must be [..][heads][d] in the cache's dtype, the dims consecutive");
    need(t.get_device() == c.device, kDevice);
    lead[0] = t.size(0);
    lead[1] = dim == 4 ? t.size(1) : 1;
    heads = t.size(dim - 2);
    strides.head_stride = t.stride(dim - 2);
    strides.seq_stride = ragged ? 0 : t.stride(0);
    strides.token_stride = ragged ? t.stride(0) : dim == 4 ? t.stride(1) : 0;
    data = t.data_ptr();
  }
  bool same(const Tokens &x) const {
    return dim == x.dim && lead[0] == x.lead[0] && lead[1] == x.lead[1];
  }
};

void *stream_of(PyObject *o) {
  if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
  void *s = PyLong_AsVoidPtr(o);
  if (PyErr_Occurred()) throw Refused{nullptr};
  return s;
}

// A logit scale; one that fp32 would turn into 0 is none (0 stands for the default).
float scale_of(PyObject *o) {
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) throw Refused{nullptr};
  const float scale = static_cast<float>(x);
  need(scale != 0.f || x == 0.0, "the scale is smaller than any fp32 value");
  return scale;
}

void *entry(PyObject *o) {
  void *f = PyLong_AsVoidPtr(o);
  if (f == nullptr) throw Refused{PyErr_Occurred() ? nullptr : "no entry point"};
  return f;
}
template <typename F>
F *entry(PyObject *o) {
  return reinterpret_cast<F *>(entry(o));
}

const Cache &cache_of(PyObject *o) {
  const void *c = PyCapsule_GetPointer(o, "ripple_paged_cache");
  if (c == nullptr) throw Refused{nullptr};
  return *static_cast<const Cache *>(c);
}

// Runs f() -> status; no C++ exception leaves.
template <typename F>
PyObject *guarded(F f) {
  try {
    return PyLong_FromLong(f());
  } catch (const Refused &r) {
    if (r.why != nullptr) PyErr_SetString(PyExc_ValueError, r.why);
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}
bool args_are(Py_ssize_t n, Py_ssize_t want) {
  if (n != want) PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
  return n == want;
}

// cache(desc address, k, v, table addresses, device, is bf16, scales address or None)
PyObject *cache(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!args_are(n, 7)) return nullptr;
  const void *desc = PyLong_AsVoidPtr(a[0]);
  Cache c;
  c.k = PyLong_AsVoidPtr(a[1]);
  c.v = PyLong_AsVoidPtr(a[2]);
  c.table = static_cast<const int32_t *>(PyLong_AsVoidPtr(a[3]));
  c.device = (int)PyLong_AsLong(a[4]);
  c.type = PyObject_IsTrue(a[5]) == 1 ? at::kBFloat16 : at::kFloat;
  c.scales = ripple_paged_scales{};
  const void *scales = a[6] == Py_None ? nullptr : PyLong_AsVoidPtr(a[6]);
  if (PyErr_Occurred()) return nullptr;
  if (scales != nullptr) c.scales = *static_cast<const ripple_paged_scales *>(scales);
  if (desc == nullptr) {
    PyErr_SetString(PyExc_ValueError, "no descriptor");
    return nullptr;
  }
  c.desc = *static_cast<const ripple_paged_desc *>(desc);
  Cache *kept = new (std::nothrow) Cache(c);
  if (kept == nullptr) return PyErr_NoMemory();
  PyObject *o = PyCapsule_New(kept, "ripple_paged_cache", [](PyObject *self) {
    delete static_cast<Cache *>(PyCapsule_GetPointer(self, "ripple_paged_cache"));
  });
  if (o == nullptr) delete kept;
  return o;
}

// paged_append(entry (of the cache's kind: 8-bit pages have one of their own), cache, rope address or
// None, lens, k, v, positions, seq_starts, q, q_out, dev_status, stream)
PyObject *paged_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!args_are(n, 12)) return nullptr;
  return guarded([&] {
    void *call = entry(a[0]);
    const Cache &c = cache_of(a[1]);
    const ripple_rope *rope = nullptr;
    if (a[2] != Py_None) {
      rope = static_cast<const ripple_rope *>(PyLong_AsVoidPtr(a[2]));
      if (PyErr_Occurred()) throw Refused{nullptr};
    }
    need(c10::cuda::current_device() == c.device, kDevice);
    const bool ragged = a[7] != Py_None;
    need(a[3] != Py_None, "lens must be int32 [B]");
    const int32_t *lens = dense<int32_t>(a[3], c.device, at::kInt, "lens must be int32 [B]", c.desc.batch);
    const Tokens k(a[4], c, ragged), v(a[5], c, ragged);
    need(k.same(v) && k.heads == c.desc.n_kv_heads && v.heads == k.heads,
         "k and v must have the same tokens and the cache's heads");
    need(ragged || k.lead[0] == c.desc.batch, "one entry per sequence");
    const int64_t tokens = k.lead[0] * k.lead[1];
    need(tokens <= 0x7fffffff, "too many tokens");
    const int32_t *positions = nullptr;
    if (a[6] != Py_None) {
      const at::Tensor &t = tensor(a[6]);
      need(t.dim() == k.dim - 2 && t.size(0) == k.lead[0] &&
               (k.dim == 3 || t.size(1) == k.lead[1]),
           "positions must be int32 with k's leading sizes");
      positions = dense<int32_t>(a[6], c.device, at::kInt,
                                 "positions must be int32 with k's leading sizes", tokens);
    }
    const int32_t *starts = dense<int32_t>(a[7], c.device, at::kInt,
                                           "seq_starts must be int32 [B + 1]",
                                           (int64_t)c.desc.batch + 1);
    need((a[8] == Py_None) == (a[9] == Py_None), "q and q_out go together");
    void *q = nullptr, *q_out = nullptr;
    ripple_token_strides qs{}, os{};
    int64_t heads = 0;
    if (a[8] != Py_None) {
      const Tokens from(a[8], c, ragged), to(a[9], c, ragged);
      need(from.same(k) && to.same(k) && from.heads == to.heads,
           "q and q_out must have k's tokens, and the same heads");
      q = from.data;
      q_out = to.data;
      qs = from.strides;
      os = to.strides;
      heads = from.heads;
    }
    int32_t *status = dense<int32_t>(a[10], c.device, at::kInt, "dev_status must be int32");
    void *stream = stream_of(a[11]);
    ripple_status s;
    Py_BEGIN_ALLOW_THREADS
    if (c.codes() != nullptr)
      s = reinterpret_cast<decltype(ripple_paged_append_q8) *>(call)(
          &c.desc, &c.scales, rope, (int32_t)tokens, starts, (int32_t)heads, q, &qs, q_out, &os,
          k.data, &k.strides, v.data, &v.strides, positions, c.k, c.v, c.table, lens, status, stream);
    else
      s = reinterpret_cast<decltype(ripple_paged_append) *>(call)(
          &c.desc, rope, (int32_t)tokens, starts, (int32_t)heads, q, &qs, q_out, &os, k.data,
          &k.strides, v.data, &v.strides, positions, c.k, c.v, c.table, lens, status, stream);
    Py_END_ALLOW_THREADS
    return (long)s;
  });
}

// paged_decode_attn(entry, cache, q, lens, out, workspace, lse, scale, dev_status, stream)
PyObject *paged_decode_attn(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!args_are(n, 10)) return nullptr;
  return guarded([&] {
    void *call = entry(a[0]);
    const float scale = scale_of(a[7]);
    const Cache &c = cache_of(a[1]);
    need(c10::cuda::current_device() == c.device, kDevice);
    const Tokens q(a[2], c, false);
    need(q.dim == 3 && q.lead[0] == c.desc.batch, "q must be [B][Hq][d]");
    need(a[3] != Py_None && a[4] != Py_None && a[5] != Py_None, "expected a tensor");
    const int32_t *lens = dense<int32_t>(a[3], c.device, at::kInt, "lens must be int32 [B]", c.desc.batch);
    const at::Tensor &o = tensor(a[4]);
    need(o.dim() == 3 && o.size(0) == q.lead[0] && o.size(1) == q.heads &&
             o.size(2) == c.desc.head_dim,
         "out must be fp32 [B][Hq][d]");
    float *out = dense<float>(a[4], c.device, at::kFloat, "out must be fp32 [B][Hq][d]");
    const at::Tensor &w = tensor(a[5]);
    need(w.get_device() == c.device, kDevice);
    need(w.is_contiguous(), "expected a contiguous tensor");
    float *lse = nullptr;
    if (a[6] != Py_None) {
      const at::Tensor &t = tensor(a[6]);
      need(t.dim() == 2 && t.size(0) == q.lead[0] && t.size(1) == q.heads,
           "lse must be fp32 [B][Hq]");
      lse = dense<float>(a[6], c.device, at::kFloat, "lse must be fp32 [B][Hq]");
    }
    int32_t *status = dense<int32_t>(a[8], c.device, at::kInt, "dev_status must be int32");
    void *stream = stream_of(a[9]);
    ripple_status s;
    Py_BEGIN_ALLOW_THREADS
    if (c.codes() != nullptr)
      s = reinterpret_cast<decltype(ripple_paged_decode_attn_q8) *>(call)(
          &c.desc, &c.scales, (int32_t)q.heads, scale, q.data, &q.strides, c.k, c.v, c.table, lens,
          out, lse, w.data_ptr(), w.nbytes(), status, stream);
    else
      s = reinterpret_cast<decltype(ripple_paged_decode_attn) *>(call)(
          &c.desc, (int32_t)q.heads, scale, q.data, &q.strides, c.k, c.v, c.table, lens, out, lse,
          w.data_ptr(), w.nbytes(), status, stream);
    Py_END_ALLOW_THREADS
    return (long)s;
  });
}

// paged_tree_attn(entry, cache, q, lens, out, workspace, masks, seq_starts, max_tokens or None, lse,
// scale, dev_status, stream)
PyObject *paged_tree_attn(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!args_are(n, 13)) return nullptr;
  return guarded([&] {
    auto *call = entry<decltype(ripple_paged_tree_attn)>(a[0]);
    const float scale = scale_of(a[10]);
    const Cache &c = cache_of(a[1]);
    need(c10::cuda::current_device() == c.device, kDevice);
    const bool ragged = a[7] != Py_None;
    const Tokens q(a[2], c, ragged);
    need(ragged || (q.dim == 4 && q.lead[0] == c.desc.batch),
         "q must be [B][n][Hq][d], or with seq_starts [tokens][Hq][d]");
    const int64_t tokens = q.lead[0] * q.lead[1];
    need(tokens <= 0x7fffffff && q.heads <= 0x7fffffff, "too many tokens");
    need(a[3] != Py_None && a[4] != Py_None && a[5] != Py_None, "expected a tensor");
    const int32_t *lens = dense<int32_t>(a[3], c.device, at::kInt, "lens must be int32 [B]", c.desc.batch);
    const at::Tensor &t = tensor(a[2]), &o = tensor(a[4]);
    need(o.sizes() == t.sizes(), "out must have q's shape and dtype");
    void *out = dense<void>(a[4], c.device, c.type, "out must have q's shape and dtype");
    const at::Tensor &w = tensor(a[5]);
    need(w.get_device() == c.device, kDevice);
    need(w.is_contiguous(), "expected a contiguous tensor");
    const at::IntArrayRef lead = t.sizes().slice(0, t.dim() - 2);
    const uint64_t *masks = nullptr;
    if (a[6] != Py_None) {
      need(tensor(a[6]).sizes() == lead, "masks must be int64 with q's leading sizes");
      masks = dense<uint64_t>(a[6], c.device, at::kLong, "masks must be int64 with q's leading sizes");
    }
    const int32_t *starts = dense<int32_t>(a[7], c.device, at::kInt,
                                           "seq_starts must be int32 [B + 1]",
                                           (int64_t)c.desc.batch + 1);
    int64_t most = RIPPLE_MAX_DRAFT;
    if (a[8] != Py_None) {
      most = PyLong_AsLongLong(a[8]);
      if (PyErr_Occurred()) throw Refused{nullptr};
      need(most >= 0 && most <= RIPPLE_MAX_DRAFT, "too many tokens of a sequence");
    } else if (!ragged) {
      most = std::max<int64_t>(1, q.lead[1]);
      need(most <= RIPPLE_MAX_DRAFT, "too many tokens of a sequence");
    }
    float *lse = nullptr;
    if (a[9] != Py_None) {
      need(tensor(a[9]).sizes() == t.sizes().slice(0, t.dim() - 1), "lse must be fp32 [..][Hq]");
      lse = dense<float>(a[9], c.device, at::kFloat, "lse must be fp32 [..][Hq]");
    }
    int32_t *status = dense<int32_t>(a[11], c.device, at::kInt, "dev_status must be int32");
    void *stream = stream_of(a[12]);
    ripple_status s;
    Py_BEGIN_ALLOW_THREADS
    s = call(&c.desc, c.codes(), (int32_t)tokens, starts, (int32_t)most, masks, (int32_t)q.heads,
             scale, q.data, &q.strides, c.k, c.v, c.table, lens, out, lse, w.data_ptr(), w.nbytes(),
             status, stream);
    Py_END_ALLOW_THREADS
    return (long)s;
  });
}

struct KeepLayers {
  ripple_paged_desc desc;
  std::vector<ripple_paged_scales> scales;  // of 8-bit pages
  std::vector<void *> k, v;
  std::vector<const int32_t *> tables;
  int device;
};

// A cache's pools (and scales), in bytes.
struct Places {
  ripple::RowSet rows;
  long long inner;
};
void add_places(const Cache &c, std::vector<Places> *to) {
  const ripple_paged_desc &d = c.desc;
  const long long elem = c.codes() != nullptr ? 1 : c.type == at::kBFloat16 ? 2 : 4;
  const auto add = [&](const void *at, long long row, long long head, long long page, long long inner) {
    to->push_back({{(long long)(uintptr_t)at, {row, head, page}, {d.page_size, d.n_kv_heads, d.n_pages}},
                   inner});
  };
  for (const void *at : {c.k, c.v})
    add(at, d.row_stride * elem, d.head_stride * elem, d.page_stride * elem, d.head_dim * elem);
  if (c.codes() != nullptr)
    for (const void *at : {c.scales.k_scales, c.scales.v_scales})
      add(at, c.scales.row_stride, c.scales.head_stride, c.scales.page_stride, 1);
}

// keep_tables(list of caches' handles): a handle of all of them. Every layer's rows are moved at the
// same time, so that no two layers may have a place in common, nor a layer's keys, values and scales.
PyObject *keep_tables(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!args_are(n, 1)) return nullptr;
  PyObject *o = nullptr;
  try {
    need(PyList_Check(a[0]) && PyList_GET_SIZE(a[0]) >= 1, "expected a list of caches");
    auto kept = std::make_unique<KeepLayers>();
    std::vector<Places> places;
    for (Py_ssize_t i = 0; i < PyList_GET_SIZE(a[0]); ++i) {
      const Cache &c = cache_of(PyList_GET_ITEM(a[0], i));
      if (i == 0) {
        kept->desc = c.desc;
        kept->device = c.device;
      }
      kept->k.push_back(c.k);
      kept->v.push_back(c.v);
      kept->tables.push_back(c.table);
      if (c.codes() != nullptr) kept->scales.push_back(c.scales);
      add_places(c, &places);
    }
    for (size_t i = 0; i < places.size(); ++i)
      for (size_t j = 0; j < i; ++j)
        need(!ripple::overlap(places[i].rows, places[j].rows, places[i].inner, places[j].inner),
             "the layers' pools and scales must be apart");
    need(kept->scales.empty() || kept->scales.size() == kept->k.size(), "caches of one kind");
    o = PyCapsule_New(kept.get(), "ripple_keep_tables", [](PyObject *self) {
      delete static_cast<KeepLayers *>(PyCapsule_GetPointer(self, "ripple_keep_tables"));
    });
    if (o != nullptr) kept.release();
  } catch (const Refused &r) {
    if (r.why != nullptr) PyErr_SetString(PyExc_ValueError, r.why);
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return o;
}

// paged_keep_rows(entry, tables, lens, kept, tokens per sequence or None, seq_starts, lens_out,
// dev_status, stream)
PyObject *paged_keep_rows(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!args_are(n, 9)) return nullptr;
  return guarded([&] {
    auto *call = entry<decltype(ripple_paged_keep_rows)>(a[0]);
    const auto *t = static_cast<const KeepLayers *>(PyCapsule_GetPointer(a[1], "ripple_keep_tables"));
    if (t == nullptr) throw Refused{nullptr};
    need(c10::cuda::current_device() == t->device, kDevice);
    const int64_t L = (int64_t)t->k.size(), B = t->desc.batch;
    const char *const lens_are = "lens and lens_out must be int32 [L][B]";
    int32_t *lens[2];
    for (int i = 0; i < 2; ++i) {
      const at::Tensor &x = tensor(a[i == 0 ? 2 : 6]);
      need(x.dim() == 2 && x.size(0) == L && x.size(1) == B, lens_are);
      lens[i] = dense<int32_t>(a[i == 0 ? 2 : 6], t->device, at::kInt, lens_are);
    }
    const at::Tensor &kept = tensor(a[3]);
    need(kept.dim() == 2 && kept.size(0) == B, "kept must be int32 [B][m]");
    const int32_t *entries = dense<int32_t>(a[3], t->device, at::kInt, "kept must be int32 [B][m]");
    const int64_t most = kept.size(1);
    need(most <= 0x7fffffff, "too many kept tokens");
    need((a[4] == Py_None) != (a[5] == Py_None), "n_tokens or seq_starts");
    int64_t tokens = 0;
    if (a[4] != Py_None) {
      tokens = PyLong_AsLongLong(a[4]);
      if (PyErr_Occurred()) throw Refused{nullptr};
      need(tokens >= 0 && tokens <= 0x7fffffff / B, "bad number of drafted tokens");
      tokens *= B;
    }
    const int32_t *starts = dense<int32_t>(a[5], t->device, at::kInt,
                                           "seq_starts must be int32 [B + 1]", B + 1);
    int32_t *status = dense<int32_t>(a[7], t->device, at::kInt, "dev_status must be int32");
    void *stream = stream_of(a[8]);
    ripple_status s;
    Py_BEGIN_ALLOW_THREADS
    s = call(&t->desc, t->scales.empty() ? nullptr : t->scales.data(), (int32_t)L, t->k.data(),
             t->v.data(), t->tables.data(), (int32_t)tokens, starts, (int32_t)most,
             most > 0 ? entries : nullptr, lens[0], lens[1], status, stream);
    Py_END_ALLOW_THREADS
    return (long)s;
  });
}

// token_logprobs(entry, logits, tokens, logprob_out, entropy_out, lse_out, top_idx, top_logprob,
// scale, dev_status, stream)
PyObject *token_logprobs(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!args_are(n, 11)) return nullptr;
  return guarded([&] {
    auto *call = entry<decltype(ripple_token_logprobs)>(a[0]);
    const float scale = scale_of(a[8]);
    const at::Tensor &x = tensor(a[1]);
    need(x.dim() == 2 && (x.stride(1) == 1 || x.size(1) == 1),
         "logits must be [n][V], a row's logits consecutive");
    need(x.scalar_type() == at::kFloat || x.scalar_type() == at::kBFloat16,
         "logits must be fp32 or bf16");
    const int64_t rows = x.size(0), vocab = x.size(1);
    need(rows <= 0x7fffffff && vocab <= 0x7fffffff, "too many logits");
    need(x.is_cuda() && x.get_device() == c10::cuda::current_device(), kDevice);
    const int device = x.get_device();
    need((a[2] == Py_None) == (a[3] == Py_None), "tokens and logprob_out go together");
    const int32_t *tokens = dense<int32_t>(a[2], device, at::kInt, "tokens must be int32 [n]", rows);
    float *logprob = dense<float>(a[3], device, at::kFloat, "outputs must be fp32 [n]", rows);
    float *entropy = dense<float>(a[4], device, at::kFloat, "outputs must be fp32 [n]", rows);
    float *lse = dense<float>(a[5], device, at::kFloat, "outputs must be fp32 [n]", rows);
    int32_t *idx = nullptr;
    float *top = nullptr;
    int64_t k = 0;
    need(a[6] != Py_None || a[7] == Py_None, "top_logprob needs top_idx");
    if (a[6] != Py_None) {
      const at::Tensor &t = tensor(a[6]);
      need(t.dim() == 2 && t.size(0) == rows, "top_idx must be int32 [n][K]");
      k = t.size(1);
      idx = dense<int32_t>(a[6], device, at::kInt, "top_idx must be int32 [n][K]");
      if (a[7] != Py_None) {
        const at::Tensor &u = tensor(a[7]);
        need(u.dim() == 2 && u.size(0) == rows && u.size(1) == k,
             "top_logprob must be fp32, top_idx's shape");
        top = dense<float>(a[7], device, at::kFloat, "top_logprob must be fp32, top_idx's shape");
      }
      need(k <= RIPPLE_MAX_TOP, "too many alternatives");
    }
    int32_t *status = dense<int32_t>(a[9], device, at::kInt, "dev_status must be int32");
    void *stream = stream_of(a[10]);
    ripple_status s;
    Py_BEGIN_ALLOW_THREADS
    s = call((int32_t)rows, (int32_t)vocab, x.stride(0),
             x.scalar_type() == at::kFloat ? RIPPLE_F32 : RIPPLE_BF16, scale, (int32_t)k,
             x.data_ptr(), tokens, logprob, entropy, lse, k > 0 ? idx : nullptr,
             k > 0 ? top : nullptr, status, stream);
    Py_END_ALLOW_THREADS
    return (long)s;
  });
}

#define RIPPLE_METHOD(name) \
  {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(name)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {RIPPLE_METHOD(cache), RIPPLE_METHOD(paged_append),
                          RIPPLE_METHOD(paged_decode_attn), RIPPLE_METHOD(paged_tree_attn),
                          RIPPLE_METHOD(keep_tables), RIPPLE_METHOD(paged_keep_rows),
                          RIPPLE_METHOD(token_logprobs),
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, kMethods,
                       nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&kModule); }
