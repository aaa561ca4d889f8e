// Argument marshalling of the calls that a serving program makes per layer and token:
// checks of the tensors, their pointers and strides, the current stream, and the call of
// the library's entry point (whose address is given, so that the bounds-checked library is
// called the same way). A pass of ripple_paged_append through ctypes took 9.1 us of the
// host's time on a GB300's Grace, 2 of them the launch; through these functions 3.6.
#include <Python.h>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "ripple.h"

namespace {

struct Cache {
  ripple_paged_desc desc;
  void *k, *v;
  const int32_t *table;
  int device;
  at::ScalarType type;
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

template <typename F>
F *entry(PyObject *o) {
  void *f = PyLong_AsVoidPtr(o);
  if (f == nullptr) throw Refused{PyErr_Occurred() ? nullptr : "no entry point"};
  return reinterpret_cast<F *>(f);
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

// cache(desc address, k, v, table addresses, device, is bf16)
PyObject *cache(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!args_are(n, 6)) return nullptr;
  const void *desc = PyLong_AsVoidPtr(a[0]);
  Cache c;
  c.k = PyLong_AsVoidPtr(a[1]);
  c.v = PyLong_AsVoidPtr(a[2]);
  c.table = static_cast<const int32_t *>(PyLong_AsVoidPtr(a[3]));
  c.device = (int)PyLong_AsLong(a[4]);
  c.type = PyObject_IsTrue(a[5]) == 1 ? at::kBFloat16 : at::kFloat;
  if (PyErr_Occurred()) return nullptr;
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

// paged_append(entry, cache, rope address or None, lens, k, v, positions, seq_starts, q, q_out,
// dev_status, stream)
PyObject *paged_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!args_are(n, 12)) return nullptr;
  return guarded([&] {
    auto *call = entry<decltype(ripple_paged_append)>(a[0]);
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
    s = call(&c.desc, rope, (int32_t)tokens, starts, (int32_t)heads, q, &qs, q_out, &os, k.data,
             &k.strides, v.data, &v.strides, positions, c.k, c.v, c.table, lens, status, stream);
    Py_END_ALLOW_THREADS
    return (long)s;
  });
}

// paged_decode_attn(entry, cache, q, lens, out, workspace, lse, scale, dev_status, stream)
PyObject *paged_decode_attn(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!args_are(n, 10)) return nullptr;
  return guarded([&] {
    auto *call = entry<decltype(ripple_paged_decode_attn)>(a[0]);
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
    s = call(&c.desc, (int32_t)q.heads, scale, q.data, &q.strides, c.k, c.v, c.table, lens,
             out, lse, w.data_ptr(), w.nbytes(), status, stream);
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
                          RIPPLE_METHOD(paged_decode_attn), RIPPLE_METHOD(token_logprobs),
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, kMethods,
                       nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&kModule); }
