// Marshalling of the attention calls: what binding.py does with ctypes for the other entry points, as a Python extension, since a
// decode step's attention is shorter (9 us) than that took (16 us a call; here 7).  Checks the tensors, allocates outputs, hands addresses
// and the current stream to the library's C functions, whose addresses and exception class binding.py gives (bind()).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/Functions.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <climits>
#include <cmath>

#include "../../include/fpt.h"

namespace {

decltype(&fpt_rope_append) c_rope_append;
decltype(&fpt_kv_gather) c_kv_gather;
decltype(&fpt_attn_decode) c_attn_decode;
decltype(&fpt_attn_prompt) c_attn_prompt;
PyObject* error_class;            // FptError(code, where)
PyObject* allocator;              // None, or allocator(is_float32, rows, columns, device index) -> tensor

struct Refused {};                // the Python error is set

[[noreturn]] void refuse(const char* where, int code) {
  PyObject* e = PyObject_CallFunction(error_class, "is", code, where);
  if (e) {
    PyErr_SetObject(error_class, e);
    Py_DECREF(e);
  }
  throw Refused{};
}

int64_t whole(PyObject* o) {
  const int64_t v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused{};
  return v;
}

int whole32(PyObject* o, const char* where) {
  const int64_t v = whole(o);
  if (v != (int)v) refuse(where, FPT_ERR_BAD_ARG);
  return (int)v;
}

bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Refused{};
  return v != 0;
}

// One call: its name for errors, the device that all of its tensors lie on, the current stream there.
struct Call {
  const char* where;
  c10::DeviceIndex dev;
  void* stream;

  Call(const char* name, const at::Tensor& first) : where(name) {
    if (!first.is_cuda() || first.get_device() != c10::cuda::current_device()) refuse(where, FPT_ERR_BAD_ARG);
    dev = first.get_device();
    stream = c10::cuda::getCurrentCUDAStream(dev).stream();
  }
  static const at::Tensor& tensor(PyObject* o, const char* where) {
    if (!THPVariable_Check(o)) refuse(where, FPT_ERR_BAD_ARG);
    return THPVariable_Unpack(o);
  }
  void need(bool ok) const {
    if (!ok) refuse(where, FPT_ERR_BAD_ARG);
  }
  const at::Tensor& on(PyObject* o, at::ScalarType type) const {
    const at::Tensor& t = tensor(o, where);
    need(t.scalar_type() == type && t.is_cuda() && t.get_device() == dev);
    return t;
  }
  // bf16 [rows, columns] with contiguous rows
  const at::Tensor& rows(PyObject* o) const {
    const at::Tensor& t = on(o, at::kBFloat16);
    need(t.dim() == 2 && t.stride(1) == 1 && t.size(0) <= INT_MAX && t.size(1) <= INT_MAX && t.stride(0) <= INT_MAX);
    return t;
  }
  static int ld(const at::Tensor& t) { return (int)(t.size(0) > 1 ? t.stride(0) : std::max(t.stride(0), t.size(1))); }
  const int32_t* indices(PyObject* o, int64_t n) const {
    const at::Tensor& t = on(o, at::kInt);
    need(t.dim() == 1 && t.size(0) == n && (n < 2 || t.stride(0) == 1));
    return static_cast<const int32_t*>(t.data_ptr());
  }
  const at::Tensor& scratch(PyObject* o) const {
    const at::Tensor& t = on(o, at::kByte);
    need(t.is_contiguous());
    return t;
  }
  // the caller's tensor, or a new one
  PyObject* result(PyObject* given, bool f32, int64_t n_rows, int64_t cols) const {
    if (given != Py_None) {
      const at::Tensor& t = rows(given);
      need(t.size(0) == n_rows && t.size(1) == cols);
      return Py_NewRef(given);
    }
    if (allocator != Py_None) {
      PyObject* t = PyObject_CallFunction(allocator, "iLLi", (int)f32, (long long)n_rows, (long long)cols, (int)dev);
      if (t && !THPVariable_Check(t)) {
        Py_CLEAR(t);
        PyErr_SetString(PyExc_TypeError, "the allocator returned no tensor");
      }
      if (!t) throw Refused{};
      return t;
    }
    return THPVariable_Wrap(at::empty({n_rows, cols}, at::TensorOptions().dtype(f32 ? at::kFloat : at::kBFloat16).device(at::kCUDA, dev)));
  }
  void done(int code) const {
    if (code != FPT_OK) refuse(where, code);
  }
};

struct Held {                     // a reference that goes with an error
  PyObject* o = nullptr;
  ~Held() { Py_XDECREF(o); }
  PyObject* release() {
    PyObject* r = o ? o : Py_NewRef(Py_None);
    o = nullptr;
    return r;
  }
  const at::Tensor& t() const { return THPVariable_Unpack(o); }
};

PyObject* pair(Held& a, Held& b) {
  PyObject* r = PyTuple_New(2);
  if (!r) throw Refused{};
  PyTuple_SET_ITEM(r, 0, a.release());
  PyTuple_SET_ITEM(r, 1, b.release());
  return r;
}

// The five tensors of a cache, as they are at this call: a caller may put another page table or other storage in their places.
struct Cache : fpt_kv_cache {
  int64_t n_seqs;
  int dev;                        // -1: not on a GPU

  // k, v, k_scale, v_scale, pages: whether they are a cache
  bool read(PyObject* const* a) {
    for (int i = 0; i < 5; ++i)
      if (!THPVariable_Check(a[i])) return false;
    const at::Tensor &tk = THPVariable_Unpack(a[0]), &tv = THPVariable_Unpack(a[1]), &ks = THPVariable_Unpack(a[2]), &vs = THPVariable_Unpack(a[3]),
                     &table = THPVariable_Unpack(a[4]);
    if (tk.dim() != 4 || table.dim() != 2 || tk.scalar_type() != at::kChar || tv.scalar_type() != at::kChar || ks.scalar_type() != at::kFloat ||
        vs.scalar_type() != at::kFloat || table.scalar_type() != at::kInt || tv.sizes() != tk.sizes() || ks.sizes() != tk.sizes().slice(0, 2) ||
        vs.sizes() != ks.sizes() || !tk.is_contiguous() || !tv.is_contiguous() || !ks.is_contiguous() || !vs.is_contiguous() ||
        !table.is_contiguous())
      return false;
    for (const at::Tensor* t : {&tv, &ks, &vs, &table})
      if (t->device() != tk.device()) return false;
    for (int i = 0; i < 4; ++i)
      if (tk.size(i) > INT_MAX) return false;
    if (table.size(0) > INT_MAX || table.size(1) > INT_MAX) return false;
    static_cast<fpt_kv_cache&>(*this) = fpt_kv_cache{};
    k = static_cast<int8_t*>(tk.data_ptr());
    v = static_cast<int8_t*>(tv.data_ptr());
    k_scale = static_cast<float*>(ks.data_ptr());
    v_scale = static_cast<float*>(vs.data_ptr());
    pages = static_cast<const int32_t*>(table.data_ptr());
    n_pages = (int)tk.size(0);
    n_kv = (int)tk.size(1);
    page = (int)tk.size(2);
    head_dim = (int)tk.size(3);
    max_pages = (int)table.size(1);
    n_seqs = table.size(0);
    dev = tk.is_cuda() ? (int)tk.get_device() : -1;
    return true;
  }
};

template <class F>
PyObject* guarded(F f) {
  HANDLE_TH_ERRORS
  try {
    return f();
  } catch (const Refused&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

bool arguments(Py_ssize_t got, Py_ssize_t wanted) {
  if (got != wanted) PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
  return got == wanted;
}

PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arguments(n, 5)) return nullptr;
  return guarded([&]() -> PyObject* {
    c_rope_append = reinterpret_cast<decltype(c_rope_append)>(whole(a[0]));
    c_kv_gather = reinterpret_cast<decltype(c_kv_gather)>(whole(a[1]));
    c_attn_decode = reinterpret_cast<decltype(c_attn_decode)>(whole(a[2]));
    c_attn_prompt = reinterpret_cast<decltype(c_attn_prompt)>(whole(a[3]));
    Py_XSETREF(error_class, Py_NewRef(a[4]));
    if (!allocator) allocator = Py_NewRef(Py_None);
    Py_RETURN_NONE;
  });
}

PyObject* set_allocator(PyObject*, PyObject* fn) {
  Py_XSETREF(allocator, Py_NewRef(fn));
  Py_RETURN_NONE;
}

// (k, v, k_scale, v_scale, pages) -> fpt_kv_cache as bytes, or None if they are no cache
PyObject* describe_cache(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arguments(n, 5)) return nullptr;
  return guarded([&]() -> PyObject* {
    Cache c;
    if (!c.read(a)) Py_RETURN_NONE;
    return PyBytes_FromStringAndSize(reinterpret_cast<const char*>(static_cast<fpt_kv_cache*>(&c)), (Py_ssize_t)sizeof(fpt_kv_cache));
  });
}

// QKV, n_q, the cache's tensors, None or (n_kv, head_dim) of a cache without storage, rope, ctx, cu_new, layout, want_k, Q, K, workspace
PyObject* rope_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arguments(n, 16)) return nullptr;
  return guarded([&]() -> PyObject* {
    const char* where = "fpt_rope_append";
    Call c(where, Call::tensor(a[0], where));
    const at::Tensor& x = c.rows(a[0]);
    const int n_q = whole32(a[1], where);
    Cache cache{};
    if (a[7] == Py_None) {
      c.need(cache.read(a + 2) && cache.k && cache.dev == c.dev);
    } else {
      c.need(PyTuple_Check(a[7]) && PyTuple_GET_SIZE(a[7]) == 2);
      cache.n_kv = whole32(PyTuple_GET_ITEM(a[7], 0), where);
      cache.head_dim = whole32(PyTuple_GET_ITEM(a[7], 1), where);
    }
    const at::Tensor &rope = c.on(a[8], at::kFloat), &ctx = c.on(a[9], at::kInt), &ws = c.scratch(a[15]);
    const int64_t M = x.size(0), hd = cache.head_dim, n_kv = cache.n_kv;
    c.need(rope.dim() == 3 && rope.size(2) == 2 && rope.is_contiguous() && rope.size(0) <= INT_MAX && rope.size(1) <= 1024 && ctx.dim() == 1);
    const int64_t n_seqs = ctx.size(0);
    c.need(n_q >= 0 && n_kv >= 0 && hd >= 0 && n_seqs <= INT_MAX && x.size(1) >= (n_q + 2 * n_kv) * hd);
    c.need(!cache.k || cache.n_seqs >= n_seqs);
    Held q{c.result(a[13], false, M, n_q * hd)}, k{a[14] != Py_None || truth(a[12]) ? c.result(a[14], false, M, n_kv * hd) : nullptr};
    const int32_t *cu = a[10] == Py_None ? nullptr : c.indices(a[10], n_seqs + 1), *have = c.indices(a[9], n_seqs);
    const int layout = whole32(a[11], where);
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = c_rope_append(c.stream, x.data_ptr(), (int)M, Call::ld(x), n_q, static_cast<const float*>(rope.data_ptr()), (int)rope.size(0),
                         2 * (int)rope.size(1), layout, cu, have, (int)n_seqs, &cache, q.t().data_ptr(), Call::ld(q.t()),
                         k.o ? k.t().data_ptr() : nullptr, k.o ? Call::ld(k.t()) : 0, ws.data_ptr(), (size_t)ws.numel());
    Py_END_ALLOW_THREADS
    c.done(code);
    return pair(q, k);
  });
}

// the cache's tensors, cu_out, M, first, K, V, workspace
PyObject* kv_gather(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arguments(n, 11)) return nullptr;
  return guarded([&]() -> PyObject* {
    const char* where = "fpt_kv_gather";
    const at::Tensor& cu = Call::tensor(a[5], where);
    Call c(where, cu);
    Cache cache;
    c.need(cache.read(a) && cache.k && cache.dev == c.dev);
    c.need(cu.dim() == 1 && cu.size(0) >= 1 && cu.size(0) <= INT_MAX);
    const int64_t n_seqs = cu.size(0) - 1, cols = (int64_t)cache.n_kv * cache.head_dim;
    const int M = whole32(a[6], where);
    c.need(M >= 0 && cache.n_seqs >= n_seqs);
    const int32_t *ends = c.indices(a[5], n_seqs + 1), *first = a[7] == Py_None ? nullptr : c.indices(a[7], n_seqs);
    const at::Tensor& ws = c.scratch(a[10]);
    Held k{c.result(a[8], false, M, cols)}, v{c.result(a[9], false, M, cols)};
    c.need(Call::ld(k.t()) == Call::ld(v.t()));
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = c_kv_gather(c.stream, &cache, first, ends, (int)n_seqs, M, M ? k.t().data_ptr() : nullptr, M ? v.t().data_ptr() : nullptr,
                       Call::ld(k.t()), ws.data_ptr(), (size_t)ws.numel());
    Py_END_ALLOW_THREADS
    c.done(code);
    return pair(k, v);
  });
}

float scale_of(PyObject* o, int64_t head_dim) {
  if (o == Py_None) return (float)std::pow((double)head_dim, -0.5);
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Refused{};
  return (float)v;
}

// Q, the cache's tensors, kv_len, scale, want_lse, O, workspace
PyObject* attn_decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arguments(n, 11)) return nullptr;
  return guarded([&]() -> PyObject* {
    const char* where = "fpt_attn_decode";
    Call c(where, Call::tensor(a[0], where));
    const at::Tensor& q = c.rows(a[0]);
    Cache cache;
    c.need(cache.read(a + 1) && cache.k && cache.dev == c.dev);
    const int64_t n_seqs = q.size(0), hd = cache.head_dim;
    c.need(hd > 0 && q.size(1) % hd == 0 && cache.n_seqs >= n_seqs);
    const int n_q = (int)(q.size(1) / hd);
    const int32_t* len = c.indices(a[6], n_seqs);
    const at::Tensor& ws = c.scratch(a[10]);
    const float scale = scale_of(a[7], hd);
    Held o{c.result(a[9], false, n_seqs, q.size(1))}, lse{truth(a[8]) ? c.result(Py_None, true, n_seqs, n_q) : nullptr};
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = c_attn_decode(c.stream, q.data_ptr(), Call::ld(q), n_q, &cache, len, (int)n_seqs, scale, o.t().data_ptr(), Call::ld(o.t()),
                         lse.o ? static_cast<float*>(lse.t().data_ptr()) : nullptr, ws.data_ptr(), (size_t)ws.numel());
    Py_END_ALLOW_THREADS
    c.done(code);
    return pair(o, lse);
  });
}

// Q, K, V, n_q, n_kv, cu_q, cu_k, causal, scale, want_lse, O, workspace
PyObject* attn_prompt(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arguments(n, 12)) return nullptr;
  return guarded([&]() -> PyObject* {
    const char* where = "fpt_attn_prompt";
    Call c(where, Call::tensor(a[0], where));
    const at::Tensor &q = c.rows(a[0]), &k = c.rows(a[1]), &v = c.rows(a[2]), &cu = c.on(a[5], at::kInt);
    const int n_q = whole32(a[3], where), n_kv = whole32(a[4], where);
    c.need(n_q > 0 && n_kv > 0 && q.size(1) % n_q == 0 && cu.dim() == 1 && cu.size(0) >= 1 && cu.size(0) <= INT_MAX);
    const int64_t hd = q.size(1) / n_q, n_seqs = cu.size(0) - 1;
    c.need(k.size(1) == n_kv * hd && v.sizes() == k.sizes());
    const int32_t *cu_q = c.indices(a[5], n_seqs + 1), *cu_k = a[6] == Py_None ? nullptr : c.indices(a[6], n_seqs + 1);
    const at::Tensor& ws = c.scratch(a[11]);
    const int causal = truth(a[7]);
    const float scale = scale_of(a[8], hd);
    Held o{c.result(a[10], false, q.size(0), q.size(1))}, lse{truth(a[9]) ? c.result(Py_None, true, q.size(0), n_q) : nullptr};
    int code;
    Py_BEGIN_ALLOW_THREADS
    const bool keys = k.size(0) > 0;
    code = c_attn_prompt(c.stream, q.data_ptr(), Call::ld(q), (int)q.size(0), keys ? k.data_ptr() : nullptr, Call::ld(k),
                         keys ? v.data_ptr() : nullptr, Call::ld(v), (int)k.size(0), n_q, n_kv, (int)hd, cu_q, cu_k, (int)n_seqs, causal, scale,
                         o.t().data_ptr(), Call::ld(o.t()), lse.o ? static_cast<float*>(lse.t().data_ptr()) : nullptr, ws.data_ptr(), (size_t)ws.numel());
    Py_END_ALLOW_THREADS
    c.done(code);
    return pair(o, lse);
  });
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr
PyMethodDef methods[] = {{"bind", FAST(bind)},
                         {"set_allocator", set_allocator, METH_O, nullptr},
                         {"describe_cache", FAST(describe_cache)},
                         {"rope_append", FAST(rope_append)},
                         {"kv_gather", FAST(kv_gather)},
                         {"attn_decode", FAST(attn_decode)},
                         {"attn_prompt", FAST(attn_prompt)},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
  PyObject* m = PyModule_Create(&module_def);
  if (m && PyModule_AddStringConstant(m, "abi", FPT_CALLS_ABI) < 0) Py_CLEAR(m);
  return m;
}
