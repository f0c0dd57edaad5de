// Argument marshalling of the serving calls for Python: checks the tensors and
// hands their addresses and strides to the C ABI.
//
// These calls are made once per layer and token, and their launches take about 3
// us.  Read from Python, the shapes, types, strides and devices of the dozen
// tensors of a call take twice that (9.4 us a call with ctypes); here they take
// 0.3 us.
//
// Every function takes (address of the C configuration, device, stream handle,
// tensors and numbers in the order of the Python call) and returns the call's
// status, or -1 where a tensor is not what the configuration asks for (the caller
// then says which).  The C ABI's entry points are given once, by address, with
// bind().
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>

#include "kvec.h"

namespace {

decltype(&kvec_prefill_attention) g_prefill;
decltype(&kvec_paged_append) g_append;
decltype(&kvec_paged_decode) g_decode;
decltype(&kvec_paged_evict) g_evict;

// The arguments of one call in order; `ok` goes false where one does not fit.
struct Args {
  PyObject* const* a;
  Py_ssize_t n, i = 0;
  bool ok = true;
  int dev = -1;

  Args(PyObject* const* args, Py_ssize_t count) : a(args), n(count) {}
  PyObject* next() {
    if (i < n) return a[i++];
    ok = false;
    return Py_None;
  }
  int64_t integer() {
    const long long v = PyLong_AsLongLong(next());
    if (v == -1 && PyErr_Occurred()) ok = false;
    return v;
  }
  int32_t int32() {
    const int64_t v = integer();
    if (v < INT32_MIN || v > INT32_MAX) {
      PyErr_SetString(PyExc_OverflowError, "an argument does not fit 32 bits");
      ok = false;
    }
    return (int32_t)v;
  }
  double number() {
    const double v = PyFloat_AsDouble(next());
    if (v == -1.0 && PyErr_Occurred()) ok = false;
    return v;
  }
  template <class T>
  T* address() { return reinterpret_cast<T*>((uintptr_t)integer()); }

  // A tensor of that type and shape on the call's device; null for None where it is
  // optional.
  const at::Tensor* tensor(at::ScalarType type, std::initializer_list<int64_t> shape, bool optional = false) {
    PyObject* o = next();
    if (optional && o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) {
      ok = false;
      return nullptr;
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.layout() != at::kStrided || t.scalar_type() != type || !t.is_cuda() || t.get_device() != dev ||
        t.sizes() != at::IntArrayRef(shape)) {
      ok = false;
      return nullptr;
    }
    return &t;
  }
  // ... contiguous: its address.
  template <class T>
  T* dense(at::ScalarType type, std::initializer_list<int64_t> shape, bool optional = false) {
    const at::Tensor* t = tensor(type, shape, optional);
    if (!t) return nullptr;
    if (!t->is_contiguous()) ok = false;
    return static_cast<T*>(t->data_ptr());
  }
  // ... of rows whose last dimension is contiguous: its address and leading strides.
  template <int N>
  void* rows(at::ScalarType type, std::initializer_list<int64_t> shape, int64_t (&strides)[N], bool optional = false) {
    const at::Tensor* t = tensor(type, shape, optional);
    if (!t) return nullptr;
    const at::IntArrayRef st = t->strides();
    for (int d = 0; d < N; ++d) strides[d] = st[d];
    if (st[N] != 1) ok = false;
    return t->data_ptr();
  }
  // A workspace: its address and size (None: no bytes).
  void* workspace(size_t* bytes) {
    PyObject* o = next();
    *bytes = 0;
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) {
      ok = false;
      return nullptr;
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.layout() != at::kStrided || !t.is_cuda() || t.get_device() != dev || !t.is_contiguous()) {
      ok = false;
      return nullptr;
    }
    *bytes = t.nbytes();
    return t.data_ptr();
  }
  int64_t length(Py_ssize_t at) {  // of the first dimension of argument `at`, 0 where it has none
    if (at >= n || !THPVariable_Check(a[at])) return 0;
    const at::Tensor& t = THPVariable_Unpack(a[at]);
    return t.dim() > 0 ? t.size(0) : 0;
  }
};

at::ScalarType element(int32_t dtype) { return dtype == KVEC_BF16 ? at::kBFloat16 : at::kFloat; }

// C++ exceptions of the tensor library become Python's.
template <class F>
PyObject* guarded(F f) {
  try {
    return f();
  } catch (const std::exception& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  } catch (...) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "kvec: unknown error");
    return nullptr;
  }
}
// The status of a call of the C interface, made without the interpreter's lock: a launch
// may wait for room in the device's queue, and other threads run meanwhile (0.03 us a call).
template <class F>
PyObject* status_of(F call) {
  kvec_status st;
  Py_BEGIN_ALLOW_THREADS
  st = call();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}
PyObject* unfit() { return PyErr_Occurred() ? nullptr : PyLong_FromLong(-1); }

PyObject* prefill_attention(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Args g(args, n);
    const auto* c = g.address<const kvec_attention_config>();
    if (!g.ok || !c || !g_prefill) return unfit();
    g.dev = (int)g.integer();
    const auto stream = g.address<ihipStream_t>();
    const auto dt = element(c->dtype);
    int64_t qs[3], ks[3], vs[3], os[3], ls[2];
    void* q = g.rows(dt, {c->batch, c->n_q_heads, c->q_len, c->head_dim}, qs);
    void* k = g.rows(dt, {c->batch, c->n_kv_heads, c->kv_len, c->head_dim}, ks);
    void* v = g.rows(dt, {c->batch, c->n_kv_heads, c->kv_len, c->head_dim}, vs);
    void* out = g.rows(dt, {c->batch, c->n_q_heads, c->q_len, c->head_dim}, os);
    size_t bytes;
    void* ws = g.workspace(&bytes);
    float* lse = static_cast<float*>(g.rows(at::kFloat, {c->batch, c->n_q_heads, c->q_len}, ls, true));
    const int32_t* q_lens = g.dense<int32_t>(at::kInt, {c->batch}, true);
    const int32_t* kv_lens = g.dense<int32_t>(at::kInt, {c->batch}, true);
    if (!g.ok) return unfit();
    return status_of([&] {
      return g_prefill(c, q, qs, k, ks, v, vs, q_lens, kv_lens, out, os, lse, lse ? ls : nullptr, ws, bytes, stream);
    });
  });
}

PyObject* paged_append(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Args g(args, n);
    const auto* c = g.address<const kvec_paged_config>();
    if (!g.ok || !c || !g_append) return unfit();
    g.dev = (int)g.integer();
    const auto stream = g.address<ihipStream_t>();
    const auto dt = element(c->dtype);
    const int64_t tokens = g.length(g.i), d = c->head_dim;
    int64_t qs[2], ks[2], vs[2], os[2], ps[3], ps2[3];
    void* q = g.rows(dt, {tokens, c->n_q_heads, d}, qs);
    void* k = g.rows(dt, {tokens, c->n_kv_heads, d}, ks);
    void* v = g.rows(dt, {tokens, c->n_kv_heads, d}, vs);
    const int32_t* positions = g.dense<int32_t>(at::kInt, {tokens});
    const int64_t* slots = g.dense<int64_t>(at::kLong, {tokens});
    void* q_out = g.rows(dt, {tokens, c->n_q_heads, d}, os);
    void* kp = g.rows(dt, {c->n_pages, c->n_kv_heads, c->page_size, d}, ps);
    void* vp = g.rows(dt, {c->n_pages, c->n_kv_heads, c->page_size, d}, ps2);
    void* wq = g.dense<void>(dt, {d}, true);
    void* wk = g.dense<void>(dt, {d}, true);
    const float eps = (float)g.number();
    const int64_t half = g.length(g.i);
    const double* freq = g.dense<double>(at::kDouble, {half}, true);
    float* acc = g.dense<float>(at::kFloat, {c->n_pages, c->n_kv_heads, c->page_size}, true);
    int32_t* pos = g.dense<int32_t>(at::kInt, {c->n_pages, c->n_kv_heads, c->page_size}, true);
    if (!g.ok || ps[0] != ps2[0] || ps[1] != ps2[1] || ps[2] != ps2[2]) return unfit();
    if (tokens > INT32_MAX || half > INT32_MAX / 2) return PyLong_FromLong(KVEC_ERR_UNSUPPORTED);
    return status_of([&] {
      return g_append(c, (int32_t)tokens, q, qs, k, ks, v, vs, wq, wk, eps, positions, freq, freq ? (int32_t)(2 * half) : 0,
                      slots, q_out, os, kp, vp, ps, acc, pos, stream);
    });
  });
}

PyObject* paged_decode(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Args g(args, n);
    const auto* c = g.address<const kvec_paged_config>();
    if (!g.ok || !c || !g_decode) return unfit();
    g.dev = (int)g.integer();
    const auto stream = g.address<ihipStream_t>();
    const auto dt = element(c->dtype);
    int64_t qs[2], ps[3], ps2[3];
    void* q = g.rows(dt, {c->batch, c->n_q_heads, c->head_dim}, qs);
    void* kp = g.rows(dt, {c->n_pages, c->n_kv_heads, c->page_size, c->head_dim}, ps);
    void* vp = g.rows(dt, {c->n_pages, c->n_kv_heads, c->page_size, c->head_dim}, ps2);
    const int32_t* table = g.dense<int32_t>(at::kInt, {c->batch, c->max_pages});
    const int32_t* lens = g.dense<int32_t>(at::kInt, {c->batch});
    float* out = g.dense<float>(at::kFloat, {c->batch, c->n_q_heads, c->head_dim});
    size_t bytes;
    void* ws = g.workspace(&bytes);
    const int32_t max_len = g.int32(), window = g.int32(), sinks = g.int32();
    float* lse = g.dense<float>(at::kFloat, {c->batch, c->n_q_heads}, true);
    float* acc = g.dense<float>(at::kFloat, {c->n_pages, c->n_kv_heads, c->page_size}, true);
    if (!g.ok || ps[0] != ps2[0] || ps[1] != ps2[1] || ps[2] != ps2[2]) return unfit();
    return status_of([&] {
      return g_decode(c, q, qs, kp, vp, ps, table, lens, max_len, window, sinks, out, lse, acc, ws, bytes, stream);
    });
  });
}

PyObject* paged_evict(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Args g(args, n);
    const auto* c = g.address<const kvec_paged_config>();
    if (!g.ok || !c || !g_evict) return unfit();
    g.dev = (int)g.integer();
    const auto stream = g.address<ihipStream_t>();
    const auto dt = element(c->dtype);
    int64_t ps[3], ps2[3];
    const int32_t budget = g.int32();
    void* kp = g.rows(dt, {c->n_pages, c->n_kv_heads, c->page_size, c->head_dim}, ps);
    void* vp = g.rows(dt, {c->n_pages, c->n_kv_heads, c->page_size, c->head_dim}, ps2);
    const int32_t* table = g.dense<int32_t>(at::kInt, {c->batch, c->max_pages});
    const int32_t* lens = g.dense<int32_t>(at::kInt, {c->batch});
    const int32_t* seen = g.dense<int32_t>(at::kInt, {c->batch});
    float* acc = g.dense<float>(at::kFloat, {c->n_pages, c->n_kv_heads, c->page_size});
    int32_t* pos = g.dense<int32_t>(at::kInt, {c->n_pages, c->n_kv_heads, c->page_size});
    int32_t* lens_out = g.dense<int32_t>(at::kInt, {c->batch});
    size_t bytes;
    void* ws = g.workspace(&bytes);
    const int32_t window = g.int32(), sinks = g.int32();
    int32_t* kept = g.dense<int32_t>(at::kInt, {c->batch, c->n_kv_heads, budget}, true);
    const int32_t max_len = g.int32();
    if (!g.ok || ps[0] != ps2[0] || ps[1] != ps2[1] || ps[2] != ps2[2]) return unfit();
    return status_of([&] {
      return g_evict(c, budget, window, sinks, kp, vp, ps, table, lens, seen, max_len, acc, pos, kept, lens_out, ws, bytes, stream);
    });
  });
}

// bind(addresses of the four entry points)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Args g(args, n);
  g_prefill = reinterpret_cast<decltype(g_prefill)>((uintptr_t)g.integer());
  g_append = reinterpret_cast<decltype(g_append)>((uintptr_t)g.integer());
  g_decode = reinterpret_cast<decltype(g_decode)>((uintptr_t)g.integer());
  g_evict = reinterpret_cast<decltype(g_evict)>((uintptr_t)g.integer());
  if (!g.ok) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "bind takes four addresses");
    return nullptr;
  }
  Py_RETURN_NONE;
}

PyMethodDef g_methods[] = {
    {"bind", (PyCFunction)(void (*)())bind, METH_FASTCALL, nullptr},
    {"prefill_attention", (PyCFunction)(void (*)())prefill_attention, METH_FASTCALL, nullptr},
    {"paged_append", (PyCFunction)(void (*)())paged_append, METH_FASTCALL, nullptr},
    {"paged_decode", (PyCFunction)(void (*)())paged_decode, METH_FASTCALL, nullptr},
    {"paged_evict", (PyCFunction)(void (*)())paged_evict, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_kvec_bind", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kvec_bind() { return PyModule_Create(&g_module); }
