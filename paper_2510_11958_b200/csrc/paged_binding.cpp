// Argument marshalling of the paged cache's calls for Python: types, devices and layouts of the tensors, their addresses, the
// current stream.  These calls are a few microseconds on the device; reading a dozen tensors through Python's own
// attributes and ctypes took the host 11 to 15 of them, here it is one.
//
// Every function returns the dmtd_status; a tensor of the wrong kind raises ValueError.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/dmtd.h"

namespace {

struct Bad {                                   // the exception is set
};

[[noreturn]] void bad(const char *name, const char *what) {
  PyErr_Format(PyExc_ValueError, "%s %s", name, what);
  throw Bad{};
}

struct Args {
  PyObject *const *a;
  Py_ssize_t n;
  mutable int device = -1;                     // the current one, once there is a CUDA tensor to compare it with
  Args(PyObject *const *a, Py_ssize_t n, Py_ssize_t want) : a(a), n(n) {
    if (n != want) {
      PyErr_Format(PyExc_TypeError, "%zd arguments, %zd wanted", n, want);
      throw Bad{};
    }
  }
  bool none(int i) const { return a[i] == Py_None; }
  const at::Tensor &tensor(int i, const char *name) const {
    if (!THPVariable_Check(a[i])) bad(name, "is no tensor");
    const at::Tensor &t = THPVariable_Unpack(a[i]);
    if (t.is_cuda() && device < 0) device = c10::cuda::current_device();
    if (!t.is_cuda() || t.get_device() != device) bad(name, "is not on the current CUDA device");
    return t;
  }
  int32_t *ints(int i, const char *name, int64_t count) const {
    const at::Tensor &t = tensor(i, name);
    if (t.scalar_type() != at::kInt || !t.is_contiguous()) bad(name, "must be contiguous int32");
    if (t.numel() != count) bad(name, "has the wrong size");
    return static_cast<int32_t *>(t.data_ptr());
  }
  int64_t number(int i) const {
    const int64_t v = PyLong_AsLongLong(a[i]);
    if (v == -1 && PyErr_Occurred()) throw Bad{};
    return v;
  }
  int32_t number32(int i, const char *name) const {
    const int64_t v = number(i);
    if (v != (int32_t)v) bad(name, "does not fit 32 bits");
    return (int32_t)v;
  }
  double real(int i) const {
    const double v = PyFloat_AsDouble(a[i]);
    if (v == -1.0 && PyErr_Occurred()) throw Bad{};
    return v;
  }
};

int32_t dtype_code(const at::Tensor &t, const char *name) {
  switch (t.scalar_type()) {
    case at::kFloat: return DMTD_F32;
    case at::kBFloat16: return DMTD_BF16;
    case at::kHalf: return DMTD_F16;
    default: bad(name, "must be float32, bfloat16 or float16");
  }
}

int32_t narrow(int64_t v, const char *name) {
  if (v != (int32_t)v) bad(name, "is too large");
  return (int32_t)v;
}

// [pages, kv heads, page_size, head_dim] in any order in memory
dmtd_paged_cache cache_of(const Args &A, int i) {
  const at::Tensor &k = A.tensor(i, "k_cache"), &v = A.tensor(i + 1, "v_cache");
  if (k.dim() != 4 || k.sizes() != v.sizes() || k.strides() != v.strides() || k.scalar_type() != v.scalar_type())
    bad("k_cache and v_cache", "must be four-dimensional and alike");
  if (k.stride(3) != 1 && k.size(3) != 1) bad("k_cache", "must have dense rows");
  return {k.data_ptr(), v.data_ptr(), dtype_code(k, "k_cache"), narrow(k.size(0), "k_cache"), narrow(k.size(2), "k_cache"),
          narrow(k.size(1), "k_cache"), narrow(k.size(3), "k_cache"), k.stride(0), k.stride(1), k.stride(2)};
}

// [rows, heads, head_dim] with dense heads
void check_rows(const at::Tensor &t, const char *name, int64_t rows, int64_t D) {
  if (t.dim() != 3 || t.size(0) != rows || t.size(2) != D) bad(name, "has the wrong shape");
  if (t.stride(2) != 1 || (t.stride(1) != D && t.size(1) != 1)) bad(name, "must have dense heads");
}

template <class F>
PyObject *guarded(F &&f) {
  try {
    return PyLong_FromLong(f());
  } catch (const Bad &) {
    return nullptr;
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

void *stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

// lens, n_new, table, free_pages, n_free, page_size, n_rows, row_start, position, slot, granted, lens_out, n_free_out
PyObject *plan(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> long {
    const Args A(a, n, 13);
    const at::Tensor &table = A.tensor(2, "table"), &free_pages = A.tensor(3, "free_pages");
    if (table.dim() != 2) bad("table", "must have two dimensions");
    const int64_t B = table.size(0), rows = A.number(6);
    if (rows < 0) bad("n_rows", "is negative");
    return dmtd_paged_plan(A.ints(0, "lens", B), A.ints(1, "n_new", B), narrow(B, "table"), A.number32(5, "page_size"),
                           A.ints(2, "table", table.numel()), narrow(table.size(1), "table"), A.ints(3, "free_pages", free_pages.numel()),
                           narrow(free_pages.numel(), "free_pages"), A.ints(4, "n_free", 1), A.number32(6, "n_rows"), A.ints(7, "row_start", B + 1),
                           A.ints(8, "position", rows), A.ints(9, "slot", rows), A.ints(10, "granted", B), A.ints(11, "lens", B),
                           A.ints(12, "n_free", 1), stream());
  });
}

// q or None, k, v, position, slot, k_cache, v_cache, q_norm or None, k_norm or None, eps, rope_theta, q_out or None
PyObject *append(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> long {
    const Args A(a, n, 12);
    const dmtd_paged_cache cache = cache_of(A, 5);
    const at::Tensor &k = A.tensor(1, "k"), &v = A.tensor(2, "v");
    if (k.dim() != 3) bad("k", "must have three dimensions");
    const int64_t T = k.size(0), D = cache.head_dim;
    check_rows(k, "k", T, D);
    check_rows(v, "v", T, D);
    if (k.size(1) != cache.n_kv_heads || v.size(1) != cache.n_kv_heads) bad("k and v", "have other heads than the cache");
    const int32_t type = dtype_code(k, "k");
    if (v.scalar_type() != k.scalar_type()) bad("v", "has another type than k");
    const void *q = nullptr;
    void *q_out = nullptr;
    int64_t nq = 0, q_stride = 0;
    if (!A.none(0)) {
      const at::Tensor &t = A.tensor(0, "q"), &o = A.tensor(11, "q_out");
      check_rows(t, "q", T, D);
      if (t.scalar_type() != k.scalar_type()) bad("q", "has another type than k");
      if (o.sizes() != t.sizes() || o.scalar_type() != t.scalar_type() || !o.is_contiguous()) bad("q_out", "must be contiguous and like q");
      q = t.data_ptr();
      q_out = o.data_ptr();
      nq = t.size(1);
      q_stride = t.stride(0);
    }
    const float *norm[2];
    for (int i = 0; i < 2; ++i) {
      norm[i] = nullptr;
      if (A.none(7 + i)) continue;
      const at::Tensor &w = A.tensor(7 + i, i ? "k_norm" : "q_norm");
      if (w.scalar_type() != at::kFloat || !w.is_contiguous() || w.numel() != D) bad(i ? "k_norm" : "q_norm", "must be float32 [head_dim]");
      norm[i] = static_cast<const float *>(w.data_ptr());
    }
    return dmtd_paged_append(q, k.data_ptr(), v.data_ptr(), type, q_stride, k.stride(0), v.stride(0), narrow(T, "k"), narrow(nq, "q"), norm[0],
                             norm[1], (float)A.real(9), (float)A.real(10), A.ints(3, "position", T), A.ints(4, "slot", T), &cache, q_out, stream());
  });
}

// q, row_start, lens, table, k_cache, v_cache, max_new, scratch, out
PyObject *attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> long {
    const Args A(a, n, 9);
    const dmtd_paged_cache cache = cache_of(A, 4);
    const at::Tensor &q = A.tensor(0, "q"), &table = A.tensor(3, "table"), &scratch = A.tensor(7, "scratch"), &out = A.tensor(8, "out");
    if (q.dim() != 3) bad("q", "must have three dimensions");
    check_rows(q, "q", q.size(0), cache.head_dim);
    if (table.dim() != 2) bad("table", "must have two dimensions");
    const int64_t B = table.size(0);
    if (out.sizes() != q.sizes() || out.scalar_type() != q.scalar_type() || !out.is_contiguous()) bad("out", "must be contiguous and like q");
    if (!scratch.is_contiguous()) bad("scratch", "must be contiguous");
    return dmtd_paged_attention(q.data_ptr(), dtype_code(q, "q"), q.stride(0), narrow(q.size(0), "q"), narrow(q.size(1), "q"),
                                A.ints(1, "row_start", B + 1), A.ints(2, "lens", B), narrow(B, "table"), A.ints(3, "table", table.numel()),
                                narrow(table.size(1), "table"), A.number32(6, "max_new"), &cache, scratch.data_ptr(), scratch.nbytes(), out.data_ptr(),
                                stream());
  });
}

PyMethodDef methods[] = {
    {"plan", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(plan)), METH_FASTCALL, nullptr},
    {"append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(append)), METH_FASTCALL, nullptr},
    {"attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(attention)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
// (the text is what build.py looks for in the file: the versions of torch and Python that it was compiled against)
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_paged", "Argument marshalling of the paged cache's calls " DMTD_MADE_FOR, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject *PyInit__paged() { return PyModule_Create(&module); }
