// The token operators' calls from torch tensors: a Python extension that reads what the entry points of include/laud.h take (pointers,
// sizes, distances of rows, the current stream) from the tensors and checks what a pointer no longer tells (device, type, shape).
// Marshalling only, as the ctypes binding of the other entry points; in C++ because a call on a few rows is a launch of two or three
// microseconds, which reading five tensors' attributes in Python would double.  The functions return the status.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "laud.h"

namespace {

// Entry points of the loaded library, handed over by bind().
decltype(&laud_norm_residual) p_norm = nullptr;
decltype(&laud_quantize_e4m3) p_quantize = nullptr;
decltype(&laud_matmul_e4m3) p_matmul = nullptr;
decltype(&laud_moe) p_moe = nullptr;

struct Refused {};  // an argument that does not fit: LAUD_ERR_INVALID_ARG

int code_of(at::ScalarType t) {
  return t == at::kFloat ? LAUD_F32 : t == at::kBFloat16 ? LAUD_BF16 : t == at::kFloat8_e4m3fn ? LAUD_E4M3 : -1;
}
int64_t blocks(int64_t n) { return (n + 127) / 128; }

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) throw Refused{};
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || t.get_device() != c10::hip::current_device()) throw Refused{};
  return t;
}

// Rows of a matrix: contiguous ones, any distance apart.
struct Rows {
  void* p = nullptr;
  int64_t n = 0, c = 0, ld = 0;
  int code = -1;
};
Rows rows(PyObject* o) {
  const at::Tensor& t = tensor(o);
  if (t.dim() != 2) throw Refused{};
  Rows r;
  r.n = t.size(0);
  r.c = t.size(1);
  if ((t.stride(1) != 1 && r.c != 1) || r.n > INT32_MAX || r.c > INT32_MAX) throw Refused{};
  r.ld = r.n > 1 ? t.stride(0) : r.c;
  r.p = t.data_ptr();
  r.code = code_of(t.scalar_type());
  return r;
}
Rows rows(PyObject* o, int64_t n, int64_t c) {
  const Rows r = rows(o);
  if (r.n != n || r.c != c) throw Refused{};
  return r;
}
// A dense float32 matrix, of n rows or, with `more`, of at least as many; None: null.
float* floats(PyObject* o, int64_t n, int64_t c, bool more = false) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o);
  if (t.scalar_type() != at::kFloat || t.dim() != 2 || t.size(0) < n || (!more && t.size(0) != n) || t.size(1) != c ||
      !t.is_contiguous())
    throw Refused{};
  return static_cast<float*>(t.data_ptr());
}
// A byte (or truth value) per row; None: null.
uint8_t* bytes(PyObject* o, int64_t n) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o);
  if (t.element_size() != 1 || t.is_floating_point() || t.numel() != n || !t.is_contiguous()) throw Refused{};
  return static_cast<uint8_t*>(t.data_ptr());
}
// A workspace: any contiguous device tensor; None: null.
void* space(PyObject* o, size_t* n) {
  *n = 0;
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o);
  if (!t.is_contiguous()) throw Refused{};
  *n = t.nbytes();
  return t.data_ptr();
}
int64_t integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if ((v == -1 && PyErr_Occurred()) || v < INT32_MIN || v > INT32_MAX) {
    PyErr_Clear();
    throw Refused{};
  }
  return v;
}
// A descriptor made by the ctypes binding.
template <typename T>
T descriptor(PyObject* o) {
  Py_buffer b;
  if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) {
    PyErr_Clear();
    throw Refused{};
  }
  const bool fits = b.len == (Py_ssize_t)sizeof(T);
  T v{};
  if (fits) v = *static_cast<const T*>(b.buf);
  PyBuffer_Release(&b);
  if (!fits) throw Refused{};
  return v;
}
void* stream() { return c10::hip::getCurrentHIPStream().stream(); }

template <typename F>
PyObject* status_of(Py_ssize_t got, Py_ssize_t want, F&& call) {
  if (got != want) {
    PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", want, got);
    return nullptr;
  }
  try {
    return PyLong_FromLong(call());
  } catch (const Refused&) {
    return PyLong_FromLong(LAUD_ERR_INVALID_ARG);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

PyObject* norm_residual(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return status_of(n, 9, [&] {
    const auto p = descriptor<laud_norm_block>(a[0]);
    const Rows x = rows(a[1]);
    if (x.c != p.C || x.code != p.dtype) throw Refused{};
    Rows y, out, z;
    if (a[2] != Py_None && (y = rows(a[2], x.n, x.c)).code != x.code) throw Refused{};
    if (a[6] != Py_None && (out = rows(a[6], x.n, x.c)).code != x.code) throw Refused{};
    int z_dtype = x.code;
    if (a[7] != Py_None) {
      z = rows(a[7], x.n, x.c);
      z_dtype = z.code;
      if (z.code != x.code && z.code != LAUD_E4M3) throw Refused{};
    }
    const int64_t per = integer(a[5]);
    float* gate = nullptr;
    if (a[4] != Py_None) {
      if (per <= 0) throw Refused{};
      gate = floats(a[4], (x.n + per - 1) / per, x.c, true);
    }
    float* zs = z_dtype == LAUD_E4M3 ? floats(a[8], x.n, blocks(x.c)) : nullptr;
    return p_norm(&p, (int)x.n, x.p, x.ld, y.p, y.ld, bytes(a[3], x.n), gate, (int)per, out.p, out.ld, z.p, z.ld, z_dtype, zs, stream());
  });
}

PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return status_of(n, 4, [&] {
    const Rows x = rows(a[0]), q = rows(a[1], x.n, x.c);
    const int64_t per = integer(a[3]);
    if (q.code != LAUD_E4M3 || (per != 1 && per != 128)) throw Refused{};
    return p_quantize(x.p, x.ld, (int)x.n, (int)x.c, x.code, (int)per, q.p, q.ld, floats(a[2], (x.n + per - 1) / per, blocks(x.c)), stream());
  });
}

PyObject* matmul(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return status_of(n, 6, [&] {
    const Rows x = rows(a[0]), w = rows(a[2]);
    if (x.code != LAUD_E4M3 || w.code != LAUD_E4M3 || x.c != w.c) throw Refused{};
    const Rows out = rows(a[4], x.n, w.n);
    size_t ws_bytes;
    void* ws = space(a[5], &ws_bytes);
    return p_matmul(x.p, x.ld, floats(a[1], x.n, blocks(x.c)), w.p, w.ld, floats(a[3], blocks(w.n), blocks(x.c)), (int)x.n, (int)w.n,
                    (int)x.c, out.p, out.ld, out.code, ws, ws_bytes, stream());
  });
}

PyObject* moe(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return status_of(n, 7, [&] {
    const auto p = descriptor<laud_moe_layer>(a[0]);
    const Rows x = rows(a[1]);
    if (x.c != p.C || x.code != p.dtype) throw Refused{};
    const Rows out = rows(a[3], x.n, x.c);
    if (out.code != x.code) throw Refused{};
    int32_t* experts = nullptr;
    if (a[4] != Py_None) {
      const at::Tensor& t = tensor(a[4]);
      if (t.scalar_type() != at::kInt || t.dim() != 2 || t.size(0) != x.n || t.size(1) != p.top_k || !t.is_contiguous()) throw Refused{};
      experts = static_cast<int32_t*>(t.data_ptr());
    }
    size_t ws_bytes;
    void* ws = space(a[6], &ws_bytes);
    return p_moe(&p, (int)x.n, x.p, x.ld, bytes(a[2], x.n), out.p, out.ld, experts, floats(a[5], x.n, p.top_k), ws, ws_bytes, stream());
  });
}

template <typename F>
void take(F& f, PyObject* address) { f = reinterpret_cast<F>(PyLong_AsVoidPtr(address)); }

PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 4) {
    PyErr_SetString(PyExc_TypeError, "4 addresses");
    return nullptr;
  }
  take(p_norm, a[0]);
  take(p_quantize, a[1]);
  take(p_matmul, a[2]);
  take(p_moe, a[3]);
  if (PyErr_Occurred()) return nullptr;
  Py_RETURN_NONE;
}

#define LAUD_METHOD(f, doc) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, doc}
PyMethodDef methods[] = {LAUD_METHOD(bind, "bind(norm_residual, quantize_e4m3, matmul_e4m3, moe): addresses of the entry points"),
                         LAUD_METHOD(norm_residual, "norm_residual(block, x, y, keep, gate, rows_per_gate, out, z, z_scale) -> status"),
                         LAUD_METHOD(quantize, "quantize(x, q, scale, block_rows) -> status"),
                         LAUD_METHOD(matmul, "matmul(a, sa, b, sb, out, ws) -> status"),
                         LAUD_METHOD(moe, "moe(layer, x, keep, out, experts, weights, ws) -> status"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_laud_torch", "Calls of liblaud.so from torch tensors.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__laud_torch(void) { return PyModule_Create(&module); }
