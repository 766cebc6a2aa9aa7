// Argument marshalling of the microscaled operators' Python wrappers (binding.py), for calls whose kernel takes less time than
// a ctypes call with its checks in Python: 6 to 9 us a call that way, of which the launch is 2.  Reads the tensors' attributes
// through Python's C API (no torch headers), checks them, and calls the C entry point with the interpreter lock released.
// Returns the entry's dq_status; raises ValueError for what the entry cannot see (types, shapes, devices, sizes of buffers).
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "dartquant.h"

namespace {

// Set by bind(): the library's entry points, torch's types and its lookups of the current device and stream.
struct {
  decltype(&dq_mx_quantize) quantize;
  decltype(&dq_mx_dequantize) dequantize;
  decltype(&dq_rmsnorm_quantize) rmsnorm_quantize;
  decltype(&dq_mx_matmul) matmul;
  decltype(&dq_mx_linear) linear;
} entry;
PyObject *types[3], *current_device, *current_stream;       // types by DQ_FP32, DQ_BF16, DQ_FP16
PyObject *s_dtype, *s_shape, *s_stride, *s_get_device, *s_data_ptr, *s_nbytes, *s_is_contiguous, *s_cuda_stream;

bool as_int(PyObject* o, long long& v) {                      // takes the reference
  if (!o) return false;
  v = PyLong_AsLongLong(o);
  Py_DECREF(o);
  return v != -1 || !PyErr_Occurred();
}
bool call_int(PyObject* t, PyObject* name, long long& v) { return as_int(PyObject_CallMethodNoArgs(t, name), v); }
bool address(PyObject* t, void*& p) {
  PyObject* o = PyObject_CallMethodNoArgs(t, s_data_ptr);
  if (!o) return false;
  p = PyLong_AsVoidPtr(o);
  Py_DECREF(o);
  return p || !PyErr_Occurred();
}

struct Matrix {
  void* p = nullptr;
  long long ld = 0, rows = 0, k = 0, device = -1;
  int dtype = -1;
};

// Both entries of a tuple of two integers; -1: an error is set, 0: not two, 1: read.
int pair_of(PyObject* tuple, long long& a, long long& b) {   // takes the reference
  if (!tuple) return -1;
  int ok = 0;
  if (PyTuple_Check(tuple) && PyTuple_GET_SIZE(tuple) == 2) {
    a = PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, 0));
    b = PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, 1));
    ok = PyErr_Occurred() ? -1 : 1;
  }
  Py_DECREF(tuple);
  return ok;
}

// A matrix of values with contiguous rows on a CUDA device; with `like`, of its shape, type and device.
bool matrix(PyObject* t, const char* name, Matrix& m, const Matrix* like = nullptr) {
  PyObject* dtype = PyObject_GetAttr(t, s_dtype);
  if (!dtype) return false;
  for (int i = 0; i < 3; ++i) if (dtype == types[i]) m.dtype = i;
  Py_DECREF(dtype);
  if (!call_int(t, s_get_device, m.device)) return false;
  long long step = 0;
  const int shaped = pair_of(PyObject_GetAttr(t, s_shape), m.rows, m.k);
  if (shaped < 0) return false;
  if (!shaped || m.dtype < 0 || m.device < 0) {
    PyErr_Format(PyExc_ValueError, "%s: a 2-D CUDA tensor of float32, bfloat16 or float16 is needed", name);
    return false;
  }
  if (like && (m.rows != like->rows || m.k != like->k || m.dtype != like->dtype || m.device != like->device)) {
    PyErr_Format(PyExc_ValueError, "%s: shape, type or device differs from the input's", name);
    return false;
  }
  if (pair_of(PyObject_CallMethodNoArgs(t, s_stride), m.ld, step) != 1) return false;
  // (a single column's step means nothing, nor does a single row's stride)
  if ((step != 1 && m.k > 1) || (m.ld < m.k && m.rows > 1)) {
    PyErr_Format(PyExc_ValueError, "%s: rows have to be contiguous and must not overlap", name);
    return false;
  }
  if (m.ld < m.k) m.ld = m.k;                                 // (one row)
  return address(t, m.p);
}
// None, or a matrix like `x`
bool optional(PyObject* t, const char* name, Matrix& m, const Matrix& x) { return t == Py_None || matrix(t, name, m, &x); }

// A contiguous buffer of at least `least` bytes on a device.
bool bytes(PyObject* t, const char* name, long long least, long long device, void*& p, long long* held = nullptr) {
  long long size, where;
  if (!as_int(PyObject_GetAttr(t, s_nbytes), size) || !call_int(t, s_get_device, where)) return false;
  PyObject* c = PyObject_CallMethodNoArgs(t, s_is_contiguous);
  if (!c) return false;
  const bool contiguous = c == Py_True;
  Py_DECREF(c);
  if (size < least || where != device || !contiguous) {
    PyErr_Format(PyExc_ValueError, "%s: a contiguous buffer of at least %lld bytes on the inputs' device is needed", name, least);
    return false;
  }
  if (held) *held = size;
  return address(t, p);
}

bool format(PyObject* o, int& fmt) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) return false;
  if (v != DQ_MXFP4 && v != DQ_MXFP8) {
    PyErr_Format(PyExc_ValueError, "format %ld: DQ_MXFP4 or DQ_MXFP8 is needed", v);
    return false;
  }
  fmt = (int)v;
  return true;
}
long long row_bytes(int fmt, long long k) { return (k + 127) / 128 * (fmt == DQ_MXFP4 ? 64 : 128); }
long long code_bytes(int fmt, long long rows, long long k) { return rows * row_bytes(fmt, k); }
long long scale_bytes(long long rows, long long k) { return (rows + 127) / 128 * ((k + 127) / 128) * 512; }

// Codes of a [rows, k] matrix: a buffer of their size, whose rows, if it has two dimensions, are theirs (another k or format
// would read on as if they were).  Whatever type they have: rows are counted in bytes.
bool codes_of(PyObject* t, const char* name, int fmt, long long rows, long long k, long long device, void*& p) {
  long long held = 0;
  if (!bytes(t, name, code_bytes(fmt, rows, k), device, p, &held)) return false;
  PyObject* shape = PyObject_GetAttr(t, s_shape);
  if (!shape) return false;
  bool fits = true;
  if (PyTuple_Check(shape) && PyTuple_GET_SIZE(shape) == 2) fits = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, 0)) * row_bytes(fmt, k) == held;
  Py_DECREF(shape);
  if (!fits) PyErr_Format(PyExc_ValueError, "%s: rows of %lld bytes are needed for %lld values in this format", name, row_bytes(fmt, k), k);
  return fits;
}

// The stream (None: torch's current one), after checking that the tensors' device is the current one.
bool stream_of(PyObject* stream, const char* name, long long device, void*& s) {
  long long now;
  if (!as_int(PyObject_CallNoArgs(current_device), now)) return false;
  if (now != device) {
    PyErr_Format(PyExc_ValueError, "%s: the tensors have to be on the current CUDA device", name);
    return false;
  }
  PyObject* o;
  if (stream == Py_None) {
    PyObject* index = PyLong_FromLongLong(device);
    if (!index) return false;
    o = PyObject_CallOneArg(current_stream, index);
    Py_DECREF(index);
  } else {
    o = PyObject_GetAttr(stream, s_cuda_stream);
  }
  if (!o) return false;
  s = PyLong_AsVoidPtr(o);
  Py_DECREF(o);
  return !PyErr_Occurred();
}
bool count(Py_ssize_t n, Py_ssize_t want) {
  if (n == want && entry.quantize) return true;
  PyErr_SetString(PyExc_TypeError, "wrong number of arguments, or bind() was not called");
  return false;
}
#define DQ_CALL(expr)                 \
  dq_status status;                   \
  Py_BEGIN_ALLOW_THREADS;             \
  status = (expr);                    \
  Py_END_ALLOW_THREADS;               \
  return PyLong_FromLong((long)status)

// quantize(X, fmt, codes, scales, values, stream)
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Matrix x, v;
  int fmt;
  void *codes, *scales, *s;
  if (!count(n, 6) || !matrix(a[0], "X", x) || !format(a[1], fmt) ||
      !codes_of(a[2], "codes", fmt, x.rows, x.k, x.device, codes) ||
      !bytes(a[3], "scales", scale_bytes(x.rows, x.k), x.device, scales) || !optional(a[4], "values", v, x) ||
      !stream_of(a[5], "dq_mx_quantize", x.device, s))
    return nullptr;
  DQ_CALL(entry.quantize(x.p, x.dtype, x.rows, x.k, x.ld, fmt, codes, scales, v.p, v.ld, s));
}

// dequantize(codes, scales, fmt, Y, stream)
PyObject* dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Matrix y;
  int fmt;
  void *codes, *scales, *s;
  if (!count(n, 5) || !matrix(a[3], "Y", y) || !format(a[2], fmt) ||
      !codes_of(a[0], "codes", fmt, y.rows, y.k, y.device, codes) ||
      !bytes(a[1], "scales", scale_bytes(y.rows, y.k), y.device, scales) || !stream_of(a[4], "dq_mx_dequantize", y.device, s))
    return nullptr;
  DQ_CALL(entry.dequantize(fmt, codes, scales, y.rows, y.k, y.p, y.dtype, y.ld, s));
}

// rmsnorm_quantize(X, gamma, eps, fmt, codes, scales, residual, sum, values, stream)
PyObject* rmsnorm_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Matrix x, r, h, v;
  int fmt, g_dtype = 0;
  void *codes, *scales, *s, *gamma = nullptr;
  if (!count(n, 10) || !matrix(a[0], "X", x) || !format(a[3], fmt)) return nullptr;
  const double eps = PyFloat_AsDouble(a[2]);
  if (eps == -1.0 && PyErr_Occurred()) return nullptr;
  g_dtype = x.dtype;
  if (a[1] != Py_None) {
    PyObject *dtype = PyObject_GetAttr(a[1], s_dtype), *shape = dtype ? PyObject_GetAttr(a[1], s_shape) : nullptr;
    if (!shape) { Py_XDECREF(dtype); return nullptr; }
    const bool fp32 = dtype == types[DQ_FP32], typed = fp32 || dtype == types[x.dtype];
    bool shaped = PyTuple_Check(shape) && PyTuple_GET_SIZE(shape) == 1;
    if (shaped) shaped = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, 0)) == x.k;
    Py_DECREF(dtype);
    Py_DECREF(shape);
    if (!typed || !shaped) {
      PyErr_Format(PyExc_ValueError, "gamma: a [%lld] tensor of X's type or float32 is needed", x.k);
      return nullptr;
    }
    if (fp32) g_dtype = DQ_FP32;
    if (!bytes(a[1], "gamma", 0, x.device, gamma)) return nullptr;
  }
  if (!codes_of(a[4], "codes", fmt, x.rows, x.k, x.device, codes) ||
      !bytes(a[5], "scales", scale_bytes(x.rows, x.k), x.device, scales) || !optional(a[6], "residual", r, x) ||
      !optional(a[7], "sum_out", h, x) || !optional(a[8], "values", v, x) || !stream_of(a[9], "dq_rmsnorm_quantize", x.device, s))
    return nullptr;
  DQ_CALL(entry.rmsnorm_quantize(x.p, r.p, x.dtype, x.rows, x.k, x.ld, r.ld, gamma, g_dtype, (float)eps, fmt, codes, scales, h.p,
                                 h.ld, v.p, v.ld, s));
}

// matmul(a_codes, a_scales, a_fmt, w_codes, w_scales, k, Y, stream)
PyObject* matmul(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Matrix y;
  int fmt;
  void *ac, *as, *wc, *ws, *s;
  if (!count(n, 8) || !matrix(a[6], "Y", y) || !format(a[2], fmt)) return nullptr;
  const long long k = PyLong_AsLongLong(a[5]);
  if (k == -1 && PyErr_Occurred()) return nullptr;
  if (k < 0 || k > (1LL << 40)) { PyErr_SetString(PyExc_ValueError, "k: out of range"); return nullptr; }
  if (!codes_of(a[0], "a_codes", fmt, y.rows, k, y.device, ac) ||
      !bytes(a[1], "a_scales", scale_bytes(y.rows, k), y.device, as) ||
      !codes_of(a[3], "w_codes", DQ_MXFP4, y.k, k, y.device, wc) ||
      !bytes(a[4], "w_scales", scale_bytes(y.k, k), y.device, ws) || !stream_of(a[7], "dq_mx_matmul", y.device, s))
    return nullptr;
  DQ_CALL(entry.matmul(fmt, ac, as, y.rows, wc, ws, y.k, k, y.p, y.dtype, y.ld, s));
}

// linear(X, a_fmt, w_codes, w_scales, Y, workspace, stream)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Matrix x, y;
  int fmt;
  void *wc, *ws, *work, *s;
  if (!count(n, 7) || !matrix(a[0], "X", x) || !format(a[1], fmt) || !matrix(a[4], "Y", y)) return nullptr;
  if (y.rows != x.rows || y.device != x.device) {
    PyErr_Format(PyExc_ValueError, "Y: %lld rows on X's device are needed", x.rows);
    return nullptr;
  }
  if (!codes_of(a[2], "w_codes", DQ_MXFP4, y.k, x.k, x.device, wc) ||
      !bytes(a[3], "w_scales", scale_bytes(y.k, x.k), x.device, ws) ||
      !bytes(a[5], "workspace", code_bytes(fmt, x.rows, x.k) + scale_bytes(x.rows, x.k), x.device, work) ||
      !stream_of(a[6], "dq_mx_linear", x.device, s))
    return nullptr;
  DQ_CALL(entry.linear(x.p, x.dtype, x.rows, x.k, x.ld, fmt, wc, ws, y.k, y.p, y.dtype, y.ld, work, s));
}

// bind((five entry addresses in the order above), (float32, bfloat16, float16), current_device, current_raw_stream)
PyObject* bind(PyObject*, PyObject* args) {
  PyObject *at, *t, *device, *stream;
  if (!PyArg_ParseTuple(args, "O!O!OO", &PyTuple_Type, &at, &PyTuple_Type, &t, &device, &stream)) return nullptr;
  if (PyTuple_GET_SIZE(at) != 5 || PyTuple_GET_SIZE(t) != 3) { PyErr_SetString(PyExc_TypeError, "bind: five entries, three types"); return nullptr; }
  void* p[5];
  for (int i = 0; i < 5; ++i) {
    p[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(at, i));
    if (!p[i]) { if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind: a null entry"); return nullptr; }
  }
  for (int i = 0; i < 3; ++i) { PyObject* o = PyTuple_GET_ITEM(t, i); Py_INCREF(o); Py_XSETREF(types[i], o); }
  Py_INCREF(device); Py_XSETREF(current_device, device);
  Py_INCREF(stream); Py_XSETREF(current_stream, stream);
  entry.quantize = (decltype(entry.quantize))p[0];
  entry.dequantize = (decltype(entry.dequantize))p[1];
  entry.rmsnorm_quantize = (decltype(entry.rmsnorm_quantize))p[2];
  entry.matmul = (decltype(entry.matmul))p[3];
  entry.linear = (decltype(entry.linear))p[4];
  Py_RETURN_NONE;
}

#define DQ_FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {DQ_FAST(quantize), DQ_FAST(dequantize), DQ_FAST(rmsnorm_quantize), DQ_FAST(matmul), DQ_FAST(linear),
                         {"bind", bind, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", "Checked calls of the microscaled operators.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void) {
  const struct { PyObject** to; const char* name; } names[] = {
      {&s_dtype, "dtype"}, {&s_shape, "shape"}, {&s_stride, "stride"}, {&s_get_device, "get_device"}, {&s_data_ptr, "data_ptr"},
      {&s_nbytes, "nbytes"}, {&s_is_contiguous, "is_contiguous"}, {&s_cuda_stream, "cuda_stream"}};
  for (const auto& n : names)
    if (!(*n.to = PyUnicode_InternFromString(n.name))) return nullptr;
  return PyModule_Create(&module);
}
