// Argument marshalling of the microscaled and key/value cache operators' Python wrappers (binding.py), for calls whose kernel takes less time than
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
struct {
  decltype(&dq_qk_norm_rope) qk_norm_rope;
  decltype(&dq_kv_append) append;
  decltype(&dq_kv_dequantize) dequantize;
  decltype(&dq_kv_attention) attention;
  decltype(&dq_kv_attention_weights) attention_weights;
  decltype(&dq_kv_evict) evict;
  decltype(&dq_kv_attention_workspace) attention_workspace;
  decltype(&dq_kv_evict_workspace) evict_workspace;
} kv_entry;                                                 // set by bind_kv()
PyObject *types[3], *current_device, *current_stream;       // types by DQ_FP32, DQ_BF16, DQ_FP16
PyObject* int32;                                             // torch's type, set by bind_kv()
PyObject *s_dtype, *s_shape, *s_stride, *s_get_device, *s_data_ptr, *s_nbytes, *s_is_contiguous, *s_cuda_stream, *s_call;

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

// ---------------------------------------------------------------------------- key/value cache
// A tensor [tokens][heads][dim] with contiguous values; `rows` and `dim` (where >= 0), type and device as given.
struct Tensor3 {
  dq_heads_t h{};
  long long rows = 0, dim = 0, device = -1;
  int dtype = -1;
};
bool three(PyObject* tuple, long long (&v)[3]) {              // takes the reference
  if (!tuple) return false;
  bool ok = PyTuple_Check(tuple) && PyTuple_GET_SIZE(tuple) == 3;
  for (int i = 0; ok && i < 3; ++i) {
    v[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, i));
    ok = !PyErr_Occurred();
  }
  Py_DECREF(tuple);
  return ok;
}
bool tensor3(PyObject* t, const char* name, Tensor3& m, const Tensor3* like = nullptr) {
  PyObject* dtype = PyObject_GetAttr(t, s_dtype);
  if (!dtype) return false;
  for (int i = 0; i < 3; ++i) if (dtype == types[i]) m.dtype = i;
  Py_DECREF(dtype);
  if (!call_int(t, s_get_device, m.device)) return false;
  long long shape[3], step[3];
  const bool shaped = three(PyObject_GetAttr(t, s_shape), shape);
  if (PyErr_Occurred()) return false;
  if (!shaped || m.dtype < 0 || m.device < 0) {
    PyErr_Format(PyExc_ValueError, "%s: a CUDA tensor [tokens, heads, head_dim] of float32, bfloat16 or float16 is needed", name);
    return false;
  }
  m.rows = shape[0]; m.dim = shape[2];
  if (like && (m.rows != like->rows || m.dim != like->dim || m.dtype != like->dtype || m.device != like->device)) {
    PyErr_Format(PyExc_ValueError, "%s: tokens, head_dim, type or device differ from the first tensor's", name);
    return false;
  }
  if (!three(PyObject_CallMethodNoArgs(t, s_stride), step)) return false;
  if (m.dim > 1 && step[2] != 1) {
    PyErr_Format(PyExc_ValueError, "%s: the values of a head have to be contiguous", name);
    return false;
  }
  // (one token's stride means nothing, nor does one head's)
  if (shape[0] <= 1) step[0] = shape[1] <= 1 || step[1] < m.dim ? m.dim : step[1];
  if (shape[1] <= 1) step[1] = m.dim;
  if (step[0] < m.dim || step[1] < m.dim) {
    PyErr_Format(PyExc_ValueError, "%s: heads must not overlap", name);
    return false;
  }
  m.h.token_stride = step[0]; m.h.head_stride = step[1];
  m.h.heads = shape[1] > 0x7fffffff ? 0 : (int32_t)shape[1];
  return address(t, m.h.d_data);
}
bool optional3(PyObject* t, const char* name, Tensor3& m, const Tensor3& like) { return t == Py_None || tensor3(t, name, m, &like); }
bool same_heads(const char* name, const Tensor3& m, long long heads) {
  if (!m.h.d_data || m.h.heads == heads) return true;
  PyErr_Format(PyExc_ValueError, "%s: %lld heads are needed", name, heads);
  return false;
}

// The handle's (address of its dq_kv_cache_t, device, tensors): read once a call.
struct CacheRef { const dq_kv_cache_t* c = nullptr; long long device = -1; long long slots() const { return (long long)c->table_width * c->page_size; } };
bool cache_of(PyObject* o, CacheRef& r) {
  PyObject* call = PyObject_GetAttr(o, s_call);
  if (!call) return false;
  bool ok = PyTuple_Check(call) && PyTuple_GET_SIZE(call) == 2;
  if (ok) {
    r.c = (const dq_kv_cache_t*)PyLong_AsVoidPtr(PyTuple_GET_ITEM(call, 0));
    r.device = PyLong_AsLongLong(PyTuple_GET_ITEM(call, 1));
    ok = r.c && !PyErr_Occurred();
  }
  Py_DECREF(call);
  if (!ok && !PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "cache: a dq_kv_cache is needed");
  return ok;
}
bool on_cache(const char* name, const Tensor3& x, const CacheRef& r) {
  if (x.device == r.device && x.dim == r.c->head_dim) return true;
  PyErr_Format(PyExc_ValueError, "%s: the cache's device and head_dim %d are needed", name, (int)r.c->head_dim);
  return false;
}
// A contiguous array of 4-byte numbers, of exactly `count` (at least, where `more`); None gives null where allowed.
bool array4(PyObject* t, const char* name, PyObject* type, long long count, bool more, bool none, long long device, void*& p) {
  p = nullptr;
  if (none && t == Py_None) return true;
  PyObject* dtype = PyObject_GetAttr(t, s_dtype);
  if (!dtype) return false;
  const bool typed = dtype == type;
  Py_DECREF(dtype);
  long long held = 0;
  if (!bytes(t, name, count * 4, device, p, &held)) return false;
  if (!typed || (!more && held != count * 4)) {
    PyErr_Format(PyExc_ValueError, "%s: a %s tensor of %lld numbers is needed", name, type == types[DQ_FP32] ? "float32" : "int32", count);
    return false;
  }
  return true;
}
// [n_seqs][heads][slots]: the row length of it
bool slots_of(PyObject* t, const char* name, PyObject* type, const CacheRef& r, bool none, long long& ld, void*& p) {
  p = nullptr;
  if (none && t == Py_None) return true;
  long long shape[3];
  const bool shaped = three(PyObject_GetAttr(t, s_shape), shape);
  if (PyErr_Occurred()) return false;
  if (!shaped || shape[0] != r.c->n_seqs || shape[1] != r.c->heads || shape[2] < r.slots() || (ld >= 0 && shape[2] != ld)) {
    PyErr_Format(PyExc_ValueError, "%s: a [%d, %d, %lld] tensor is needed (all of one size, or more slots)", name, (int)r.c->n_seqs,
                 (int)r.c->heads, r.slots());
    return false;
  }
  ld = shape[2];
  return array4(t, name, type, shape[0] * shape[1] * shape[2], false, false, r.device, p);
}
bool starts_of(PyObject* t, const CacheRef& r, void*& p) { return array4(t, "starts", int32, (long long)r.c->n_seqs + 1, false, true, r.device, p); }
bool kv_count(Py_ssize_t n, Py_ssize_t want) {
  if (n == want && kv_entry.evict) return true;
  PyErr_SetString(PyExc_TypeError, "wrong number of arguments, or bind_kv() was not called");
  return false;
}
bool number(PyObject* o, double& v) {
  v = PyFloat_AsDouble(o);
  return v != -1.0 || !PyErr_Occurred();
}
bool integer(PyObject* o, const char* name, long long least, long long& v) {
  v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) return false;
  if (v >= least && v <= 0x7fffffff) return true;
  PyErr_Format(PyExc_ValueError, "%s: %lld is out of range", name, v);
  return false;
}

// qk_norm_rope(Q, K, positions, inv_freq, Q_out, K_out, q_gamma, k_gamma, eps, flags, stream)
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Tensor3 q, k, qo, ko;
  long long flags, rot = 0, held = 0;
  double eps;
  void *positions = nullptr, *freq = nullptr, *gamma[2] = {nullptr, nullptr}, *s;
  if (!kv_count(n, 11) || !tensor3(a[0], "Q", q) || !optional3(a[1], "K", k, q) || !tensor3(a[4], "Q_out", qo, &q) ||
      !optional3(a[5], "K_out", ko, q) || !number(a[8], eps) || !integer(a[9], "flags", 0, flags))
    return nullptr;
  if ((a[1] == Py_None) != (a[5] == Py_None)) { PyErr_SetString(PyExc_ValueError, "K and K_out: both or neither"); return nullptr; }
  if (!same_heads("Q_out", qo, q.h.heads) || (a[1] != Py_None && !same_heads("K_out", ko, k.h.heads))) return nullptr;
  if (a[3] != Py_None) {
    if (!bytes(a[3], "inv_freq", 0, q.device, freq, &held) || !array4(a[3], "inv_freq", types[DQ_FP32], held / 4, false, false, q.device, freq) ||
        !array4(a[2], "positions", int32, q.rows, false, false, q.device, positions))
      return nullptr;
    rot = held / 2;                                           // two values of a pair for each frequency
    if (rot > q.dim) { PyErr_Format(PyExc_ValueError, "inv_freq: at most %lld frequencies", q.dim / 2); return nullptr; }
  }
  int g_dtype = -1;
  for (int i = 0; i < 2; ++i) {
    PyObject* t = a[6 + i];
    if (t == Py_None) continue;
    PyObject* dtype = PyObject_GetAttr(t, s_dtype);
    if (!dtype) return nullptr;
    const int type = dtype == types[DQ_FP32] ? DQ_FP32 : dtype == types[q.dtype] ? q.dtype : -1;
    Py_DECREF(dtype);
    if (!bytes(t, "gamma", 0, q.device, gamma[i], &held)) return nullptr;
    if (type < 0 || held != q.dim * (type == DQ_FP32 ? 4 : 2) || (g_dtype >= 0 && g_dtype != type)) {
      PyErr_Format(PyExc_ValueError, "q_gamma, k_gamma: [%lld] tensors of one type, Q's or float32, are needed", q.dim);
      return nullptr;
    }
    g_dtype = type;
  }
  if (!stream_of(a[10], "dq_qk_norm_rope", q.device, s)) return nullptr;
  const bool with_k = a[1] != Py_None;
  DQ_CALL(kv_entry.qk_norm_rope(&q.h, with_k ? &k.h : nullptr, q.dtype, q.rows, (int32_t)(q.dim > 0x7fffffff ? 0 : q.dim), (const int32_t*)positions,
                                (const float*)freq, (int32_t)rot, gamma[0], gamma[1], g_dtype < 0 ? q.dtype : g_dtype, (float)eps,
                                (int32_t)flags, &qo.h, with_k ? &ko.h : nullptr, s));
}

// append(K, V, cache, starts, k_values, v_values, positions, slot_positions, stream)
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Tensor3 k, v, kv, vv;
  CacheRef r;
  long long ld = -1;
  void *starts, *positions, *slots, *s;
  if (!kv_count(n, 9) || !tensor3(a[0], "K", k) || !tensor3(a[1], "V", v, &k) || !cache_of(a[2], r) || !on_cache("K", k, r) ||
      !starts_of(a[3], r, starts) || !optional3(a[4], "k_values", kv, k) || !optional3(a[5], "v_values", vv, k) ||
      !array4(a[6], "positions", int32, k.rows, false, true, k.device, positions) ||
      !slots_of(a[7], "slot_positions", int32, r, true, ld, slots) || !same_heads("K", k, r.c->heads) || !same_heads("V", v, r.c->heads) ||
      !same_heads("k_values", kv, r.c->heads) || !same_heads("v_values", vv, r.c->heads) || !stream_of(a[8], "dq_kv_append", k.device, s))
    return nullptr;
  DQ_CALL(kv_entry.append(&k.h, &v.h, k.dtype, k.rows, r.c, (const int32_t*)starts, a[4] == Py_None ? nullptr : &kv.h,
                          a[5] == Py_None ? nullptr : &vv.h, (const int32_t*)positions, (int32_t*)slots, ld, s));
}

// kv_dequantize(cache, K, V, starts, stream)
PyObject* kv_dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Tensor3 k, v;
  CacheRef r;
  void *starts, *s;
  if (!kv_count(n, 5) || !cache_of(a[0], r) || !tensor3(a[1], "K", k) || !tensor3(a[2], "V", v, &k) || !on_cache("K", k, r) ||
      !starts_of(a[3], r, starts) || !same_heads("K", k, r.c->heads) || !same_heads("V", v, r.c->heads) ||
      !stream_of(a[4], "dq_kv_dequantize", k.device, s))
    return nullptr;
  DQ_CALL(kv_entry.dequantize(r.c, (const int32_t*)starts, k.rows, &k.h, &v.h, k.dtype, s));
}

// attention(Q, cache, scale, out, workspace, starts, lse, stream)
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Tensor3 q, o;
  CacheRef r;
  double scale;
  void *work, *starts, *lse, *s;
  if (!kv_count(n, 8) || !tensor3(a[0], "Q", q) || !cache_of(a[1], r) || !on_cache("Q", q, r) || !number(a[2], scale) ||
      !tensor3(a[3], "out", o, &q) || !same_heads("out", o, q.h.heads) ||
      !bytes(a[4], "workspace", kv_entry.attention_workspace(r.c->head_dim), q.device, work) || !starts_of(a[5], r, starts) ||
      !array4(a[6], "lse", types[DQ_FP32], q.rows * q.h.heads, false, true, q.device, lse) || !stream_of(a[7], "dq_kv_attention", q.device, s))
    return nullptr;
  DQ_CALL(kv_entry.attention(&q.h, q.dtype, q.rows, r.c, (const int32_t*)starts, (float)scale, &o.h, (float*)lse, work, s));
}

// attention_weights(Q, lse, cache, scale, weights_out, weights, starts, stream)
PyObject* attention_weights(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Tensor3 q;
  CacheRef r;
  long long ld = -1;
  double scale;
  void *lse, *out, *weights, *starts, *s;
  if (!kv_count(n, 8) || !tensor3(a[0], "Q", q) || !cache_of(a[2], r) || !on_cache("Q", q, r) || !number(a[3], scale) ||
      !array4(a[1], "lse", types[DQ_FP32], q.rows * q.h.heads, false, false, q.device, lse) ||
      !slots_of(a[4], "weights_out", types[DQ_FP32], r, false, ld, out) || !slots_of(a[5], "weights", types[DQ_FP32], r, true, ld, weights) ||
      !starts_of(a[6], r, starts) || !stream_of(a[7], "dq_kv_attention_weights", q.device, s))
    return nullptr;
  DQ_CALL(kv_entry.attention_weights(&q.h, q.dtype, q.rows, (const float*)lse, r.c, (const int32_t*)starts, (float)scale, (const float*)weights,
                                     (float*)out, ld, s));
}

// evict(cache, weights, positions, keep, recent, weights_out, positions_out, lengths_out, workspace, stream)
PyObject* evict(PyObject*, PyObject* const* a, Py_ssize_t n) {
  CacheRef r;
  long long ld = -1, keep, recent;
  void *weights, *positions, *w_out, *p_out, *lengths, *work, *s;
  if (!kv_count(n, 10) || !cache_of(a[0], r) || !slots_of(a[1], "weights", types[DQ_FP32], r, false, ld, weights) ||
      !slots_of(a[2], "positions", int32, r, false, ld, positions) || !integer(a[3], "keep", 1, keep) || !integer(a[4], "recent", 0, recent) ||
      !slots_of(a[5], "weights_out", types[DQ_FP32], r, false, ld, w_out) || !slots_of(a[6], "positions_out", int32, r, false, ld, p_out) ||
      !array4(a[7], "lengths_out", int32, r.c->n_seqs, false, false, r.device, lengths) ||
      !bytes(a[8], "workspace", kv_entry.evict_workspace(r.c->n_seqs, r.c->heads, (int32_t)keep), r.device, work) ||
      !stream_of(a[9], "dq_kv_evict", r.device, s))
    return nullptr;
  DQ_CALL(kv_entry.evict(r.c, (const float*)weights, (const int32_t*)positions, ld, (int32_t)keep, (int32_t)recent, (float*)w_out,
                         (int32_t*)p_out, (int32_t*)lengths, work, s));
}

// bind_kv((eight entry addresses in the order of kv_entry), int32)
PyObject* bind_kv(PyObject*, PyObject* args) {
  PyObject *at, *type;
  if (!PyArg_ParseTuple(args, "O!O", &PyTuple_Type, &at, &type)) return nullptr;
  if (PyTuple_GET_SIZE(at) != 8) { PyErr_SetString(PyExc_TypeError, "bind_kv: eight entries"); return nullptr; }
  void* p[8];
  for (int i = 0; i < 8; ++i) {
    p[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(at, i));
    if (!p[i]) { if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind_kv: a null entry"); return nullptr; }
  }
  Py_INCREF(type); Py_XSETREF(int32, type);
  kv_entry.qk_norm_rope = (decltype(kv_entry.qk_norm_rope))p[0];
  kv_entry.append = (decltype(kv_entry.append))p[1];
  kv_entry.dequantize = (decltype(kv_entry.dequantize))p[2];
  kv_entry.attention = (decltype(kv_entry.attention))p[3];
  kv_entry.attention_weights = (decltype(kv_entry.attention_weights))p[4];
  kv_entry.evict = (decltype(kv_entry.evict))p[5];
  kv_entry.attention_workspace = (decltype(kv_entry.attention_workspace))p[6];
  kv_entry.evict_workspace = (decltype(kv_entry.evict_workspace))p[7];
  Py_RETURN_NONE;
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
                         DQ_FAST(qk_norm_rope), DQ_FAST(append), DQ_FAST(kv_dequantize), DQ_FAST(attention), DQ_FAST(attention_weights),
                         DQ_FAST(evict), {"bind_kv", bind_kv, METH_VARARGS, nullptr},
                         {"bind", bind, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", "Checked calls of the microscaled and key/value cache operators.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void) {
  const struct { PyObject** to; const char* name; } names[] = {
      {&s_dtype, "dtype"}, {&s_shape, "shape"}, {&s_stride, "stride"}, {&s_get_device, "get_device"}, {&s_data_ptr, "data_ptr"},
      {&s_nbytes, "nbytes"}, {&s_is_contiguous, "is_contiguous"}, {&s_cuda_stream, "cuda_stream"},
      {&s_call, "_call"}};
  for (const auto& n : names)
    if (!(*n.to = PyUnicode_InternFromString(n.name))) return nullptr;
  return PyModule_Create(&module);
}
