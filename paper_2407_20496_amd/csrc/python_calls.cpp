// Python calls of the per-product and per-layer entry points of libhinm (include/hinm.h): argument marshalling only.
//
// A decode-sized product runs 4 .. 10 us on the GPU, and building the shape structure, converting seventeen arguments
// and asking for the current stream in interpreted code took 6 .. 7 us of the calling thread: calls in a row were bound by that.
// Here a call costs about a microsecond besides the launch itself.  binding.py hands over the addresses of the entry
// points of the library it has loaded, so this module links to nothing; the interpreter lock is released around
// every library call.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <vector>

#include "hinm.h"

namespace {

decltype(&hinm_pack) f_pack;
decltype(&hinm_prepare) f_prepare;
decltype(&hinm_spmm) f_spmm;
decltype(&hinm_spmm_vectors) f_spmm_vectors;
decltype(&hinm_spmm_prepared) f_spmm_prepared;
decltype(&hinm_chain) f_chain;
decltype(&hinm_mx4_quantize) f_mx4_quantize;
decltype(&hinm_mx4_unpack) f_mx4_unpack;
decltype(&hinm_mx4_product) f_mx4_product;
decltype(&hinm_mx4_linear) f_mx4_linear;
decltype(&hinm_block_norm) f_block_norm;
decltype(&hinm_block_norm_grad) f_block_norm_grad;
decltype(&hinm_linear) f_linear;
decltype(&hinm_linear_grad) f_linear_grad;
decltype(&hinm_layer_norm) f_layer_norm;
decltype(&hinm_layer_norm_grad) f_layer_norm_grad;

PyObject* g_dtype_code;      // any accepted dtype -> HINM_F16 / HINM_BF16
PyObject* g_current_stream;  // () -> raw pointer of the current stream or None; used until a source is set
PyObject* g_get_device;      // () -> current device, and
PyObject* g_raw_stream;      // (device) -> raw pointer of its current stream
PyObject* s_data_ptr;
PyObject* s_cuda_stream;
PyObject* s_f16;
PyObject* s_bf16;
PyObject* s_layer[12];

// The low 64 bits, as ctypes converts integers: sizes use all of them (2**64 - 1 for "any").
bool to_i64(PyObject* o, int64_t* out) {
  if (PyLong_Check(o)) {
    *out = (int64_t)PyLong_AsUnsignedLongLongMask(o);
  } else {
    PyObject* n = PyNumber_Long(o);
    if (!n) return false;
    *out = (int64_t)PyLong_AsUnsignedLongLongMask(n);
    Py_DECREF(n);
  }
  return !(*out == -1 && PyErr_Occurred());
}

// None -> NULL, an integer is the address, anything else has data_ptr()
bool to_ptr(PyObject* o, void** out) {
  if (o == Py_None) {
    *out = nullptr;
    return true;
  }
  PyObject* n = nullptr;
  if (!PyLong_Check(o)) {
    n = PyObject_CallMethodNoArgs(o, s_data_ptr);
    if (!n) return false;
    o = n;
  }
  *out = PyLong_AsVoidPtr(o);
  Py_XDECREF(n);
  return !(*out == nullptr && PyErr_Occurred());
}

bool to_float(PyObject* o, float* out) {
  const double v = PyFloat_AsDouble(o);
  *out = (float)v;
  return !(v == -1.0 && PyErr_Occurred());
}

// n pointers / n sizes in a row
bool to_ptrs(PyObject* const* a, int n, void** out) {
  for (int i = 0; i < n; ++i)
    if (!to_ptr(a[i], &out[i])) return false;
  return true;
}
// The nearest value that fits: what 32 bits do not hold, the library refuses as out of range, and must not see as what is
// left of it.
bool to_nearest(PyObject* o, int64_t low, int64_t high, int64_t* out) {
  PyObject* n = PyNumber_Long(o);
  if (!n) return false;
  int beyond;
  const long long v = PyLong_AsLongLongAndOverflow(n, &beyond);
  Py_DECREF(n);
  if (v == -1 && PyErr_Occurred()) return false;
  *out = beyond > 0 || v > high ? high : beyond < 0 || v < low ? low : (int64_t)v;
  return true;
}
bool to_sizes(PyObject* const* a, int n, int32_t* out) {
  for (int i = 0; i < n; ++i) {
    int64_t v;
    if (!to_nearest(a[i], INT32_MIN, INT32_MAX, &v)) return false;
    out[i] = (int32_t)v;
  }
  return true;
}
bool to_flags(PyObject* o, uint32_t* out) {
  int64_t v;
  if (!to_nearest(o, -1, UINT32_MAX, &v)) return false;
  *out = (uint32_t)v;
  return true;
}

bool to_stream(PyObject* o, void** out) {
  if (o != Py_None && !PyLong_Check(o)) {
    PyObject* n = PyObject_GetAttr(o, s_cuda_stream);
    if (!n) return false;
    const bool ok = to_ptr(n, out);
    Py_DECREF(n);
    return ok;
  }
  if (o != Py_None) return to_ptr(o, out);
  PyObject* raw;
  if (g_raw_stream) {
    PyObject* device = PyObject_CallNoArgs(g_get_device);
    if (!device) return false;
    raw = PyObject_CallOneArg(g_raw_stream, device);
    Py_DECREF(device);
  } else {
    raw = PyObject_CallOneArg(g_current_stream, Py_None);
  }
  if (!raw) return false;
  const bool ok = to_ptr(raw, out);
  Py_DECREF(raw);
  return ok;
}

bool to_dtype(PyObject* o, int32_t* out) {
  if (o == s_f16) {
    *out = HINM_F16;
    return true;
  }
  if (o == s_bf16) {
    *out = HINM_BF16;
    return true;
  }
  PyObject* code = PyObject_CallOneArg(g_dtype_code, o);
  if (!code) return false;
  int64_t v;
  const bool ok = to_i64(code, &v);
  Py_DECREF(code);
  *out = (int32_t)v;
  return ok;
}

// M, K, V, Kv, dtype
bool to_shape(PyObject* const* a, hinm_shape* s) {
  int64_t m, k, v, kv;
  if (!to_i64(a[0], &m) || !to_i64(a[1], &k) || !to_i64(a[2], &v) || !to_i64(a[3], &kv) || !to_dtype(a[4], &s->dtype))
    return false;
  s->M = (int32_t)m;
  s->K = (int32_t)k;
  s->V = (int32_t)v;
  s->Kv = (int32_t)kv;
  return true;
}

bool takes(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_Format(PyExc_TypeError, "%zd arguments where %zd are wanted", n, want);
  return false;
}

template <class Call>
PyObject* status_of(Call call) {
  hinm_status st;
  Py_BEGIN_ALLOW_THREADS
  st = call();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong((long)st);
}

// (M, K, V, Kv, dtype, W, vals, nm_idx, vec_idx, workspace, workspace_bytes, stream)
PyObject* pack(PyObject*, PyObject* const* a, Py_ssize_t n) {
  hinm_shape s;
  void* p[5];
  void* stream;
  int64_t bytes;
  if (!takes(n, 12) || !to_shape(a, &s)) return nullptr;
  for (int i = 0; i < 5; ++i)
    if (!to_ptr(a[5 + i], &p[i])) return nullptr;
  if (!to_i64(a[10], &bytes) || !to_stream(a[11], &stream)) return nullptr;
  return status_of([&] {
    return f_pack(&s, p[0], p[1], static_cast<uint8_t*>(p[2]), static_cast<int32_t*>(p[3]), p[4], (size_t)bytes, stream);
  });
}

// (M, K, V, Kv, dtype, vals, nm_idx, vec_idx, pi_in, pi_out, prepared, prepared_bytes, stream)
PyObject* prepare(PyObject*, PyObject* const* a, Py_ssize_t n) {
  hinm_shape s;
  void* p[6];
  void* stream;
  int64_t bytes;
  if (!takes(n, 13) || !to_shape(a, &s)) return nullptr;
  for (int i = 0; i < 6; ++i)
    if (!to_ptr(a[5 + i], &p[i])) return nullptr;
  if (!to_i64(a[11], &bytes) || !to_stream(a[12], &stream)) return nullptr;
  return status_of([&] {
    return f_prepare(&s, p[0], static_cast<uint8_t*>(p[1]), static_cast<int32_t*>(p[2]), static_cast<int32_t*>(p[3]),
                     static_cast<int32_t*>(p[4]), p[5], (size_t)bytes, stream);
  });
}

// (M, K, V, Kv, dtype, N, vals, nm_idx, vec_idx, pi_in, pi_out, X, ldx, Y, ldy, flags, workspace, workspace_bytes, stream)
PyObject* spmm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  hinm_shape s;
  void *p[6], *y, *ws, *stream;
  int64_t cols, ldx, ldy, flags, bytes;
  if (!takes(n, 19) || !to_shape(a, &s) || !to_i64(a[5], &cols)) return nullptr;
  for (int i = 0; i < 6; ++i)
    if (!to_ptr(a[6 + i], &p[i])) return nullptr;
  if (!to_i64(a[12], &ldx) || !to_ptr(a[13], &y) || !to_i64(a[14], &ldy) || !to_i64(a[15], &flags) || !to_ptr(a[16], &ws) ||
      !to_i64(a[17], &bytes) || !to_stream(a[18], &stream))
    return nullptr;
  return status_of([&] {
    return f_spmm(&s, (int32_t)cols, p[0], static_cast<uint8_t*>(p[1]), static_cast<int32_t*>(p[2]),
                  static_cast<int32_t*>(p[3]), static_cast<int32_t*>(p[4]), p[5], ldx, y, ldy, (uint32_t)flags, ws,
                  (size_t)bytes, stream);
  });
}

// (M, K, V, Kv, dtype, N, vals_v, vec_idx, pi_in, pi_out, X, ldx, Y, ldy, flags, stream)
PyObject* spmm_vectors(PyObject*, PyObject* const* a, Py_ssize_t n) {
  hinm_shape s;
  void *p[5], *y, *stream;
  int64_t cols, ldx, ldy, flags;
  if (!takes(n, 16) || !to_shape(a, &s) || !to_i64(a[5], &cols)) return nullptr;
  for (int i = 0; i < 5; ++i)
    if (!to_ptr(a[6 + i], &p[i])) return nullptr;
  if (!to_i64(a[11], &ldx) || !to_ptr(a[12], &y) || !to_i64(a[13], &ldy) || !to_i64(a[14], &flags) ||
      !to_stream(a[15], &stream))
    return nullptr;
  return status_of([&] {
    return f_spmm_vectors(&s, (int32_t)cols, p[0], static_cast<int32_t*>(p[1]), static_cast<int32_t*>(p[2]),
                          static_cast<int32_t*>(p[3]), p[4], ldx, y, ldy, (uint32_t)flags, stream);
  });
}

// (M, K, V, Kv, dtype, N, prepared, X, ldx, Y, ldy, flags, workspace, workspace_bytes, stream)
PyObject* spmm_prepared(PyObject*, PyObject* const* a, Py_ssize_t n) {
  hinm_shape s;
  void *prepared, *x, *y, *ws, *stream;
  int64_t cols, ldx, ldy, flags, bytes;
  if (!takes(n, 15) || !to_shape(a, &s) || !to_i64(a[5], &cols) || !to_ptr(a[6], &prepared) || !to_ptr(a[7], &x) ||
      !to_i64(a[8], &ldx) || !to_ptr(a[9], &y) || !to_i64(a[10], &ldy) || !to_i64(a[11], &flags) || !to_ptr(a[12], &ws) ||
      !to_i64(a[13], &bytes) || !to_stream(a[14], &stream))
    return nullptr;
  return status_of([&] {
    return f_spmm_prepared(&s, (int32_t)cols, prepared, x, ldx, y, ldy, (uint32_t)flags, ws, (size_t)bytes, stream);
  });
}

// one attribute of a layer, converted
template <class Convert, class T>
bool field(PyObject* layer, int which, Convert convert, T* out) {
  PyObject* o = PyObject_GetAttr(layer, s_layer[which]);
  if (!o) return false;
  const bool ok = convert(o, out);
  Py_DECREF(o);
  return ok;
}

// (layers, N, X, ldx, Y, ldy, scratch, scratch_bytes, stream)
PyObject* chain(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!takes(n, 9)) return nullptr;
  if (PyObject_Size(a[0]) < 0) return nullptr;  // an iterator that is used up by one pass is no sequence of layers
  PyObject* seq = PySequence_Fast(a[0], "layers must be a sequence");
  if (!seq) return nullptr;
  const Py_ssize_t count = PySequence_Fast_GET_SIZE(seq);
  std::vector<hinm_layer> layers;
  layers.reserve((size_t)count + 1);  // an address also for a chain of no layers, which is an error of shape
  layers.resize((size_t)count);
  bool ok = true;
  for (Py_ssize_t i = 0; i < count && ok; ++i) {
    PyObject* l = PySequence_Fast_GET_ITEM(seq, i);
    hinm_layer& d = layers[(size_t)i];
    int64_t v[4], flags = 0;
    void *vals, *nm, *vec, *pin, *pout, *prep;
    for (int q = 0; q < 4 && ok; ++q) ok = field(l, q, to_i64, &v[q]);
    ok = ok && field(l, 4, to_dtype, &d.shape.dtype) && field(l, 5, to_ptr, &vals) && field(l, 6, to_ptr, &nm) &&
         field(l, 7, to_ptr, &vec) && field(l, 8, to_ptr, &pin) && field(l, 9, to_ptr, &pout) &&
         field(l, 10, to_i64, &flags) && field(l, 11, to_ptr, &prep);
    if (!ok) break;
    d.shape.M = (int32_t)v[0];
    d.shape.K = (int32_t)v[1];
    d.shape.V = (int32_t)v[2];
    d.shape.Kv = (int32_t)v[3];
    d.vals = vals;
    d.nm_idx = static_cast<uint8_t*>(nm);
    d.vec_idx = static_cast<int32_t*>(vec);
    d.pi_in = static_cast<int32_t*>(pin);
    d.pi_out = static_cast<int32_t*>(pout);
    d.flags = (uint32_t)flags;
    d.prepared = prep;
  }
  Py_DECREF(seq);
  void *x, *y, *scratch, *stream;
  int64_t cols, ldx, ldy, bytes;
  if (!ok || !to_i64(a[1], &cols) || !to_ptr(a[2], &x) || !to_i64(a[3], &ldx) || !to_ptr(a[4], &y) || !to_i64(a[5], &ldy) ||
      !to_ptr(a[6], &scratch) || !to_i64(a[7], &bytes) || !to_stream(a[8], &stream))
    return nullptr;
  return status_of([&] {
    return f_chain((int32_t)count, layers.data(), (int32_t)cols, x, ldx, y, ldy, scratch, (size_t)bytes, stream);
  });
}

// (rows, cols, dtype, src, ld, along, codes, scales, stream)
PyObject* mx4_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  int32_t d[2], dtype, along;
  void *src, *form[2], *stream;
  int64_t ld;
  if (!takes(n, 9) || !to_sizes(a, 2, d) || !to_dtype(a[2], &dtype) || !to_ptr(a[3], &src) || !to_i64(a[4], &ld) ||
      !to_sizes(a + 5, 1, &along) || !to_ptrs(a + 6, 2, form) || !to_stream(a[8], &stream))
    return nullptr;
  return status_of([&] {
    return f_mx4_quantize(d[0], d[1], dtype, src, ld, along, static_cast<uint8_t*>(form[0]), static_cast<uint8_t*>(form[1]),
                          stream);
  });
}

// (rows, length, dtype, codes, scales, dst, ld, stream)
PyObject* mx4_unpack(PyObject*, PyObject* const* a, Py_ssize_t n) {
  int32_t d[2], dtype;
  void *p[3], *stream;
  int64_t ld;
  if (!takes(n, 8) || !to_sizes(a, 2, d) || !to_dtype(a[2], &dtype) || !to_ptrs(a + 3, 3, p) || !to_i64(a[6], &ld) ||
      !to_stream(a[7], &stream))
    return nullptr;
  return status_of([&] {
    return f_mx4_unpack(d[0], d[1], dtype, static_cast<uint8_t*>(p[0]), static_cast<uint8_t*>(p[1]), p[2], ld, stream);
  });
}

// (M, N, K, dtype, a_codes, a_scales, b_codes, b_scales, Y, ldy, flags, stream)
PyObject* mx4_product(PyObject*, PyObject* const* a, Py_ssize_t n) {
  int32_t d[3], dtype;
  void *p[5], *stream;
  int64_t ldy;
  uint32_t flags;
  if (!takes(n, 12) || !to_sizes(a, 3, d) || !to_dtype(a[3], &dtype) || !to_ptrs(a + 4, 5, p) || !to_i64(a[9], &ldy) ||
      !to_flags(a[10], &flags) || !to_stream(a[11], &stream))
    return nullptr;
  return status_of([&] {
    return f_mx4_product(d[0], d[1], d[2], dtype, static_cast<uint8_t*>(p[0]), static_cast<uint8_t*>(p[1]),
                         static_cast<uint8_t*>(p[2]), static_cast<uint8_t*>(p[3]), p[4], ldy, flags, stream);
  });
}

// (M, K, N, dtype, codes, scales, X, ldx, Y, ldy, flags, workspace, workspace_bytes, stream)
PyObject* mx4_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  int32_t d[3], dtype;
  void *form[2], *x, *y, *ws, *stream;
  int64_t ldx, ldy, bytes;
  uint32_t flags;
  if (!takes(n, 14) || !to_sizes(a, 3, d) || !to_dtype(a[3], &dtype) || !to_ptrs(a + 4, 2, form) || !to_ptr(a[6], &x) ||
      !to_i64(a[7], &ldx) || !to_ptr(a[8], &y) || !to_i64(a[9], &ldy) || !to_flags(a[10], &flags) || !to_ptr(a[11], &ws) ||
      !to_i64(a[12], &bytes) || !to_stream(a[13], &stream))
    return nullptr;
  return status_of([&] {
    return f_mx4_linear(d[0], d[1], d[2], dtype, static_cast<uint8_t*>(form[0]), static_cast<uint8_t*>(form[1]), x, ldx, y, ldy,
                        flags, ws, (size_t)bytes, stream);
  });
}

// (K, N, dtype, residual_scale, eps, x, y, w_post, gate, token_gate, w_pre, h, ld_stream, u, ld_block, rstd_y, rstd_h, workspace,
//  workspace_bytes, stream)
PyObject* block_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  int32_t d[2], dtype;
  float scale, eps;
  void *in[6], *h, *u, *out[2], *ws, *stream;
  int64_t ld_stream, ld_block, bytes;
  if (!takes(n, 20) || !to_sizes(a, 2, d) || !to_dtype(a[2], &dtype) || !to_float(a[3], &scale) || !to_float(a[4], &eps) ||
      !to_ptrs(a + 5, 6, in) || !to_ptr(a[11], &h) || !to_i64(a[12], &ld_stream) || !to_ptr(a[13], &u) ||
      !to_i64(a[14], &ld_block) || !to_ptrs(a + 15, 2, out) || !to_ptr(a[17], &ws) || !to_i64(a[18], &bytes) ||
      !to_stream(a[19], &stream))
    return nullptr;
  return status_of([&] {
    return f_block_norm(d[0], d[1], dtype, scale, eps, in[0], in[1], static_cast<float*>(in[2]), static_cast<float*>(in[3]),
                        static_cast<float*>(in[4]), static_cast<float*>(in[5]), h, ld_stream, u, ld_block,
                        static_cast<float*>(out[0]), static_cast<float*>(out[1]), ws, (size_t)bytes, stream);
  });
}

// (K, N, dtype, residual_scale, h, y, w_post, gate, token_gate, w_pre, rstd_y, rstd_h, dh, du, dx, ld_stream, dy, ld_block, dw_post,
//  dgate, dtoken_gate, dw_pre, workspace, workspace_bytes, stream)
PyObject* block_norm_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  int32_t d[2], dtype;
  float scale;
  void *in[10], *dx, *dy, *out[4], *ws, *stream;
  int64_t ld_stream, ld_block, bytes;
  if (!takes(n, 25) || !to_sizes(a, 2, d) || !to_dtype(a[2], &dtype) || !to_float(a[3], &scale) || !to_ptrs(a + 4, 10, in) ||
      !to_ptr(a[14], &dx) || !to_i64(a[15], &ld_stream) || !to_ptr(a[16], &dy) || !to_i64(a[17], &ld_block) ||
      !to_ptrs(a + 18, 4, out) || !to_ptr(a[22], &ws) || !to_i64(a[23], &bytes) || !to_stream(a[24], &stream))
    return nullptr;
  return status_of([&] {
    auto f = [&](int i) { return static_cast<float*>(in[i]); };
    auto g = [&](int i) { return static_cast<float*>(out[i]); };
    return f_block_norm_grad(d[0], d[1], dtype, scale, in[0], in[1], f(2), f(3), f(4), f(5), f(6), f(7), in[8], in[9], dx,
                             ld_stream, dy, ld_block, g(0), g(1), g(2), g(3), ws, (size_t)bytes, stream);
  });
}

// (M, K, N, dtype, W, ldw, X, ldx, bias, residual, ldr, Z, Y, ldy, flags, workspace, workspace_bytes, stream)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  int32_t d[3], dtype;
  void *w, *x, *in[2], *out[2], *ws, *stream;
  int64_t ldw, ldx, ldr, ldy, bytes;
  uint32_t flags;
  if (!takes(n, 18) || !to_sizes(a, 3, d) || !to_dtype(a[3], &dtype) || !to_ptr(a[4], &w) || !to_i64(a[5], &ldw) || !to_ptr(a[6], &x) ||
      !to_i64(a[7], &ldx) || !to_ptrs(a + 8, 2, in) || !to_i64(a[10], &ldr) || !to_ptrs(a + 11, 2, out) || !to_i64(a[13], &ldy) ||
      !to_flags(a[14], &flags) || !to_ptr(a[15], &ws) || !to_i64(a[16], &bytes) || !to_stream(a[17], &stream))
    return nullptr;
  return status_of([&] {
    return f_linear(d[0], d[1], d[2], dtype, w, ldw, x, ldx, static_cast<float*>(in[0]), in[1], ldr, out[0], out[1], ldy, flags, ws,
                    (size_t)bytes, stream);
  });
}

// (M, K, N, dtype, W, ldw, X, ldx, Z, dY, ldy, dX, dW, dbias, flags, workspace, workspace_bytes, stream)
PyObject* linear_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  int32_t d[3], dtype;
  void *w, *x, *in[2], *out[3], *ws, *stream;
  int64_t ldw, ldx, ldy, bytes;
  uint32_t flags;
  if (!takes(n, 18) || !to_sizes(a, 3, d) || !to_dtype(a[3], &dtype) || !to_ptr(a[4], &w) || !to_i64(a[5], &ldw) || !to_ptr(a[6], &x) ||
      !to_i64(a[7], &ldx) || !to_ptrs(a + 8, 2, in) || !to_i64(a[10], &ldy) || !to_ptrs(a + 11, 3, out) || !to_flags(a[14], &flags) ||
      !to_ptr(a[15], &ws) || !to_i64(a[16], &bytes) || !to_stream(a[17], &stream))
    return nullptr;
  return status_of([&] {
    return f_linear_grad(d[0], d[1], d[2], dtype, w, ldw, x, ldx, in[0], in[1], ldy, out[0], out[1], static_cast<float*>(out[2]), flags, ws,
                         (size_t)bytes, stream);
  });
}

// (K, N, dtype, eps, x, ldx, w, b, u, ldu, mean, rstd, workspace, workspace_bytes, stream)
PyObject* layer_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  int32_t d[2], dtype;
  float eps;
  void *x, *in[2], *u, *out[2], *ws, *stream;
  int64_t ldx, ldu, bytes;
  if (!takes(n, 15) || !to_sizes(a, 2, d) || !to_dtype(a[2], &dtype) || !to_float(a[3], &eps) || !to_ptr(a[4], &x) || !to_i64(a[5], &ldx) ||
      !to_ptrs(a + 6, 2, in) || !to_ptr(a[8], &u) || !to_i64(a[9], &ldu) || !to_ptrs(a + 10, 2, out) || !to_ptr(a[12], &ws) ||
      !to_i64(a[13], &bytes) || !to_stream(a[14], &stream))
    return nullptr;
  return status_of([&] {
    return f_layer_norm(d[0], d[1], dtype, eps, x, ldx, static_cast<float*>(in[0]), static_cast<float*>(in[1]), u, ldu,
                        static_cast<float*>(out[0]), static_cast<float*>(out[1]), ws, (size_t)bytes, stream);
  });
}

// (K, N, dtype, x, ldx, w, mean, rstd, du, ldu, dh, dx, dw, db, workspace, workspace_bytes, stream)
PyObject* layer_norm_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  int32_t d[2], dtype;
  void *x, *in[4], *out[4], *ws, *stream;
  int64_t ldx, ldu, bytes;
  if (!takes(n, 17) || !to_sizes(a, 2, d) || !to_dtype(a[2], &dtype) || !to_ptr(a[3], &x) || !to_i64(a[4], &ldx) || !to_ptrs(a + 5, 4, in) ||
      !to_i64(a[9], &ldu) || !to_ptrs(a + 10, 4, out) || !to_ptr(a[14], &ws) || !to_i64(a[15], &bytes) || !to_stream(a[16], &stream))
    return nullptr;
  return status_of([&] {
    auto f = [](void* p) { return static_cast<float*>(p); };
    return f_layer_norm_grad(d[0], d[1], dtype, x, ldx, f(in[0]), f(in[1]), f(in[2]), in[3], ldu, out[0], out[1], f(out[2]), f(out[3]), ws,
                             (size_t)bytes, stream);
  });
}

// (addresses in the order below, dtype_code, current_stream)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  constexpr int kEntries = 16;
  void* f[kEntries];
  if (!takes(n, kEntries + 2) || !to_ptrs(a, kEntries, f)) return nullptr;
  f_pack = reinterpret_cast<decltype(f_pack)>(f[0]);
  f_prepare = reinterpret_cast<decltype(f_prepare)>(f[1]);
  f_spmm = reinterpret_cast<decltype(f_spmm)>(f[2]);
  f_spmm_vectors = reinterpret_cast<decltype(f_spmm_vectors)>(f[3]);
  f_spmm_prepared = reinterpret_cast<decltype(f_spmm_prepared)>(f[4]);
  f_chain = reinterpret_cast<decltype(f_chain)>(f[5]);
  f_mx4_quantize = reinterpret_cast<decltype(f_mx4_quantize)>(f[6]);
  f_mx4_unpack = reinterpret_cast<decltype(f_mx4_unpack)>(f[7]);
  f_mx4_product = reinterpret_cast<decltype(f_mx4_product)>(f[8]);
  f_mx4_linear = reinterpret_cast<decltype(f_mx4_linear)>(f[9]);
  f_block_norm = reinterpret_cast<decltype(f_block_norm)>(f[10]);
  f_block_norm_grad = reinterpret_cast<decltype(f_block_norm_grad)>(f[11]);
  f_linear = reinterpret_cast<decltype(f_linear)>(f[12]);
  f_linear_grad = reinterpret_cast<decltype(f_linear_grad)>(f[13]);
  f_layer_norm = reinterpret_cast<decltype(f_layer_norm)>(f[14]);
  f_layer_norm_grad = reinterpret_cast<decltype(f_layer_norm_grad)>(f[15]);
  Py_INCREF(a[kEntries]);
  Py_XSETREF(g_dtype_code, a[kEntries]);
  Py_INCREF(a[kEntries + 1]);
  Py_XSETREF(g_current_stream, a[kEntries + 1]);
  Py_RETURN_NONE;
}

// (get_device, raw_stream): from now on the current stream is asked for directly
PyObject* set_stream_source(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!takes(n, 2)) return nullptr;
  Py_INCREF(a[0]);
  Py_XSETREF(g_get_device, a[0]);
  Py_INCREF(a[1]);
  Py_XSETREF(g_raw_stream, a[1]);
  Py_RETURN_NONE;
}

#define HINM_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {HINM_METHOD(pack),    HINM_METHOD(prepare), HINM_METHOD(spmm), HINM_METHOD(spmm_vectors),
                         HINM_METHOD(spmm_prepared), HINM_METHOD(chain), HINM_METHOD(mx4_quantize),
                         HINM_METHOD(mx4_unpack), HINM_METHOD(mx4_product), HINM_METHOD(mx4_linear), HINM_METHOD(block_norm),
                         HINM_METHOD(block_norm_grad), HINM_METHOD(linear), HINM_METHOD(linear_grad), HINM_METHOD(layer_norm),
                         HINM_METHOD(layer_norm_grad), HINM_METHOD(bind), HINM_METHOD(set_stream_source),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  s_f16 = PyUnicode_InternFromString("f16");
  s_bf16 = PyUnicode_InternFromString("bf16");
  const char* names[12] = {"M", "K", "V", "Kv", "dtype", "vals", "nm_idx", "vec_idx", "pi_in", "pi_out", "flags", "prepared"};
  for (int i = 0; i < 12; ++i) s_layer[i] = PyUnicode_InternFromString(names[i]);
  return PyModule_Create(&module);
}
