// The entry points that a program calls once per layer and pass, as native functions: a call of a few microseconds spent more
// than a third of its host time marshalling its arguments in Python (hbmm_quantize of a 1 x 4096 row: 5.0 us, of which the
// library, its checks and the launch included, takes 3.2).  Names, arguments, defaults, checks and errors are those of the
// Python functions they stand for; the C functions of libhbmm.so are handed over as addresses when hbmm.py is imported, and
// run without the interpreter lock, as ctypes runs them.
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/Exceptions.h>
#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include "hbmm.h"

namespace {

decltype(&hbmm_quantize) f_quantize;
decltype(&hbmm_gemm) f_gemm;
decltype(&hbmm_gemm_ex) f_gemm_ex;
decltype(&hbmm_conv_im2col_ex) f_conv;
decltype(&hbmm_conv_im2col_fused) f_conv_fused;
decltype(&hbmm_binarize_dense) f_dense;
decltype(&hbmm_binarize_backward) f_backward;
decltype(&hbmm_fp8_quantize) f_fp8_quantize;
decltype(&hbmm_fp8_gemm) f_fp8_gemm;
decltype(&hbmm_fp8_input_grad) f_fp8_input_grad;
decltype(&hbmm_fp8_weight_grad) f_fp8_weight_grad;
decltype(&hbmm_fp8_binarize_backward) f_fp8_backward;
PyObject* g_error;                 // HbmmError
PyTypeObject* t_fp8;               // Fp8Operand
PyTypeObject *t_operand, *t_geom, *t_epilogue;      // the ctypes structures that stand for hbmm_operand, hbmm_conv_geom, hbmm_epilogue
PyObject *s_desc, *s_cuda_stream, *s_codes, *s_scales, *s_K, *s_block_rows;

// Arguments of a METH_FASTCALL | METH_KEYWORDS call in the order of `names`; absent ones stay null.
bool take(const char* what, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames, const char* const* names, int n, int required, PyObject** out) {
  if (nargs > n) {
    PyErr_Format(PyExc_TypeError, "%s() takes at most %d positional arguments (%zd given)", what, n, nargs);
    return false;
  }
  for (int i = 0; i < n; i++) out[i] = i < nargs ? args[i] : nullptr;
  const Py_ssize_t nk = kwnames ? PyTuple_GET_SIZE(kwnames) : 0;
  for (Py_ssize_t k = 0; k < nk; k++) {
    PyObject* key = PyTuple_GET_ITEM(kwnames, k);
    int at = 0;
    while (at < n && PyUnicode_CompareWithASCIIString(key, names[at]) != 0) at++;
    if (at == n) {
      PyErr_Format(PyExc_TypeError, "%s() got an unexpected keyword argument '%U'", what, key);
      return false;
    }
    if (out[at]) {
      PyErr_Format(PyExc_TypeError, "%s() got multiple values for argument '%s'", what, names[at]);
      return false;
    }
    out[at] = args[nargs + k];
  }
  for (int i = 0; i < required; i++)
    if (!out[i]) {
      PyErr_Format(PyExc_TypeError, "%s() missing required argument '%s'", what, names[i]);
      return false;
    }
  return true;
}

const at::Tensor* tensor_of(PyObject* o) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "a torch.Tensor is expected, got %s", Py_TYPE(o)->tp_name);
    return nullptr;
  }
  return &THPVariable_Unpack(o);
}
bool none(PyObject* o) { return !o || o == Py_None; }

bool device_ptr(const at::Tensor& t, void** p) {
  if (!t.is_cuda()) {
    PyErr_SetString(PyExc_ValueError, "device tensor expected");
    return false;
  }
  *p = t.data_ptr();
  return true;
}
bool dtype_code(const at::Tensor& t, int32_t* code) {
  const at::ScalarType s = t.scalar_type();
  if (s == at::kFloat) { *code = HBMM_F32; return true; }
  if (s == at::kBFloat16) { *code = HBMM_BF16; return true; }
  PyErr_Format(PyExc_TypeError, "only float32 and bfloat16 tensors are accepted, got torch.%s", c10::toString(s));
  return false;
}
bool integer(PyObject* o, long long* v) {
  *v = PyLong_AsLongLong(o);
  return !(*v == -1 && PyErr_Occurred());
}
bool small_integer(PyObject* o, int32_t* v) {
  long long w;
  if (!integer(o, &w)) return false;
  *v = static_cast<int32_t>(w);               // as ctypes passes it on
  return true;
}
// The bytes behind a ctypes structure, of the type it is declared as and no other: what they hold is taken for sizes and addresses.
template <typename T>
struct Struct {
  Py_buffer view{};
  const T* p = nullptr;
  ~Struct() { if (view.obj) PyBuffer_Release(&view); }
  bool open(PyObject* o, PyTypeObject* type) {
    if (!PyObject_TypeCheck(o, type)) {
      PyErr_Format(PyExc_TypeError, "%s expected, got %s", type->tp_name, Py_TYPE(o)->tp_name);
      return false;
    }
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) return false;
    if (view.len < static_cast<Py_ssize_t>(sizeof(T))) {
      PyErr_Format(PyExc_TypeError, "%s is shorter than the library's", type->tp_name);
      return false;
    }
    p = static_cast<const T*>(view.buf);
    return true;
  }
  bool open_desc(PyObject* operand) {
    PyObject* d = PyObject_GetAttr(operand, s_desc);
    if (!d) return false;
    const bool ok = open(d, t_operand);
    Py_DECREF(d);                             // the view holds it
    return ok;
  }
};
bool stream_of(PyObject* o, void** s) {
  if (none(o)) {
    *s = c10::cuda::getCurrentCUDAStream().stream();
    return true;
  }
  PyObject* h = PyObject_GetAttr(o, s_cuda_stream);
  if (!h) return false;
  const unsigned long long v = PyLong_AsUnsignedLongLong(h);
  Py_DECREF(h);
  if (v == static_cast<unsigned long long>(-1) && PyErr_Occurred()) return false;
  *s = reinterpret_cast<void*>(static_cast<uintptr_t>(v));
  return true;
}
struct Owned {                     // one reference, given back at the end
  PyObject* o;
  ~Owned() { Py_XDECREF(o); }
};
struct Buffer {
  void* p = nullptr;
  size_t bytes = 0;
  bool open(PyObject* o) {                    // None: no workspace
    if (none(o)) return true;
    const at::Tensor* t = tensor_of(o);
    if (!t || !device_ptr(*t, &p)) return false;
    bytes = t->nbytes();
    return true;
  }
};
PyObject* done(int32_t status, const char* where, PyObject* result) {
  if (status != HBMM_OK) {
    PyObject* e = PyObject_CallFunction(g_error, "is", static_cast<int>(status), where);
    if (e) {
      PyErr_SetObject(g_error, e);
      Py_DECREF(e);
    }
    return nullptr;
  }
  Py_INCREF(result);
  return result;
}
#define HBMM_CALL(expr)            \
  int32_t status;                  \
  Py_BEGIN_ALLOW_THREADS;          \
  status = (expr);                 \
  Py_END_ALLOW_THREADS

PyObject* py_quantize(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  HANDLE_TH_ERRORS
  static const char* const names[] = {"x", "out", "stream"};
  PyObject* a[3];
  if (!take("quantize", args, nargs, kw, names, 3, 2, a)) return nullptr;
  const at::Tensor* x = tensor_of(a[0]);
  if (!x) return nullptr;
  if (x->dim() != 2 || x->stride(1) != 1) {
    PyErr_SetString(PyExc_ValueError, "x must be a row-major 2-D tensor");
    return nullptr;
  }
  void *p, *s;
  int32_t dt;
  Struct<hbmm_operand> out;
  if (!out.open_desc(a[1]) || !device_ptr(*x, &p) || !dtype_code(*x, &dt) || !stream_of(a[2], &s)) return nullptr;
  const int64_t rows = x->size(0), K = x->size(1), ld = x->stride(0);
  HBMM_CALL(f_quantize(p, dt, rows, K, ld, out.p, s));
  return done(status, "hbmm_quantize", a[1]);
  END_HANDLE_TH_ERRORS
}

PyObject* gemm_any(const char* what, const char* where, bool ex, PyObject** a, PyObject* path_o, PyObject* ws_o, PyObject* stream_o) {
  Buffer ws;
  Struct<hbmm_operand> A, W;
  void *c, *s;
  int32_t path = HBMM_PATH_AUTO;
  if (!ws.open(ws_o) || !A.open_desc(a[0]) || !W.open_desc(a[1])) return nullptr;
  const at::Tensor* C = tensor_of(a[2]);
  if (!C || !device_ptr(*C, &c) || (ex && !small_integer(path_o, &path)) || !stream_of(stream_o, &s)) return nullptr;
  const int64_t ldc = C->stride(0);
  HBMM_CALL(ex ? f_gemm_ex(A.p, W.p, static_cast<float*>(c), ldc, ws.p, ws.bytes, path, s) : f_gemm(A.p, W.p, static_cast<float*>(c), ldc, ws.p, ws.bytes, s));
  return done(status, where, a[2]);
}
PyObject* py_gemm(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  HANDLE_TH_ERRORS
  static const char* const names[] = {"A", "W", "C", "workspace", "stream"};
  PyObject* a[5];
  if (!take("gemm", args, nargs, kw, names, 5, 3, a)) return nullptr;
  return gemm_any("gemm", "hbmm_gemm", false, a, nullptr, a[3], a[4]);
  END_HANDLE_TH_ERRORS
}
PyObject* py_gemm_ex(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  HANDLE_TH_ERRORS
  static const char* const names[] = {"A", "W", "C", "path", "workspace", "stream"};
  PyObject* a[6];
  if (!take("gemm_ex", args, nargs, kw, names, 6, 4, a)) return nullptr;
  return gemm_any("gemm_ex", "hbmm_gemm_ex", true, a, a[3], a[4], a[5]);
  END_HANDLE_TH_ERRORS
}

PyObject* py_conv_im2col(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  HANDLE_TH_ERRORS
  static const char* const names[] = {"x", "geom", "beta_a", "a_scale_dtype", "W", "C_out", "workspace", "stream", "flags"};
  PyObject* a[9];
  if (!take("conv_im2col", args, nargs, kw, names, 9, 7, a)) return nullptr;
  const at::Tensor* x = tensor_of(a[0]);
  if (!x) return nullptr;
  if (!x->is_contiguous()) {
    PyErr_SetString(PyExc_ValueError, "x must be a contiguous NCHW tensor");
    return nullptr;
  }
  void *p, *c = nullptr, *s;
  int32_t dt, beta, sdt;
  long long flags = 0;
  int64_t ldc = 0;
  Struct<hbmm_conv_geom> geom;
  Struct<hbmm_operand> W;
  Buffer ws;
  if (!geom.open(a[1], t_geom) || !W.open_desc(a[4]) || !device_ptr(*x, &p) || !dtype_code(*x, &dt) || !small_integer(a[2], &beta) ||
      !small_integer(a[3], &sdt) || (!none(a[8]) && !integer(a[8], &flags)))
    return nullptr;
  if (!none(a[5])) {
    const at::Tensor* C = tensor_of(a[5]);
    if (!C || !device_ptr(*C, &c)) return nullptr;
    ldc = C->stride(0);
  }
  if (!ws.open(a[6]) || !stream_of(a[7], &s)) return nullptr;
  HBMM_CALL(f_conv(p, dt, geom.p, beta, sdt, W.p, static_cast<float*>(c), ldc, ws.p, ws.bytes, static_cast<uint32_t>(flags), s));
  return done(status, flags ? "hbmm_conv_im2col_ex" : "hbmm_conv_im2col", a[5]);
  END_HANDLE_TH_ERRORS
}

PyObject* py_conv_im2col_fused(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  HANDLE_TH_ERRORS
  static const char* const names[] = {"x", "geom", "beta_a", "a_scale_dtype", "W", "ep", "workspace", "stream", "flags"};
  PyObject* a[9];
  if (!take("conv_im2col_fused", args, nargs, kw, names, 9, 7, a)) return nullptr;
  const at::Tensor* x = tensor_of(a[0]);
  if (!x) return nullptr;
  if (!x->is_contiguous()) {
    PyErr_SetString(PyExc_ValueError, "x must be contiguous");
    return nullptr;
  }
  void *p, *s;
  int32_t dt, beta, sdt;
  long long flags = 0;
  Struct<hbmm_conv_geom> geom;
  Struct<hbmm_operand> W;
  Struct<hbmm_epilogue> ep;
  Buffer ws;
  if (!geom.open(a[1], t_geom) || !W.open_desc(a[4]) || !ep.open(a[5], t_epilogue) || !device_ptr(*x, &p) || !dtype_code(*x, &dt) ||
      !small_integer(a[2], &beta) || !small_integer(a[3], &sdt) || !ws.open(a[6]) || !stream_of(a[7], &s) || (a[8] && !integer(a[8], &flags)))
    return nullptr;
  HBMM_CALL(f_conv_fused(p, dt, geom.p, beta, sdt, W.p, ep.p, ws.p, ws.bytes, static_cast<uint32_t>(flags), s));
  return done(status, "hbmm_conv_im2col_fused", Py_None);
  END_HANDLE_TH_ERRORS
}

PyObject* py_binarize_backward(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  HANDLE_TH_ERRORS
  static const char* const names[] = {"x", "gy", "beta", "gx", "stream"};
  PyObject* a[5];
  if (!take("binarize_backward", args, nargs, kw, names, 5, 3, a)) return nullptr;
  const at::Tensor *x = tensor_of(a[0]), *gy = x ? tensor_of(a[1]) : nullptr;
  if (!gy) return nullptr;
  if (x->scalar_type() != at::kFloat || gy->scalar_type() != at::kFloat || x->sizes() != gy->sizes() || x->dim() != 2) {
    PyErr_SetString(PyExc_ValueError, "x and gy must be fp32 matrices of one shape");
    return nullptr;
  }
  if (x->stride(1) != 1 || gy->stride(1) != 1) {
    PyErr_SetString(PyExc_ValueError, "rows must be contiguous");
    return nullptr;
  }
  at::Tensor own;
  PyObject* result = a[3];
  if (none(result)) {
    own = at::empty(x->sizes(), at::TensorOptions().dtype(at::kFloat).device(x->device()));
    result = THPVariable_Wrap(own);
    if (!result) return nullptr;
  } else {
    Py_INCREF(result);
  }
  const Owned keep{result};
  const at::Tensor* gx = tensor_of(result);
  void *px, *pg, *po, *s;
  int32_t beta;
  if (!gx || !device_ptr(*x, &px) || !device_ptr(*gy, &pg) || !small_integer(a[2], &beta) || !device_ptr(*gx, &po) || !stream_of(a[4], &s)) return nullptr;
  const int64_t ldx = x->stride(0), ldg = gy->stride(0), rows = x->size(0), K = x->size(1), ldo = gx->stride(0);
  HBMM_CALL(f_backward(static_cast<const float*>(px), ldx, static_cast<const float*>(pg), ldg, rows, K, beta, static_cast<float*>(po), ldo, s));
  return done(status, "hbmm_binarize_backward", result);
  END_HANDLE_TH_ERRORS
}

PyObject* py_binarize_dense(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  HANDLE_TH_ERRORS
  static const char* const names[] = {"x", "beta", "out_dtype", "out", "stream"};
  PyObject* a[5];
  if (!take("binarize_dense", args, nargs, kw, names, 5, 2, a)) return nullptr;
  const at::Tensor* x = tensor_of(a[0]);
  if (!x) return nullptr;
  if (x->scalar_type() != at::kFloat || x->dim() != 2 || x->stride(1) != 1) {
    PyErr_SetString(PyExc_ValueError, "x must be an fp32 matrix with contiguous rows");
    return nullptr;
  }
  int32_t beta, out_code = HBMM_F32;
  if ((a[2] && !small_integer(a[2], &out_code)) || !small_integer(a[1], &beta)) return nullptr;
  const at::ScalarType tdt = out_code == HBMM_BF16 ? at::kBFloat16 : at::kFloat;
  PyObject* result = a[3];
  if (none(result)) {
    at::Tensor own = at::empty(x->sizes(), at::TensorOptions().dtype(tdt).device(x->device()));
    result = THPVariable_Wrap(own);
    if (!result) return nullptr;
  } else {
    Py_INCREF(result);
  }
  const Owned keep{result};
  const at::Tensor* out = tensor_of(result);
  if (!out) return nullptr;
  if (out->scalar_type() != tdt || out->sizes() != x->sizes() || out->stride(1) != 1) {
    PyErr_SetString(PyExc_ValueError, "out must match x's shape and the requested type");
    return nullptr;
  }
  void *px, *po, *s;
  if (!device_ptr(*x, &px) || !device_ptr(*out, &po) || !stream_of(a[4], &s)) return nullptr;
  const int64_t ldx = x->stride(0), rows = x->size(0), K = x->size(1), ldo = out->stride(0);
  HBMM_CALL(f_dense(static_cast<const float*>(px), ldx, rows, K, beta, po, out_code, ldo, s));
  return done(status, "hbmm_binarize_dense", result);
  END_HANDLE_TH_ERRORS
}

// ---- 8-bit operands.  The descriptor is made from the tensors of an Fp8Operand at each call, so that a call takes what they are now.

// Tensors of one call lie on the current device: the launch and the default stream are that device's.
bool on_current_device(const at::Tensor& t) {
  if (!t.is_cuda()) {
    PyErr_SetString(PyExc_ValueError, "device tensor expected");
    return false;
  }
  if (t.get_device() != c10::cuda::current_device()) {
    PyErr_SetString(PyExc_ValueError, "tensors of the current device expected");
    return false;
  }
  return true;
}
// A matrix with contiguous rows; `pitch`: elements between rows, a whole number of 16 bytes for a single row, whose stride says nothing.
bool matrix(const at::Tensor& t, const char* what, int64_t* pitch) {
  if (t.dim() != 2 || (t.size(1) > 1 && t.stride(1) != 1)) {
    PyErr_Format(PyExc_ValueError, "%s must be a matrix with contiguous rows", what);
    return false;
  }
  const int64_t per = 16 / static_cast<int64_t>(t.element_size());
  *pitch = t.size(0) == 1 ? (t.size(1) + per - 1) / per * per : t.stride(0);
  return true;
}
struct Fp8 {
  hbmm_fp8_operand d{};
  PyObject *codes = nullptr, *scales = nullptr;       // held while the call runs
  ~Fp8() { Py_XDECREF(codes); Py_XDECREF(scales); }
  bool number(PyObject* o, PyObject* name, long long* v) {
    PyObject* p = PyObject_GetAttr(o, name);
    if (!p) return false;
    const bool ok = integer(p, v);
    Py_DECREF(p);
    return ok;
  }
  bool open(PyObject* o) {
    if (!PyObject_TypeCheck(o, t_fp8)) {
      PyErr_Format(PyExc_TypeError, "Fp8Operand expected, got %s", Py_TYPE(o)->tp_name);
      return false;
    }
    long long K, block_rows;
    if (!(codes = PyObject_GetAttr(o, s_codes)) || !(scales = PyObject_GetAttr(o, s_scales)) || !number(o, s_K, &K) ||
        !number(o, s_block_rows, &block_rows))
      return false;
    const at::Tensor *c = tensor_of(codes), *s = c ? tensor_of(scales) : nullptr;
    if (!s) return false;
    const at::ScalarType ct = c->scalar_type();
    if ((ct != at::kByte && ct != at::kFloat8_e4m3fn) || s->scalar_type() != at::kFloat) {
      PyErr_SetString(PyExc_ValueError, "codes must be float8_e4m3fn or uint8, scales float32");
      return false;
    }
    if (!matrix(*c, "codes", &d.ld_codes) || !matrix(*s, "scales", &d.ld_scales)) return false;
    if (block_rows != 1 && block_rows != 128) {
      PyErr_SetString(PyExc_ValueError, "block_rows must be 1 or 128");
      return false;
    }
    if (K < 1 || c->size(0) < 1 || c->size(1) < K || s->size(0) < (c->size(0) + block_rows - 1) / block_rows || s->size(1) < (K + 127) / 128) {
      PyErr_SetString(PyExc_ValueError, "codes or scales are smaller than their operand");
      return false;
    }
    if (!on_current_device(*c) || !on_current_device(*s)) return false;
    d.rows = c->size(0); d.K = K; d.block_rows = static_cast<int32_t>(block_rows);
    d.codes = static_cast<uint8_t*>(c->data_ptr());
    d.scales = static_cast<float*>(s->data_ptr());
    return true;
  }
};
// A tensor argument of the given extents.
const at::Tensor* sized(PyObject* o, const char* what, int64_t rows, int64_t cols, int64_t* pitch) {
  const at::Tensor* t = tensor_of(o);
  if (!t || !matrix(*t, what, pitch)) return nullptr;
  if (t->size(0) != rows || t->size(1) != cols) {
    PyErr_Format(PyExc_ValueError, "%s must be [%lld, %lld]", what, static_cast<long long>(rows), static_cast<long long>(cols));
    return nullptr;
  }
  return on_current_device(*t) ? t : nullptr;
}

PyObject* py_fp8_quantize(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  HANDLE_TH_ERRORS
  static const char* const names[] = {"x", "out", "stream"};
  PyObject* a[3];
  Fp8 out;
  if (!take("fp8_quantize", args, nargs, kw, names, 3, 2, a) || !out.open(a[1])) return nullptr;
  int64_t ld;
  int32_t dt;
  void* s;
  const at::Tensor* x = sized(a[0], "x", out.d.rows, out.d.K, &ld);
  if (!x || !dtype_code(*x, &dt) || !stream_of(a[2], &s)) return nullptr;
  const void* p = x->data_ptr();
  HBMM_CALL(f_fp8_quantize(p, dt, out.d.rows, out.d.K, ld, &out.d, s));
  return done(status, "hbmm_fp8_quantize", a[1]);
  END_HANDLE_TH_ERRORS
}

PyObject* fp8_product(const char* where, bool transposed, PyObject** a) {
  Fp8 A, W;
  if (!A.open(a[0]) || !W.open(a[1])) return nullptr;
  int64_t ld;
  int32_t dt;
  void* s;
  const at::Tensor* C = sized(a[2], transposed ? "GX" : "C", A.d.rows, transposed ? W.d.K : W.d.rows, &ld);
  if (!C || !dtype_code(*C, &dt) || !stream_of(a[3], &s)) return nullptr;
  void* p = C->data_ptr();
  HBMM_CALL((transposed ? f_fp8_input_grad : f_fp8_gemm)(&A.d, &W.d, p, dt, ld, s));
  return done(status, where, a[2]);
}
PyObject* py_fp8_gemm(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  HANDLE_TH_ERRORS
  static const char* const names[] = {"A", "W", "C", "stream"};
  PyObject* a[4];
  return take("fp8_gemm", args, nargs, kw, names, 4, 3, a) ? fp8_product("hbmm_fp8_gemm", false, a) : nullptr;
  END_HANDLE_TH_ERRORS
}
PyObject* py_fp8_input_grad(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  HANDLE_TH_ERRORS
  static const char* const names[] = {"GY", "W", "GX", "stream"};
  PyObject* a[4];
  return take("fp8_input_grad", args, nargs, kw, names, 4, 3, a) ? fp8_product("hbmm_fp8_input_grad", true, a) : nullptr;
  END_HANDLE_TH_ERRORS
}

PyObject* py_fp8_weight_grad(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  HANDLE_TH_ERRORS
  static const char* const names[] = {"gy", "X", "GW", "base", "stream"};
  PyObject* a[5];
  Fp8 X;
  if (!take("fp8_weight_grad", args, nargs, kw, names, 5, 3, a) || !X.open(a[1])) return nullptr;
  const at::Tensor *gy = tensor_of(a[0]), *gw = gy ? tensor_of(a[2]) : nullptr, *base = nullptr;
  if (!gw || gw->dim() != 2) {
    if (gw) PyErr_SetString(PyExc_ValueError, "GW must be a matrix with contiguous rows");
    return nullptr;
  }
  const int64_t N = gw->size(0);
  int64_t ldg, ldw, ldb = 0;
  int32_t dt;
  void* s;
  if (!sized(a[0], "gy", X.d.rows, N, &ldg) || !sized(a[2], "GW", N, X.d.K, &ldw) || !dtype_code(*gy, &dt)) return nullptr;
  if (!none(a[3]) && !(base = sized(a[3], "base", N, X.d.K, &ldb))) return nullptr;
  if (gw->scalar_type() != at::kFloat || (base && base->scalar_type() != at::kFloat)) {
    PyErr_SetString(PyExc_ValueError, "GW and base must be float32");
    return nullptr;
  }
  if (!stream_of(a[4], &s)) return nullptr;
  const void* pg = gy->data_ptr();
  const float* pb = base ? static_cast<const float*>(base->data_ptr()) : nullptr;
  float* pw = static_cast<float*>(gw->data_ptr());
  HBMM_CALL(f_fp8_weight_grad(pg, dt, N, ldg, &X.d, pb, ldb, pw, ldw, s));
  return done(status, "hbmm_fp8_weight_grad", a[2]);
  END_HANDLE_TH_ERRORS
}

PyObject* py_fp8_binarize_backward(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  HANDLE_TH_ERRORS
  static const char* const names[] = {"X", "gy", "beta", "gx", "stream"};
  PyObject* a[5];
  Fp8 X;
  if (!take("fp8_binarize_backward", args, nargs, kw, names, 5, 3, a) || !X.open(a[0])) return nullptr;
  int64_t ldg, ldo;
  int32_t dt, beta;
  void* s;
  const at::Tensor* gy = sized(a[1], "gy", X.d.rows, X.d.K, &ldg);
  if (!gy || !dtype_code(*gy, &dt)) return nullptr;
  PyObject* result = a[3];
  if (none(result)) {
    const at::Tensor own = at::empty(gy->sizes(), gy->options());
    if (!(result = THPVariable_Wrap(own))) return nullptr;
  } else {
    Py_INCREF(result);
  }
  const Owned keep{result};
  const at::Tensor* gx = sized(result, "gx", X.d.rows, X.d.K, &ldo);
  if (!gx) return nullptr;
  if (gx->scalar_type() != gy->scalar_type()) {
    PyErr_SetString(PyExc_ValueError, "gx must have gy's type");
    return nullptr;
  }
  if (!small_integer(a[2], &beta) || !stream_of(a[4], &s)) return nullptr;
  const void* pg = gy->data_ptr();
  void* po = gx->data_ptr();
  HBMM_CALL(f_fp8_backward(&X.d, pg, dt, ldg, beta, po, ldo, s));
  return done(status, "hbmm_fp8_binarize_backward", result);
  END_HANDLE_TH_ERRORS
}

// connect_fp8(Fp8Operand, addresses of the C functions in the order of the f_fp8 pointers above)
PyObject* py_connect_fp8(PyObject*, PyObject* args) {
  PyObject* type;
  unsigned long long p[5];
  if (!PyArg_ParseTuple(args, "O!KKKKK", &PyType_Type, &type, &p[0], &p[1], &p[2], &p[3], &p[4])) return nullptr;
  f_fp8_quantize = reinterpret_cast<decltype(f_fp8_quantize)>(p[0]);
  f_fp8_gemm = reinterpret_cast<decltype(f_fp8_gemm)>(p[1]);
  f_fp8_input_grad = reinterpret_cast<decltype(f_fp8_input_grad)>(p[2]);
  f_fp8_weight_grad = reinterpret_cast<decltype(f_fp8_weight_grad)>(p[3]);
  f_fp8_backward = reinterpret_cast<decltype(f_fp8_backward)>(p[4]);
  Py_INCREF(type);
  Py_XSETREF(t_fp8, reinterpret_cast<PyTypeObject*>(type));
  Py_RETURN_NONE;
}

// connect(HbmmError, hbmm_operand, hbmm_conv_geom, hbmm_epilogue, addresses of the C functions in the order of the f_ pointers above)
PyObject* py_connect(PyObject*, PyObject* args) {
  PyObject *err, *types[3];
  unsigned long long p[7];
  if (!PyArg_ParseTuple(args, "OO!O!O!KKKKKKK", &err, &PyType_Type, &types[0], &PyType_Type, &types[1], &PyType_Type, &types[2], &p[0], &p[1],
                        &p[2], &p[3], &p[4], &p[5], &p[6]))
    return nullptr;
  f_quantize = reinterpret_cast<decltype(f_quantize)>(p[0]);
  f_gemm = reinterpret_cast<decltype(f_gemm)>(p[1]);
  f_gemm_ex = reinterpret_cast<decltype(f_gemm_ex)>(p[2]);
  f_conv = reinterpret_cast<decltype(f_conv)>(p[3]);
  f_conv_fused = reinterpret_cast<decltype(f_conv_fused)>(p[4]);
  f_dense = reinterpret_cast<decltype(f_dense)>(p[5]);
  f_backward = reinterpret_cast<decltype(f_backward)>(p[6]);
  Py_INCREF(err);
  Py_XSETREF(g_error, err);
  PyTypeObject** const held[] = {&t_operand, &t_geom, &t_epilogue};
  for (int i = 0; i < 3; i++) {
    Py_INCREF(types[i]);
    Py_XSETREF(*held[i], reinterpret_cast<PyTypeObject*>(types[i]));
  }
  Py_RETURN_NONE;
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL | METH_KEYWORDS
PyMethodDef methods[] = {
    {"quantize", FAST(py_quantize),
     "quantize($module, /, x, out, stream=None)\n--\n\nhbmm_quantize: Hadamard-binarize and pack the rows of ``x`` [rows, K] into ``out``."},
    {"gemm", FAST(py_gemm),
     "gemm($module, /, A, W, C, workspace=None, stream=None)\n--\n\nhbmm_gemm: C[M, N] (fp32, row-major, caller-allocated) = A~ W~^T."},
    {"gemm_ex", FAST(py_gemm_ex),
     "gemm_ex($module, /, A, W, C, path, workspace=None, stream=None)\n--\n\nhbmm_gemm_ex: hbmm_gemm on the path asked for."},
    {"conv_im2col", FAST(py_conv_im2col),
     "conv_im2col($module, /, x, geom, beta_a, a_scale_dtype, W, C_out, workspace, stream=None, flags=0)\n--\n\n"
     "hbmm_conv_im2col (flags == 0) / hbmm_conv_im2col_ex: x NCHW contiguous; C_out fp32 [B*Ho*Wo, N]."},
    {"conv_im2col_fused", FAST(py_conv_im2col_fused),
     "conv_im2col_fused($module, /, x, geom, beta_a, a_scale_dtype, W, ep, workspace, stream=None, flags=0)\n--\n\n"
     "hbmm_conv_im2col_fused: x NCHW contiguous (or NHWC bf16 with CONV_INPUT_NHWC)."},
    {"binarize_dense", FAST(py_binarize_dense),
     "binarize_dense($module, /, x, beta, out_dtype=0, out=None, stream=None)\n--\n\n"
     "hbmm_binarize_dense: x fp32 [rows, K] (row stride >= K, unit column stride); returns delta (.) Sign(x) as fp32 or bf16."},
    {"binarize_backward", FAST(py_binarize_backward),
     "binarize_backward($module, /, x, gy, beta, gx=None, stream=None)\n--\n\n"
     "hbmm_binarize_backward: x, gy fp32 [rows, K] (row stride >= K, unit column stride); returns gx = dC/dX."},
    {"fp8_quantize", FAST(py_fp8_quantize),
     "fp8_quantize($module, /, x, out, stream=None)\n--\n\n"
     "hbmm_fp8_quantize: x [rows, K] fp32 / bf16 into the Fp8Operand ``out``, which is returned."},
    {"fp8_gemm", FAST(py_fp8_gemm),
     "fp8_gemm($module, /, A, W, C, stream=None)\n--\n\nhbmm_fp8_gemm: C[M, N] (fp32 / bf16, caller-allocated) = A^ W^^T."},
    {"fp8_input_grad", FAST(py_fp8_input_grad),
     "fp8_input_grad($module, /, GY, W, GX, stream=None)\n--\n\nhbmm_fp8_input_grad: GX[M, K] (fp32 / bf16, caller-allocated) = GY^ W^."},
    {"fp8_weight_grad", FAST(py_fp8_weight_grad),
     "fp8_weight_grad($module, /, gy, X, GW, base=None, stream=None)\n--\n\n"
     "hbmm_fp8_weight_grad: GW[N, K] (fp32, caller-allocated) = gy^T X^ (+ base, which may be GW); gy bf16 [M, N], X the 8-bit copy of the\n"
     "activations."},
    {"fp8_binarize_backward", FAST(py_fp8_binarize_backward),
     "fp8_binarize_backward($module, /, X, gy, beta, gx=None, stream=None)\n--\n\n"
     "hbmm_fp8_binarize_backward: binarize_backward from the 8-bit copy X of x; gy, gx [rows, K] fp32 / bf16."},
    {"connect", py_connect, METH_VARARGS, nullptr},
    {"connect_fp8", py_connect_fp8, METH_VARARGS, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() {
  s_desc = PyUnicode_InternFromString("desc");
  s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  s_codes = PyUnicode_InternFromString("codes");
  s_scales = PyUnicode_InternFromString("scales");
  s_K = PyUnicode_InternFromString("K");
  s_block_rows = PyUnicode_InternFromString("block_rows");
  if (!s_desc || !s_cuda_stream || !s_codes || !s_scales || !s_K || !s_block_rows) return nullptr;
  PyObject* m = PyModule_Create(&module_def);
  if (m && PyModule_AddStringConstant(m, "BUILT_FOR", HBMM_BUILT_FOR) != 0) Py_CLEAR(m);
  return m;
}
