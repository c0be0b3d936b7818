// Argument marshalling of the Python binding: torch tensors -> device pointers -> C entry points.
// Nothing is computed here.  A call through ctypes costs 8 to 12 us of interpreter time (four
// attribute look-ups and a conversion per tensor), as long as a small layer takes on the GPU;
// through this module 1.3 us.  The entry points are called by address (bind()), so the module
// works with whichever build of the library the Python side has loaded.
#define PY_SSIZE_T_CLEAN
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <algorithm>
#include <climits>
#include <cstring>
#include <optional>
#include <string>

#include "xnor.h"

namespace {

// The entry points this module calls, in the order bind() takes their addresses.
struct Entry {
  decltype(&xnor_binarize_weights) binarize_weights;
  decltype(&xnor_binactiv) binactiv;
  decltype(&xnor_conv2d_forward) conv2d_forward;
  decltype(&xnor_shortcut_conv1x1) shortcut_conv1x1;
  decltype(&xnor_conv2d_forward_binactiv) conv2d_forward_binactiv;
  decltype(&xnor_binactiv_finish) binactiv_finish;
  decltype(&xnor_maxpool2d) maxpool2d;
  decltype(&xnor_binactiv_kbit) binactiv_kbit;
  decltype(&xnor_conv2d_forward_kbit) conv2d_forward_kbit;
  decltype(&xnor_bwn_prepare_input) bwn_prepare_input;
  decltype(&xnor_bwn_conv2d_forward) bwn_conv2d_forward;
  decltype(&xnor_binarize_weights_transposed) binarize_weights_transposed;
  decltype(&xnor_binary_gradient_backward) binary_gradient_backward;
  decltype(&xnor_rmsnorm) rmsnorm;
  decltype(&xnor_rmsnorm_quant) rmsnorm_quant;
  decltype(&xnor_rmsnorm_backward) rmsnorm_backward;
  decltype(&xnor_w4_quantize) w4_quantize;
  decltype(&xnor_w4_pack) w4_pack;
  decltype(&xnor_w4_dequantize) w4_dequantize;
  decltype(&xnor_w4_matmul) w4_matmul;
} E;
constexpr Py_ssize_t kEntries = sizeof(Entry) / sizeof(void *);
PyObject *desc_type = nullptr;         // the ctypes structure xnor_conv_desc
PyObject *py_address = nullptr;        // (object, type name) -> its checked address through Python attributes
PyObject *w4_desc_type = nullptr;      // the ctypes structure xnor_w4_desc
PyObject *py_describe = nullptr;       // object -> (address, type, shape, strides, device) through Python attributes

// Arguments of one call, converted in order; the first failure sets a Python error and sticks.
struct Args {
  PyObject *const *a;
  Py_ssize_t n;
  bool ok;
  Py_ssize_t i = 0;

  Args(PyObject *const *args, Py_ssize_t nargs, Py_ssize_t want) : a(args), n(nargs), ok(nargs == want) {
    if (!ok) PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, nargs);
  }
  void fail_attr(const char *fmt, PyObject *t, const char *attr) {
    if (PyObject *v = PyObject_GetAttrString(t, attr)) {
      PyErr_Format(PyExc_ValueError, fmt, v);
      Py_DECREF(v);
    }
    ok = false;
  }
  // Tensors and parameters are read here.  Subclasses and other objects with a tensor's attributes may
  // define these in Python, so they are asked there.
  void *ptr(at::ScalarType type, const char *name) {
    PyObject *o = a[i++];
    if (!ok || o == Py_None) return nullptr;
    if (!THPVariable_CheckExact(o)) {
      PyObject *v = PyObject_CallFunction(py_address, "Os", o, name);
      void *p = v != nullptr ? PyLong_AsVoidPtr(v) : nullptr;
      Py_XDECREF(v);
      ok = !PyErr_Occurred();
      return p;
    }
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda()) {
      fail_attr("libxnor takes device pointers: tensor is on %S", o, "device");
    } else if (!t.is_contiguous()) {
      PyErr_SetString(PyExc_ValueError, "tensor must be contiguous");
      ok = false;
    } else if (t.scalar_type() != type) {
      const std::string fmt = std::string("expected torch.") + name + ", got %S";
      fail_attr(fmt.c_str(), o, "dtype");
    } else {
      return t.data_ptr();
    }
    return nullptr;
  }
  float *f32() { return (float *)ptr(at::kFloat, "float32"); }
  uint32_t *u32() { return (uint32_t *)ptr(at::kInt, "int32"); }
  int32_t *i32() { return (int32_t *)ptr(at::kInt, "int32"); }
  uint16_t *bf16() { return (uint16_t *)ptr(at::kBFloat16, "bfloat16"); }
  int num() {
    PyObject *o = a[i++];
    if (!ok) return 0;
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) ok = false;
    else if (v != (long)(int)v) { PyErr_SetString(PyExc_OverflowError, "argument out of int range"); ok = false; }
    return (int)v;
  }
  // an xnor_conv_desc and nothing else of its size, read through the buffer protocol
  xnor_conv_desc desc() {
    xnor_conv_desc d = {};
    PyObject *o = a[i++];
    if (!ok) return d;
    Py_buffer b;
    const int is = PyObject_IsInstance(o, desc_type);
    if (is == 0) PyErr_Format(PyExc_TypeError, "expected an xnor_conv_desc, got %S", (PyObject *)Py_TYPE(o));
    if (is != 1 || PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) { ok = false; return d; }
    memcpy(&d, b.buf, std::min((size_t)b.len, sizeof(d)));
    PyBuffer_Release(&b);
    return d;
  }
  // None: torch's current stream; else a torch stream, or a raw cudaStream_t as anything int() takes
  void *stream() {
    PyObject *o = a[i++];
    if (!ok) return nullptr;
    if (o == Py_None) return (void *)c10::cuda::getCurrentCUDAStream().stream();
    PyObject *v = PyObject_GetAttrString(o, "cuda_stream");
    if (v == nullptr && PyErr_ExceptionMatches(PyExc_AttributeError)) {
      PyErr_Clear();
      v = PyNumber_Long(o);
    }
    ok = v != nullptr;
    if (!ok) return nullptr;
    void *s = nullptr;
    if (PyLong_Check(v)) s = PyLong_AsVoidPtr(v);
    else PyErr_Format(PyExc_TypeError, "expected a stream, got %S", (PyObject *)Py_TYPE(o));
    Py_DECREF(v);
    if (s == nullptr && PyErr_Occurred()) ok = false;
    return s;
  }
};

// Runs the call without the GIL and returns its status.
template <class F>
PyObject *finish(const Args &A, F &&call) {
  if (!A.ok) return nullptr;
  xnor_status s;
  Py_BEGIN_ALLOW_THREADS
  s = call();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong((long)s);
}

// Sizes of a tensor argument of `dims` dimensions (0: any number, the first size); anything else is an error.
void sizes_of(Args &A, PyObject *o, int dims, int *out) {
  if (!A.ok) return;
  const int want = dims > 0 ? dims : 1;
  if (THPVariable_CheckExact(o)) {
    const at::Tensor &t = THPVariable_Unpack(o);
    A.ok = dims > 0 ? t.dim() == dims : t.dim() > 0;
    for (int i = 0; A.ok && i < want; ++i) out[i] = (int)t.size(i);
  } else {
    PyObject *shape = PyObject_GetAttrString(o, "shape"), *s = shape != nullptr ? PySequence_Tuple(shape) : nullptr;
    Py_XDECREF(shape);
    if (s != nullptr) A.ok = dims > 0 ? PyTuple_GET_SIZE(s) == dims : PyTuple_GET_SIZE(s) > 0;
    for (int i = 0; s != nullptr && A.ok && i < want; ++i) out[i] = (int)PyLong_AsLong(PyTuple_GET_ITEM(s, i));
    Py_XDECREF(s);
    if (PyErr_Occurred()) { A.ok = false; return; }
  }
  if (!A.ok) PyErr_Format(PyExc_ValueError, "expected a tensor of %d dimensions", want);
}

// Torch's accessors throw (a tensor under vmap has no data pointer, one with symbolic sizes no size): an
// exception must become a Python error before it reaches the interpreter, which is C.
template <PyObject *(*kCall)(PyObject *const *, Py_ssize_t)>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  return kCall(args, nargs);
  END_HANDLE_TH_ERRORS
}

#define XNOR_PY(name) PyObject *name(PyObject *const *args, Py_ssize_t nargs)

XNOR_PY(binarize_weights) {          // w, w_packed, alpha, stream
  Args A(args, nargs, 4);
  int z[4] = {};
  if (A.ok) sizes_of(A, args[0], 4, z);
  if (!A.ok) return nullptr;
  const float *w = A.f32(); uint32_t *wp = A.u32(); float *alpha = A.f32(); void *st = A.stream();
  return finish(A, [&] { return E.binarize_weights(w, z[0], z[1], z[2], z[3], wp, alpha, st); });
}

XNOR_PY(binarize_weights_transposed) {   // w, wT_packed, stream
  Args A(args, nargs, 3);
  int z[4] = {};
  if (A.ok) sizes_of(A, args[0], 4, z);
  if (!A.ok) return nullptr;
  const float *w = A.f32(); uint32_t *wp = A.u32(); void *st = A.stream();
  return finish(A, [&] { return E.binarize_weights_transposed(w, z[0], z[1], z[2], z[3], wp, st); });
}

XNOR_PY(binactiv) {                  // x, bn_scale, bn_shift, d, x_packed, A, K, stream
  Args A(args, nargs, 8);
  if (!A.ok) return nullptr;
  const float *x = A.f32(), *sc = A.f32(), *sh = A.f32(); const xnor_conv_desc d = A.desc();
  uint32_t *xp = A.u32(); float *a = A.f32(), *k = A.f32(); void *st = A.stream();
  return finish(A, [&] { return E.binactiv(x, sc, sh, &d, xp, a, k, st); });
}

XNOR_PY(binactiv_kbit) {             // x, bn_scale, bn_shift, d, kbits, x_planes, A, K, stream
  Args A(args, nargs, 9);
  if (!A.ok) return nullptr;
  const float *x = A.f32(), *sc = A.f32(), *sh = A.f32(); const xnor_conv_desc d = A.desc();
  const int kb = A.num(); uint32_t *xp = A.u32(); float *a = A.f32(), *k = A.f32(); void *st = A.stream();
  return finish(A, [&] { return E.binactiv_kbit(x, sc, sh, &d, kb, xp, a, k, st); });
}

XNOR_PY(conv2d_forward) {            // x_packed, w_packed, alpha, K, residual, d, out, acc_out, stream
  Args A(args, nargs, 9);
  if (!A.ok) return nullptr;
  const uint32_t *xp = A.u32(), *wp = A.u32(); const float *al = A.f32(), *k = A.f32(), *res = A.f32();
  const xnor_conv_desc d = A.desc(); float *out = A.f32(); int32_t *acc = A.i32(); void *st = A.stream();
  return finish(A, [&] { return E.conv2d_forward(xp, wp, al, k, res, &d, out, acc, st); });
}

XNOR_PY(conv2d_forward_kbit) {       // x_planes, kbits, w_packed, alpha, K, residual, d, out, acc_out, stream
  Args A(args, nargs, 10);
  if (!A.ok) return nullptr;
  const uint32_t *xp = A.u32(); const int kb = A.num(); const uint32_t *wp = A.u32();
  const float *al = A.f32(), *k = A.f32(), *res = A.f32(); const xnor_conv_desc d = A.desc();
  float *out = A.f32(); int32_t *acc = A.i32(); void *st = A.stream();
  return finish(A, [&] { return E.conv2d_forward_kbit(xp, kb, wp, al, k, res, &d, out, acc, st); });
}

XNOR_PY(conv2d_forward_binactiv) {   // x_packed, w_packed, alpha, K, residual, d, out, next_scale, next_shift,
  Args A(args, nargs, 12);           // x_packed_next, A_parts, stream
  if (!A.ok) return nullptr;
  const uint32_t *xp = A.u32(), *wp = A.u32(); const float *al = A.f32(), *k = A.f32(), *res = A.f32();
  const xnor_conv_desc d = A.desc(); float *out = A.f32(); const float *ns = A.f32(), *nh = A.f32();
  uint32_t *xn = A.u32(); float *ap = A.f32(); void *st = A.stream();
  return finish(A, [&] { return E.conv2d_forward_binactiv(xp, wp, al, k, res, &d, out, ns, nh, xn, ap, st); });
}

XNOR_PY(binactiv_finish) {           // A_parts, parts, d_next, A, K, stream
  Args A(args, nargs, 6);
  if (!A.ok) return nullptr;
  const float *ap = A.f32(); const int parts = A.num(); const xnor_conv_desc d = A.desc();
  float *a = A.f32(), *k = A.f32(); void *st = A.stream();
  return finish(A, [&] { return E.binactiv_finish(ap, parts, &d, a, k, st); });
}

XNOR_PY(shortcut_conv1x1) {          // x, w, stride, out, stream
  Args A(args, nargs, 5);
  int z[4] = {};
  if (A.ok) sizes_of(A, args[0], 4, z);
  if (!A.ok) return nullptr;
  const float *x = A.f32(), *w = A.f32(); const int s = A.num(); float *out = A.f32(); void *st = A.stream();
  int co = 0;                        // filters are [C_out][C_in] or [C_out][C_in][1][1]
  if (args[1] != Py_None) sizes_of(A, args[1], 0, &co);
  return finish(A, [&] { return E.shortcut_conv1x1(x, w, z[0], z[1], z[2], z[3], co, s, out, st); });
}

XNOR_PY(maxpool2d) {                 // x, k, stride, pad, relu, out, stream
  Args A(args, nargs, 7);
  int z[4] = {};
  if (A.ok) sizes_of(A, args[0], 4, z);
  if (!A.ok) return nullptr;
  const float *x = A.f32(); const int k = A.num(), s = A.num(), p = A.num(), r = A.num();
  float *out = A.f32(); void *st = A.stream();
  return finish(A, [&] { return E.maxpool2d(x, z[0], z[1], z[2], z[3], k, s, p, r, out, st); });
}

XNOR_PY(bwn_prepare_input) {         // x, bn_scale, bn_shift, d, x_stream, stream
  Args A(args, nargs, 6);
  if (!A.ok) return nullptr;
  const float *x = A.f32(), *sc = A.f32(), *sh = A.f32(); const xnor_conv_desc d = A.desc();
  uint16_t *xs = A.bf16(); void *st = A.stream();
  return finish(A, [&] { return E.bwn_prepare_input(x, sc, sh, &d, xs, st); });
}

XNOR_PY(bwn_conv2d_forward) {        // x_stream, w_packed, alpha, residual, d, out, stream
  Args A(args, nargs, 7);
  if (!A.ok) return nullptr;
  const uint16_t *xs = A.bf16(); const uint32_t *wp = A.u32(); const float *al = A.f32(), *res = A.f32();
  const xnor_conv_desc d = A.desc(); float *out = A.f32(); void *st = A.stream();
  return finish(A, [&] { return E.bwn_conv2d_forward(xs, wp, al, res, &d, out, st); });
}

XNOR_PY(binary_gradient_backward) {  // g, wT_packed, alpha, d, gmax, g_stream, grad_in, stream
  Args A(args, nargs, 8);
  if (!A.ok) return nullptr;
  const float *g = A.f32(); const uint32_t *wT = A.u32(); const float *al = A.f32();
  const xnor_conv_desc d = A.desc(); float *gm = A.f32(); uint16_t *gs = A.bf16(); float *gi = A.f32();
  void *st = A.stream();
  return finish(A, [&] { return E.binary_gradient_backward(g, wT, al, &d, gm, gs, gi, st); });
}

decltype(&xnor_rmsnorm_work_elems) xnor_work_elems = nullptr;      // a query, not an entry point that launches

// ---- tensors of rows ----------------------------------------------------------------------
// Their calls take sizes, types and strides from the tensors, and refuse tensors that do not fit together.
struct Dense {
  void *p = nullptr;
  int type = -1;                      // at::ScalarType
  int dims = 0;
  long long size[4] = {}, stride[4] = {};
  long long numel = 1;
  int device = -1;
  bool there() const { return type >= 0; }
};

struct RowArgs {
  PyObject *const *a;
  Py_ssize_t n;
  bool ok = true;
  int device = -1;

  RowArgs(PyObject *const *args, Py_ssize_t nargs, Py_ssize_t want) : a(args), n(nargs), ok(nargs == want) {
    if (!ok) PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, nargs);
  }
  void bad(const char *name, const char *what) {
    if (ok) PyErr_Format(PyExc_ValueError, "%s: %s", name, what);
    ok = false;
  }
  bool none(int i) const { return a[i] == Py_None; }

  // A CUDA tensor of up to four dimensions, on the device of the call's other tensors.
  Dense tensor(int i, const char *name) {
    Dense d;
    if (!ok) return d;
    PyObject *o = a[i];
    if (THPVariable_CheckExact(o)) {
      const at::Tensor &t = THPVariable_Unpack(o);
      if (!t.is_cuda()) { bad(name, "libxnor takes device pointers: the tensor is not on a GPU"); return d; }
      d.dims = (int)t.dim();
      if (d.dims > 4) { bad(name, "too many dimensions"); return d; }
      for (int k = 0; k < d.dims; ++k) { d.size[k] = t.size(k); d.stride[k] = t.stride(k); d.numel *= t.size(k); }
      d.type = (int)t.scalar_type();
      d.device = t.get_device();
      d.p = t.data_ptr();
    } else {
      // subclasses and other objects with a tensor's attributes say it themselves
      PyObject *v = PyObject_CallFunctionObjArgs(py_describe, o, nullptr);
      PyObject *shape = nullptr, *strides = nullptr;
      unsigned long long p = 0;
      ok = v != nullptr && PyArg_ParseTuple(v, "KiO!O!i", &p, &d.type, &PyTuple_Type, &shape, &PyTuple_Type, &strides, &d.device);
      if (ok) {
        d.p = (void *)(uintptr_t)p;
        d.dims = (int)PyTuple_GET_SIZE(shape);
        if (d.dims > 4 || PyTuple_GET_SIZE(strides) != d.dims) bad(name, "too many dimensions");
        for (int k = 0; ok && k < d.dims; ++k) {
          d.size[k] = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, k));
          d.stride[k] = PyLong_AsLongLong(PyTuple_GET_ITEM(strides, k));
          d.numel *= d.size[k];
          if (PyErr_Occurred()) ok = false;
        }
      }
      Py_XDECREF(v);
      if (!ok) return Dense();
    }
    if (device < 0) device = d.device;
    else if (device != d.device) { bad(name, "on another device than the tensors before it"); return Dense(); }
    for (int k = 0; k < d.dims; ++k)
      if (d.size[k] > INT_MAX) { bad(name, "a dimension is too large"); return Dense(); }
    return d;
  }
  void want_type(const Dense &d, const char *name, at::ScalarType t) {
    if (ok && d.type != (int)t) PyErr_Format(PyExc_ValueError, "%s: expected %s, got %s", name, c10::toString(t), c10::toString((at::ScalarType)d.type)), ok = false;
  }
  // [rows][cols], columns contiguous; gives the stride from row to row
  Dense rows(int i, const char *name, long long *stride) {
    const Dense d = tensor(i, name);
    *stride = 0;
    if (!ok) return d;
    if (d.dims != 2) bad(name, "expected a tensor of 2 dimensions");
    else if (d.size[1] > 1 && d.stride[1] != 1) bad(name, "the columns must be contiguous");
    *stride = d.size[0] > 1 ? d.stride[0] : d.size[1];
    return d;
  }
  Dense like(int i, const char *name, const Dense &other, long long *stride) {
    const Dense d = rows(i, name, stride);
    if (ok && (d.size[0] != other.size[0] || d.size[1] != other.size[1])) bad(name, "another shape than the rows");
    if (ok) want_type(d, name, (at::ScalarType)other.type);
    return d;
  }
  // dense, of exactly these sizes (0 dimensions given: only of this many elements)
  Dense dense(int i, const char *name, at::ScalarType t, std::initializer_list<long long> sizes) {
    const Dense d = tensor(i, name);
    if (!ok) return d;
    want_type(d, name, t);
    long long want = 1;
    bool same = d.dims == (int)sizes.size();
    int k = 0;
    for (long long s : sizes) { same = same && d.size[k] == s; ++k; want *= s; }
    if (ok && !same) { bad(name, "wrong shape"); return d; }
    long long step = 1;
    for (k = d.dims - 1; ok && k >= 0; --k) {
      if (d.numel > 0 && d.size[k] > 1 && d.stride[k] != step) bad(name, "tensor must be contiguous");
      step *= d.size[k];
    }
    return d;
  }
  int xnor_type_of(const Dense &d, const char *name, bool bytes) {
    switch (d.type) {
      case (int)at::kFloat: return XNOR_F32;
      case (int)at::kBFloat16: return XNOR_BF16;
      case (int)at::kHalf: return XNOR_F16;
      case (int)at::kChar: if (bytes) return XNOR_I8; break;
      case (int)at::kFloat8_e4m3fn: if (bytes) return XNOR_E4M3; break;
      default: break;
    }
    if (ok) PyErr_Format(PyExc_ValueError, "%s: rows of %s are not supported", name, c10::toString((at::ScalarType)d.type));
    ok = false;
    return 0;
  }
  xnor_w4_desc w4(int i) {
    xnor_w4_desc d = {};
    if (!ok) return d;
    Py_buffer b;
    const int is = PyObject_IsInstance(a[i], w4_desc_type);
    if (is == 0) PyErr_Format(PyExc_TypeError, "expected an xnor_w4_desc, got %S", (PyObject *)Py_TYPE(a[i]));
    if (is != 1 || PyObject_GetBuffer(a[i], &b, PyBUF_SIMPLE) != 0) { ok = false; return d; }
    memcpy(&d, b.buf, std::min((size_t)b.len, sizeof(d)));
    PyBuffer_Release(&b);
    if (d.N < 1 || d.K < 1 || d.group < 1) bad("d", "not a descriptor of 4-bit weights");
    return d;
  }
  double number(int i) {
    if (!ok) return 0.0;
    const double v = PyFloat_AsDouble(a[i]);
    if (v == -1.0 && PyErr_Occurred()) ok = false;
    return v;
  }
  int whole(int i) {
    if (!ok) return 0;
    const long v = PyLong_AsLong(a[i]);
    if (v == -1 && PyErr_Occurred()) ok = false;
    else if (v != (long)(int)v) { PyErr_SetString(PyExc_OverflowError, "argument out of int range"); ok = false; }
    return (int)v;
  }
  // None: the current stream of the tensors' device
  void *stream(int i) {
    if (!ok) return nullptr;
    if (none(i)) return (void *)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
    Args s(a + i, 1, 1);
    void *p = s.stream();
    ok = s.ok;
    return p;
  }
  // The call, without the GIL, with the tensors' device current.
  template <class F>
  PyObject *run(F &&call) {
    if (!ok) return nullptr;
    xnor_status s;
    {
      std::optional<c10::cuda::CUDAGuard> guard;
      if (c10::cuda::device_count() > 1) guard.emplace((c10::DeviceIndex)device);
      Py_BEGIN_ALLOW_THREADS
      s = call();
      Py_END_ALLOW_THREADS
    }
    return PyLong_FromLong((long)s);
  }
};

// What xnor_rmsnorm and xnor_rmsnorm_quant read: x, residual, weight, and the optional sum and rstd.
struct NormIn {
  xnor_norm_desc d = {};
  Dense x, residual, weight, sum, rstd;
  NormIn(RowArgs &A, int sum_at, int rstd_at) {
    x = A.rows(0, "x", &d.x_stride);
    if (!A.ok) return;
    if (!A.none(1)) residual = A.like(1, "residual", x, &d.residual_stride);
    norm_weight(A, 2, x, &weight, &d);
    d.eps = (float)A.number(3);
    if (A.ok && !A.none(sum_at)) sum = A.like(sum_at, "sum", x, &d.sum_stride);
    if (A.ok && !A.none(rstd_at)) rstd = A.dense(rstd_at, "rstd", at::kFloat, {x.size[0]});
    if (!A.ok) return;
    d.rows = (int)x.size[0];
    d.cols = (int)x.size[1];
  }
  static void norm_weight(RowArgs &A, int i, const Dense &x, Dense *weight, xnor_norm_desc *d) {
    d->type = A.xnor_type_of(x, "x", false);
    d->weight_type = XNOR_F32;
    if (!A.ok || A.none(i)) return;
    *weight = A.tensor(i, "weight");
    if (!A.ok) return;
    *weight = A.dense(i, "weight", weight->type == x.type ? (at::ScalarType)x.type : at::kFloat, {x.size[1]});
    if (A.ok) d->weight_type = A.xnor_type_of(*weight, "weight", false);
  }
};

XNOR_PY(rmsnorm) {                   // x, residual, weight, eps, sum, y, rstd, stream
  RowArgs A(args, nargs, 8);
  if (!A.ok) return nullptr;
  NormIn in(A, 4, 6);
  const Dense y = A.like(5, "y", in.x, &in.d.y_stride);
  void *st = A.stream(7);
  return A.run([&] { return E.rmsnorm(in.x.p, in.residual.p, in.weight.p, &in.d, in.sum.p, y.p, (float *)in.rstd.p, st); });
}

XNOR_PY(rmsnorm_quant) {             // x, residual, weight, eps, group, sum, q, scales, rstd, stream
  RowArgs A(args, nargs, 10);
  if (!A.ok) return nullptr;
  NormIn in(A, 5, 8);
  const int group = A.whole(4);
  if (!A.ok) return nullptr;
  Dense q = A.tensor(6, "q");
  const int type = A.ok ? A.xnor_type_of(q, "q", true) : 0;
  if (A.ok && type != XNOR_I8 && type != XNOR_E4M3) A.bad("q", "expected 8-bit values (int8 or float8_e4m3fn)");
  if (A.ok) q = A.dense(6, "q", (at::ScalarType)q.type, {in.x.size[0], in.x.size[1]});
  const Dense s = A.dense(7, "scales", at::kFloat, {in.x.size[0], group > 0 ? in.x.size[1] / group : 1});
  void *st = A.stream(9);
  return A.run([&] { return E.rmsnorm_quant(in.x.p, in.residual.p, in.weight.p, &in.d, type, group, in.sum.p, q.p, (float *)s.p, (float *)in.rstd.p, st); });
}

XNOR_PY(rmsnorm_backward) {          // dy, dsum, h, weight, rstd, dx, dweight, work, stream
  RowArgs A(args, nargs, 9);
  if (!A.ok) return nullptr;
  xnor_norm_desc d = {};
  const Dense dy = A.rows(0, "dy", &d.y_stride);
  if (!A.ok) return nullptr;
  Dense dsum, weight, dweight, work;
  if (!A.none(1)) dsum = A.like(1, "dsum", dy, &d.residual_stride);
  const Dense h = A.like(2, "h", dy, &d.x_stride);
  NormIn::norm_weight(A, 3, dy, &weight, &d);
  const Dense rstd = A.dense(4, "rstd", at::kFloat, {dy.size[0]});
  const Dense dx = A.like(5, "dx", dy, &d.sum_stride);
  if (A.ok && !A.none(6)) {
    dweight = A.dense(6, "dweight", at::kFloat, {dy.size[1]});
    if (A.ok && !A.none(7)) {
      work = A.tensor(7, "work");
      if (A.ok) work = A.dense(7, "work", at::kFloat, {work.numel});
      if (A.ok && work.numel < (long long)xnor_work_elems((int)dy.size[0], (int)dy.size[1])) A.bad("work", "too few elements");
    }
  }
  d.rows = (int)dy.size[0];
  d.cols = (int)dy.size[1];
  void *st = A.stream(8);
  return A.run([&] { return E.rmsnorm_backward(dy.p, dsum.p, h.p, weight.p, (const float *)rstd.p, &d, dx.p, (float *)dweight.p, (float *)work.p, st); });
}

// Packed codes, scales and optional zero points of the matrix d.
struct W4In {
  Dense packed, scales, zeros;
  W4In(RowArgs &A, const xnor_w4_desc &d, int packed_at, int scales_at, int zeros_at) {
    if (!A.ok) return;
    const long long G = (d.K + (long long)d.group - 1) / d.group;
    packed = A.dense(packed_at, "w_packed", at::kInt, {(d.N + 127ll) / 128, (d.K + 63ll) / 64, 256, 4});
    if (scales_at >= 0) scales = A.dense(scales_at, "scales", at::kFloat, {G, d.N});
    if (zeros_at >= 0 && A.ok && !A.none(zeros_at)) zeros = A.dense(zeros_at, "zeros", at::kByte, {G, d.N});
  }
};

XNOR_PY(w4_quantize) {               // w, d, w_packed, scales, zeros, stream
  RowArgs A(args, nargs, 6);
  if (!A.ok) return nullptr;
  const xnor_w4_desc d = A.w4(1);
  Dense w = A.tensor(0, "w");
  const int type = A.ok ? A.xnor_type_of(w, "w", false) : 0;
  if (A.ok) w = A.dense(0, "w", (at::ScalarType)w.type, {d.N, d.K});
  const W4In in(A, d, 2, 3, 4);
  void *st = A.stream(5);
  return A.run([&] { return E.w4_quantize(w.p, type, &d, (uint32_t *)in.packed.p, (float *)in.scales.p, (uint8_t *)in.zeros.p, st); });
}

XNOR_PY(w4_pack) {                   // codes, d, w_packed, stream
  RowArgs A(args, nargs, 4);
  if (!A.ok) return nullptr;
  const xnor_w4_desc d = A.w4(1);
  const Dense c = A.dense(0, "codes", at::kByte, {d.N, d.K});
  const W4In in(A, d, 2, -1, -1);
  void *st = A.stream(3);
  return A.run([&] { return E.w4_pack((const uint8_t *)c.p, &d, (uint32_t *)in.packed.p, st); });
}

XNOR_PY(w4_dequantize) {             // w_packed, scales, zeros, d, w, stream
  RowArgs A(args, nargs, 6);
  if (!A.ok) return nullptr;
  const xnor_w4_desc d = A.w4(3);
  const W4In in(A, d, 0, 1, 2);
  Dense w = A.tensor(4, "w");
  const int type = A.ok ? A.xnor_type_of(w, "w", false) : 0;
  if (A.ok) w = A.dense(4, "w", (at::ScalarType)w.type, {d.N, d.K});
  void *st = A.stream(5);
  return A.run([&] { return E.w4_dequantize((const uint32_t *)in.packed.p, (const float *)in.scales.p, (const uint8_t *)in.zeros.p, &d, type, w.p, st); });
}

XNOR_PY(w4_matmul) {                 // x, x_scales, w_packed, scales, zeros, d, out, stream
  RowArgs A(args, nargs, 8);
  if (!A.ok) return nullptr;
  const xnor_w4_desc d = A.w4(5);
  xnor_w4_rows r = {};
  const Dense x = A.rows(0, "x", &r.x_stride);
  if (A.ok && x.size[1] != d.K) A.bad("x", "as many columns as the weights' K are expected");
  const W4In in(A, d, 2, 3, 4);
  const Dense out = A.rows(6, "out", &r.out_stride);
  if (A.ok && (out.size[0] != x.size[0] || out.size[1] != d.N)) A.bad("out", "wrong shape");
  if (!A.ok) return nullptr;
  r.rows = (int)x.size[0];
  r.x_type = A.xnor_type_of(x, "x", true);
  r.out_type = A.xnor_type_of(out, "out", false);
  Dense xs;
  if (A.ok && !A.none(1)) {
    const long long G = (d.K + (long long)d.group - 1) / d.group;
    xs = A.tensor(1, "x_scales");
    // [rows][1]: a scale for each row; [rows][groups]: for each group (the same where there is one group)
    r.x_group = A.ok && xs.dims == 2 && xs.size[1] > 1 ? d.group : 0;
    if (A.ok) xs = A.dense(1, "x_scales", at::kFloat, {x.size[0], r.x_group ? G : 1});
  }
  void *st = A.stream(7);
  return A.run([&] { return E.w4_matmul(x.p, (const float *)xs.p, (const uint32_t *)in.packed.p, (const float *)in.scales.p, (const uint8_t *)in.zeros.p, &d, &r, out.p, st); });
}

// describe(class, function, address): the descriptor of 4-bit weights, the Python description of what is not exactly
// a tensor, and xnor_rmsnorm_work_elems
PyObject *describe(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  if (nargs != 3) return PyErr_Format(PyExc_TypeError, "expected 3 arguments, got %zd", nargs);
  void *p = PyLong_AsVoidPtr(args[2]);
  if (p == nullptr) { if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null address"); return nullptr; }
  xnor_work_elems = (decltype(&xnor_rmsnorm_work_elems))p;
  Py_XSETREF(w4_desc_type, Py_NewRef(args[0]));
  Py_XSETREF(py_describe, Py_NewRef(args[1]));
  Py_RETURN_NONE;
}

// bind(addresses, descriptor, address): the entry points' addresses, in the order of struct Entry, the
// descriptor's class, and the Python conversion of what is not exactly a tensor
PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
  if (nargs != 3) return PyErr_Format(PyExc_TypeError, "expected 3 arguments, got %zd", nargs);
  PyObject *t = PySequence_Tuple(args[0]);
  if (t == nullptr) return nullptr;
  void *p[kEntries];
  bool ok = PyTuple_GET_SIZE(t) == kEntries;
  if (!ok) PyErr_Format(PyExc_ValueError, "expected %zd addresses", kEntries);
  for (Py_ssize_t i = 0; ok && i < kEntries; ++i) {
    p[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(t, i));
    if (p[i] == nullptr) { ok = false; if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null address"); }
  }
  Py_DECREF(t);
  if (!ok) return nullptr;
  memcpy((void *)&E, p, sizeof(E));
  Py_XSETREF(desc_type, Py_NewRef(args[1]));
  Py_XSETREF(py_address, Py_NewRef(args[2]));
  Py_RETURN_NONE;
}

#define XNOR_FAST(name) {#name, (PyCFunction)(void (*)(void))entry<name>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, nullptr},
    XNOR_FAST(binarize_weights), XNOR_FAST(binactiv), XNOR_FAST(conv2d_forward), XNOR_FAST(shortcut_conv1x1),
    XNOR_FAST(conv2d_forward_binactiv), XNOR_FAST(binactiv_finish), XNOR_FAST(maxpool2d), XNOR_FAST(binactiv_kbit),
    XNOR_FAST(conv2d_forward_kbit), XNOR_FAST(bwn_prepare_input), XNOR_FAST(bwn_conv2d_forward),
    XNOR_FAST(binarize_weights_transposed), XNOR_FAST(binary_gradient_backward),
    {"describe", (PyCFunction)(void (*)(void))describe, METH_FASTCALL, nullptr},
    XNOR_FAST(rmsnorm), XNOR_FAST(rmsnorm_quant), XNOR_FAST(rmsnorm_backward), XNOR_FAST(w4_quantize), XNOR_FAST(w4_pack),
    XNOR_FAST(w4_dequantize), XNOR_FAST(w4_matmul),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pymarshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pymarshal(void) { return PyModule_Create(&module); }
