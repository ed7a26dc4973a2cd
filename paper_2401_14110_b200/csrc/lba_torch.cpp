// Calls of the C ABI straight from PyTorch tensors: the regular call of binding.py's entry points in one native function each.
//
// A call through ctypes spends 10 to 12 us of host time on checks, conversions and torch.empty, as long as the kernels of
// small problems run.  Here the same checks, the output's allocation and the call take about 4.  Every function returns None for
// anything that is not the regular case -- a tensor of another type, device or layout, an explicit stream, formats of other
// types, an active torch-function or dispatch mode, an exception -- and has then done nothing that a caller can see: binding.py
// goes on as it would without this module, and raises what it raises.  A status other than 0 is returned as an integer.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/ops/empty.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <cmath>
#include <optional>

#include "lba.h"

namespace {

PyObject* g_format_type = nullptr;     // formats.LbaFormat
PyObject* g_parameter_type = nullptr;  // torch.nn.Parameter: a tensor like any other here, as weights, scales and biases often are
PyObject* g_field[5];               // its attribute names, interned

struct NotRegular {};

[[noreturn]] void not_regular() { throw NotRegular(); }

int as_int(PyObject* o) {
  if (!PyLong_CheckExact(o)) not_regular();
  int overflow = 0;
  const long v = PyLong_AsLongAndOverflow(o, &overflow);
  if (overflow || v < INT_MIN || v > INT_MAX) not_regular();
  return (int)v;
}

lba_fmt as_format(PyObject* o) {
  int32_t v[5];
  if (Py_TYPE(o) == (PyTypeObject*)g_format_type) {
    for (int i = 0; i < 5; ++i) {
      PyObject* const a = PyObject_GetAttr(o, g_field[i]);
      if (!a) {
        PyErr_Clear();
        not_regular();
      }
      const bool plain = PyLong_CheckExact(a);
      int overflow = 0;
      const long x = plain ? PyLong_AsLongAndOverflow(a, &overflow) : 0;
      Py_DECREF(a);
      if (!plain || overflow || x < INT_MIN || x > INT_MAX) not_regular();
      v[i] = (int32_t)x;
    }
  } else if (PyTuple_CheckExact(o) && PyTuple_GET_SIZE(o) == 5) {
    for (int i = 0; i < 5; ++i) v[i] = as_int(PyTuple_GET_ITEM(o, i));
  } else {
    not_regular();
  }
  lba_fmt f;
  f.man_bits = v[0];
  f.exp_bits = v[1];
  f.bias = v[2];
  f.rounding = v[3];
  f.flags = v[4];
  return f;
}

// a contiguous tensor of `dtype` on the current device
const at::Tensor& as_tensor(PyObject* o, c10::ScalarType dtype, int dim, int device) {
  if (Py_TYPE(o) != (PyTypeObject*)THPVariableClass && Py_TYPE(o) != (PyTypeObject*)g_parameter_type) not_regular();  // no other subclass
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.get_device() != device || t.scalar_type() != dtype || !t.is_contiguous() ||
      (dim >= 0 && t.dim() != dim))
    not_regular();
  return t;
}

void pair_of(PyObject* o, int (&v)[2]) {
  if (!PyTuple_CheckExact(o) || PyTuple_GET_SIZE(o) != 2) not_regular();
  v[0] = as_int(PyTuple_GET_ITEM(o, 0));
  v[1] = as_int(PyTuple_GET_ITEM(o, 1));
}

struct Call {
  int device;
  void* stream;
  explicit Call(PyObject* stream_arg) {
    if (stream_arg != Py_None || at::impl::PythonTorchFunctionTLS::stack_len() > 0 || c10::impl::TorchDispatchModeTLS::any_modes_set())
      not_regular();
    device = c10::cuda::current_device();
    stream = (void*)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
  }
  at::Tensor fresh(at::IntArrayRef sizes, c10::ScalarType dtype) const {
    return at::empty(sizes, at::TensorOptions().dtype(dtype).device(c10::Device(c10::kCUDA, (c10::DeviceIndex)device)));
  }
};

// scales and bias, as every forward entry point takes them
struct Scales {
  const float *a, *b, *bias;
  int a_len, b_len;
  Scales(PyObject* sa, PyObject* sb, PyObject* bi, int device) {
    const at::Tensor &ta = as_tensor(sa, at::kFloat, -1, device), &tb = as_tensor(sb, at::kFloat, -1, device);
    if (ta.numel() > INT_MAX || tb.numel() > INT_MAX) not_regular();
    a = (const float*)ta.data_ptr();
    b = (const float*)tb.data_ptr();
    a_len = (int)ta.numel();
    b_len = (int)tb.numel();
    bias = bi == Py_None ? nullptr : (const float*)as_tensor(bi, at::kFloat, -1, device).data_ptr();
  }
};

// the output a caller passed, or a new one
at::Tensor output(PyObject* out, const Call& call, at::IntArrayRef sizes, c10::ScalarType dtype) {
  return out == Py_None ? call.fresh(sizes, dtype) : as_tensor(out, dtype, -1, call.device);
}

PyObject* result(int status, PyObject* given, const at::Tensor& out) {
  if (status != 0) return PyLong_FromLong(status);
  if (given != Py_None) return Py_NewRef(given);
  return THPVariable_Wrap(out);
}

template <typename F>
int without_gil(F f) {
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = f();
  Py_END_ALLOW_THREADS
  return status;
}

template <typename F>
PyObject* regular_or_none(Py_ssize_t n, Py_ssize_t want, F f) {
  if (n != want) Py_RETURN_NONE;
  try {
    return f();
  } catch (...) {  // NotRegular, or an error that the caller's own path runs into and reports
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// A, B, scale_a, scale_b, bias, prod_fmt, acc_fmt, order, chunk, out, stream
PyObject* gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return regular_or_none(n, 11, [&]() -> PyObject* {
    const Call call(a[10]);
    const at::Tensor &A = as_tensor(a[0], at::kByte, 2, call.device), &B = as_tensor(a[1], at::kByte, 2, call.device);
    const int64_t M = A.size(0), N = B.size(0), K = A.size(1);
    if (B.size(1) != K) not_regular();
    const Scales s(a[2], a[3], a[4], call.device);
    const lba_fmt pf = as_format(a[5]), af = as_format(a[6]);
    const int order = as_int(a[7]), chunk = as_int(a[8]);
    const at::Tensor out = output(a[9], call, {M, N}, at::kFloat);
    const uint8_t *const pa = (const uint8_t*)A.data_ptr(), *const pb = (const uint8_t*)B.data_ptr();
    float* const po = (float*)out.data_ptr();
    return result(without_gil([&] {
                    return lba_gemm(pa, pb, s.a, s.a_len, s.b, s.b_len, s.bias, M, N, K, &pf, &af, order, chunk, po, call.stream);
                  }), a[9], out);
  });
}

// the same with A [Z][M][K], B [Z][N][K] or [N][K]
PyObject* gemm_batched(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return regular_or_none(n, 11, [&]() -> PyObject* {
    const Call call(a[10]);
    const at::Tensor &A = as_tensor(a[0], at::kByte, 3, call.device), &B = as_tensor(a[1], at::kByte, -1, call.device);
    const int64_t Z = A.size(0), M = A.size(1), K = A.size(2);
    const bool shared = B.dim() == 2;
    if (!shared && (B.dim() != 3 || B.size(0) != Z)) not_regular();
    const int64_t N = B.size(shared ? 0 : 1);
    if (B.size(shared ? 1 : 2) != K) not_regular();
    const Scales s(a[2], a[3], a[4], call.device);
    const lba_fmt pf = as_format(a[5]), af = as_format(a[6]);
    const int order = as_int(a[7]), chunk = as_int(a[8]);
    const at::Tensor out = output(a[9], call, {Z, M, N}, at::kFloat);
    const uint8_t *const pa = (const uint8_t*)A.data_ptr(), *const pb = (const uint8_t*)B.data_ptr();
    float* const po = (float*)out.data_ptr();
    return result(without_gil([&] {
                    return lba_gemm_batched(pa, pb, s.a, s.a_len, s.b, s.b_len, s.bias, Z, M, N, K, M * K, shared ? 0 : N * K, M * N, &pf,
                                            &af, order, chunk, po, call.stream);
                  }), a[9], out);
  });
}

// x, w, scale_x, scale_w, bias, stride, pad, prod_fmt, acc_fmt, order, chunk, out, stream
PyObject* conv2d(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return regular_or_none(n, 13, [&]() -> PyObject* {
    const Call call(a[12]);
    const at::Tensor &x = as_tensor(a[0], at::kByte, 4, call.device), &w = as_tensor(a[1], at::kByte, 4, call.device);
    int64_t d[7] = {x.size(0), x.size(1), x.size(2), x.size(3), w.size(0), w.size(1), w.size(2)};
    int stride[2], pad[2];
    pair_of(a[5], stride);
    pair_of(a[6], pad);
    if (w.size(3) != d[3] || stride[0] < 1 || stride[1] < 1 || pad[0] < 0 || pad[1] < 0) not_regular();
    for (int64_t v : d)
      if (v < 1 || v > INT_MAX / 4) not_regular();
    if (pad[0] > INT_MAX / 4 || pad[1] > INT_MAX / 4) not_regular();
    const int64_t h = d[1] + 2 * (int64_t)pad[0] - d[5], v = d[2] + 2 * (int64_t)pad[1] - d[6];
    if (h < 0 || v < 0) not_regular();
    const Scales s(a[2], a[3], a[4], call.device);
    const lba_fmt pf = as_format(a[7]), af = as_format(a[8]);
    const int order = as_int(a[9]), chunk = as_int(a[10]);
    const at::Tensor out = output(a[11], call, {d[0], h / stride[0] + 1, v / stride[1] + 1, d[4]}, at::kFloat);
    const uint8_t *const px = (const uint8_t*)x.data_ptr(), *const pw = (const uint8_t*)w.data_ptr();
    float* const po = (float*)out.data_ptr();
    return result(without_gil([&] {
                    return lba_conv2d(px, pw, s.a, s.a_len, s.b, s.b_len, s.bias, (int)d[0], (int)d[1], (int)d[2], (int)d[3], (int)d[4],
                                      (int)d[5], (int)d[6], stride[0], stride[1], pad[0], pad[1], &pf, &af, order, chunk, po, call.stream);
                  }), a[11], out);
  });
}

// ------------------------------------------------------------------ layers
int float_type(c10::ScalarType t) {
  switch (t) {
    case at::kFloat: return LBA_TYPE_F32;
    case at::kBFloat16: return LBA_TYPE_BF16;
    case at::kHalf: return LBA_TYPE_F16;
    default: not_regular();
  }
}
c10::ScalarType as_dtype(PyObject* o) {
  if (!THPDtype_Check(o)) not_regular();
  return ((THPDtype*)o)->scalar_type;
}
// a contiguous tensor of 32- or 16-bit floats of these sizes
const at::Tensor& as_floats(PyObject* o, const Call& call, at::IntArrayRef sizes, int* type) {
  if (Py_TYPE(o) != (PyTypeObject*)THPVariableClass && Py_TYPE(o) != (PyTypeObject*)g_parameter_type) not_regular();
  const c10::ScalarType dtype = THPVariable_Unpack(o).scalar_type();
  *type = float_type(dtype);
  const at::Tensor& t = as_tensor(o, dtype, -1, call.device);
  if (t.sizes() != sizes) not_regular();
  return t;
}
int as_activation(PyObject* o) {
  static const char* const names[5] = {"none", "relu", "gelu", "gelu_tanh", "silu"};
  if (!PyUnicode_CheckExact(o)) not_regular();
  for (int i = 0; i < 5; ++i)
    if (PyUnicode_CompareWithASCIIString(o, names[i]) == 0) return i;
  not_regular();
}
double as_real(PyObject* o) {
  if (PyFloat_CheckExact(o)) return PyFloat_AS_DOUBLE(o);
  return as_int(o);
}
const uint64_t* as_rng(PyObject* o, double dropout, int device) {
  if (dropout == 0.0) return nullptr;
  const at::Tensor& t = as_tensor(o, at::kLong, -1, device);
  if (t.numel() != 2) not_regular();
  return (const uint64_t*)t.data_ptr();
}
const float* as_vector(PyObject* o, int64_t n, int device) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = as_tensor(o, at::kFloat, 1, device);
  if (t.size(0) != n) not_regular();
  return (const float*)t.data_ptr();
}

// output, pre-activations and the C struct of a forward layer call; arguments as binding._layer takes them
struct Layer {
  at::Tensor out, pre;
  bool fresh_pre = false;
  lba_layer l = {};
  Layer(const Call& call, at::IntArrayRef sizes, at::IntArrayRef pre_sizes, PyObject* activation, PyObject* out_dtype, PyObject* out_scale,
        PyObject* preact, PyObject* given) {
    l.activation = as_activation(activation);
    c10::ScalarType dtype;
    if (given == Py_None) {
      dtype = as_dtype(out_dtype);
    } else {
      if (Py_TYPE(given) != (PyTypeObject*)THPVariableClass) not_regular();
      dtype = THPVariable_Unpack(given).scalar_type();
    }
    l.out_type = dtype == at::kByte ? (int)LBA_TYPE_CODES : float_type(dtype);
    if (dtype == at::kByte) {
      const at::Tensor& s = as_tensor(out_scale, at::kFloat, -1, call.device);
      if (s.numel() != 1) not_regular();
      l.out_scale = (const float*)s.data_ptr();
    }
    int type = 0;
    if (preact != Py_None) {
      if (THPDtype_Check(preact)) {
        type = float_type(as_dtype(preact));
      } else {
        pre = as_floats(preact, call, pre_sizes, &type);
      }
    }
    if (given == Py_None) {
      out = call.fresh(sizes, dtype);
    } else {
      out = as_tensor(given, dtype, -1, call.device);
      if (out.sizes() != sizes) not_regular();
    }
    if (preact != Py_None && !pre.defined()) {
      pre = call.fresh(pre_sizes, as_dtype(preact));
      fresh_pre = true;
    }
    if (pre.defined()) l.preact = pre.data_ptr();
    l.preact_type = type;
  }
  PyObject* result(int status, PyObject* preact, PyObject* given) const {
    if (status != 0) return PyLong_FromLong(status);
    PyObject* const o = given != Py_None ? Py_NewRef(given) : THPVariable_Wrap(out);
    if (!pre.defined() || !o) return o;
    PyObject* const q = fresh_pre ? THPVariable_Wrap(pre) : Py_NewRef(preact);
    if (!q) {
      Py_DECREF(o);
      return nullptr;
    }
    PyObject* const both = PyTuple_Pack(2, o, q);
    Py_DECREF(o);
    Py_DECREF(q);
    return both;
  }
};

// A, B, scale_a, scale_b, bias, prod_fmt, acc_fmt, order, chunk, activation, residual, dropout, rng, out_dtype, out_scale, preact, out, stream
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return regular_or_none(n, 18, [&]() -> PyObject* {
    const Call call(a[17]);
    const at::Tensor &A = as_tensor(a[0], at::kByte, 2, call.device), &B = as_tensor(a[1], at::kByte, 2, call.device);
    const int64_t M = A.size(0), N = B.size(0), K = A.size(1);
    if (B.size(1) != K) not_regular();
    const Scales s(a[2], a[3], Py_None, call.device);
    const float* const bias = as_vector(a[4], N, call.device);
    const lba_fmt pf = as_format(a[5]), af = as_format(a[6]);
    const int order = as_int(a[7]), chunk = as_int(a[8]);
    const double dropout = as_real(a[11]);
    const uint64_t* const rng = as_rng(a[12], dropout, call.device);
    int res_type = 0;
    const void* const residual = a[10] == Py_None ? nullptr : as_floats(a[10], call, {M, N}, &res_type).data_ptr();
    Layer y(call, {M, N}, {M, N}, a[9], a[13], a[14], a[15], a[16]);
    y.l.residual = residual;
    y.l.residual_type = res_type;
    y.l.dropout = dropout;
    y.l.rng = rng;
    const uint8_t *const pa = (const uint8_t*)A.data_ptr(), *const pb = (const uint8_t*)B.data_ptr();
    void* const po = y.out.data_ptr();
    return y.result(without_gil([&] {
                      return lba_linear(pa, pb, s.a, s.a_len, s.b, s.b_len, bias, M, N, K, &pf, &af, order, chunk, &y.l, po, call.stream);
                    }), a[15], a[16]);
  });
}

// A, B_gate, B_up, scale_a, scale_gate, scale_up, bias_gate, bias_up, prod_fmt, acc_fmt, order, chunk, activation, out_dtype, out_scale,
// preact, out, stream
PyObject* gated(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return regular_or_none(n, 18, [&]() -> PyObject* {
    const Call call(a[17]);
    const at::Tensor &A = as_tensor(a[0], at::kByte, 2, call.device), &G = as_tensor(a[1], at::kByte, 2, call.device),
                     &U = as_tensor(a[2], at::kByte, 2, call.device);
    const int64_t M = A.size(0), N = G.size(0), K = A.size(1);
    if (G.size(1) != K || U.size(0) != N || U.size(1) != K) not_regular();
    const Scales s(a[3], a[4], Py_None, call.device), up(a[3], a[5], Py_None, call.device);
    if (s.b_len != up.b_len) not_regular();
    const float *const bg = as_vector(a[6], N, call.device), *const bu = as_vector(a[7], N, call.device);
    const lba_fmt pf = as_format(a[8]), af = as_format(a[9]);
    const int order = as_int(a[10]), chunk = as_int(a[11]);
    Layer y(call, {M, N}, {2, M, N}, a[12], a[13], a[14], a[15], a[16]);
    const uint8_t *const pa = (const uint8_t*)A.data_ptr(), *const pg = (const uint8_t*)G.data_ptr(), *const pu = (const uint8_t*)U.data_ptr();
    void* const po = y.out.data_ptr();
    return y.result(without_gil([&] {
                      return lba_gated(pa, pg, pu, s.a, s.a_len, s.b, up.b, s.b_len, bg, bu, M, N, K, &pf, &af, order, chunk, &y.l, po, call.stream);
                    }), a[15], a[16]);
  });
}

// what both backward passes share
struct Backward {
  lba_backward h = {};
  const void* grad;
  c10::ScalarType dtype;
  bool needs[3];
  at::Tensor ws;
  Backward(const Call& call, bool gated, int64_t M, int64_t N, int64_t K, const Scales& s, PyObject* grad_out, PyObject* prod_fmt, PyObject* preact,
           PyObject* activation, double dropout, const uint64_t* rng, PyObject* grad_dtype, PyObject* need, PyObject* workspace) {
    int type = 0;
    const at::Tensor& g = as_floats(grad_out, call, {M, N}, &type);
    grad = g.data_ptr();
    h.grad_type = type;
    dtype = grad_dtype == Py_None ? g.scalar_type() : as_dtype(grad_dtype);
    h.out_type = float_type(dtype);
    h.activation = as_activation(activation);
    type = 0;
    if (preact != Py_None) {
      h.preact = gated ? as_floats(preact, call, {2, M, N}, &type).data_ptr() : as_floats(preact, call, {M, N}, &type).data_ptr();
    }
    h.preact_type = type;
    h.dropout = dropout;
    h.rng = rng;
    h.input_flags = as_format(prod_fmt).flags & LBA_FLAG_INPUT_M4E3;
    if (!PyTuple_CheckExact(need) || PyTuple_GET_SIZE(need) != 3) not_regular();
    int mask = 0;
    for (int i = 0; i < 3; ++i) {
      PyObject* const o = PyTuple_GET_ITEM(need, i);
      if (!PyBool_Check(o)) not_regular();
      needs[i] = o == Py_True;
      mask |= needs[i] << i;
    }
    if (workspace != Py_None) {
      ws = as_tensor(workspace, at::kByte, -1, call.device);
    } else {
      ws = call.fresh({(int64_t)lba_backward_workspace_bytes(gated, M, N, K, s.a_len, s.b_len, &h, mask)}, at::kByte);
    }
  }
  at::Tensor fresh(const Call& call, int need, at::IntArrayRef sizes, c10::ScalarType t) const { return needs[need] ? call.fresh(sizes, t) : at::Tensor(); }
};
template <typename T = void>
T* pointer(const at::Tensor& t) {
  return t.defined() ? (T*)t.data_ptr() : nullptr;
}
PyObject* results(int status, std::initializer_list<at::Tensor> outs) {
  if (status != 0) return PyLong_FromLong(status);
  PyObject* const all = PyTuple_New((Py_ssize_t)outs.size());
  if (!all) return nullptr;
  Py_ssize_t i = 0;
  for (const at::Tensor& t : outs) {
    PyObject* const o = t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None);
    if (!o) {
      Py_DECREF(all);
      return nullptr;
    }
    PyTuple_SET_ITEM(all, i++, o);
  }
  return all;
}

// grad_out, A, B, scale_a, scale_b, prod_fmt, preact, activation, dropout, rng, grad_dtype, needs, workspace, stream
PyObject* linear_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return regular_or_none(n, 14, [&]() -> PyObject* {
    const Call call(a[13]);
    const at::Tensor &A = as_tensor(a[1], at::kByte, 2, call.device), &B = as_tensor(a[2], at::kByte, 2, call.device);
    const int64_t M = A.size(0), N = B.size(0), K = A.size(1);
    if (B.size(1) != K) not_regular();
    const Scales s(a[3], a[4], Py_None, call.device);
    const double dropout = as_real(a[8]);
    const Backward b(call, false, M, N, K, s, a[0], a[5], a[6], a[7], dropout, as_rng(a[9], dropout, call.device), a[10], a[11], a[12]);
    const at::Tensor ga = b.fresh(call, 0, {M, K}, b.dtype), gb = b.fresh(call, 1, {N, K}, b.dtype), gc = b.fresh(call, 2, {N}, at::kFloat);
    const uint8_t *const pa = (const uint8_t*)A.data_ptr(), *const pb = (const uint8_t*)B.data_ptr();
    return results(without_gil([&] {
                     return lba_linear_backward(b.grad, pa, pb, s.a, s.a_len, s.b, s.b_len, M, N, K, &b.h, pointer(ga), pointer(gb),
                                                pointer<float>(gc), b.ws.data_ptr(), b.ws.numel(), call.stream);
                   }), {ga, gb, gc});
  });
}

// grad_out, A, B_gate, B_up, scale_a, scale_gate, scale_up, prod_fmt, preact, activation, grad_dtype, needs, workspace, stream
PyObject* gated_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return regular_or_none(n, 14, [&]() -> PyObject* {
    const Call call(a[13]);
    const at::Tensor &A = as_tensor(a[1], at::kByte, 2, call.device), &G = as_tensor(a[2], at::kByte, 2, call.device),
                     &U = as_tensor(a[3], at::kByte, 2, call.device);
    const int64_t M = A.size(0), N = G.size(0), K = A.size(1);
    if (G.size(1) != K || U.size(0) != N || U.size(1) != K) not_regular();
    const Scales s(a[4], a[5], Py_None, call.device), up(a[4], a[6], Py_None, call.device);
    if (s.b_len != up.b_len) not_regular();
    const Backward b(call, true, M, N, K, s, a[0], a[7], a[8], a[9], 0.0, nullptr, a[10], a[11], a[12]);
    const at::Tensor ga = b.fresh(call, 0, {M, K}, b.dtype), gg = b.fresh(call, 1, {N, K}, b.dtype), gu = b.fresh(call, 1, {N, K}, b.dtype),
                     cg = b.fresh(call, 2, {N}, at::kFloat), cu = b.fresh(call, 2, {N}, at::kFloat);
    const uint8_t *const pa = (const uint8_t*)A.data_ptr(), *const pg = (const uint8_t*)G.data_ptr(), *const pu = (const uint8_t*)U.data_ptr();
    return results(without_gil([&] {
                     return lba_gated_backward(b.grad, pa, pg, pu, s.a, s.a_len, s.b, up.b, s.b_len, M, N, K, &b.h, pointer(ga), pointer(gg),
                                               pointer(gu), pointer<float>(cg), pointer<float>(cu), b.ws.data_ptr(), b.ws.numel(), call.stream);
                   }), {ga, gg, gu, cg, cu});
  });
}

// ------------------------------------------------------------------ between the linear layers
bool as_bool(PyObject* o) {
  if (!PyBool_Check(o)) not_regular();
  return o == Py_True;
}
// a tensor [rows][heads][dim] of this type whose heads' values are contiguous
struct Heads {
  const at::Tensor& t;
  lba_strides at;
  void* data;
  static const at::Tensor& checked(PyObject* o, const Call& call) {
    if (Py_TYPE(o) != (PyTypeObject*)THPVariableClass && Py_TYPE(o) != (PyTypeObject*)g_parameter_type) not_regular();
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.get_device() != call.device || t.dim() != 3 || t.layout() != at::kStrided || (t.size(2) > 1 && t.stride(2) != 1))
      not_regular();
    return t;
  }
  Heads(PyObject* o, const Call& call) : t(checked(o, call)), at{t.stride(0), t.stride(1)}, data(t.data_ptr()) {}
};
// int32 values, n of them; None: null
const int32_t* as_ints(PyObject* o, int64_t n, int device) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = as_tensor(o, at::kInt, -1, device);
  if (t.numel() != n) not_regular();
  return (const int32_t*)t.data_ptr();
}
int half_type(c10::ScalarType t) {
  if (t != at::kBFloat16 && t != at::kHalf) not_regular();
  return float_type(t);
}
int as_size(int64_t v) {
  if (v > INT_MAX) not_regular();
  return (int)v;
}
at::Tensor given_or_fresh(PyObject* o, const Call& call, at::IntArrayRef sizes, c10::ScalarType dtype) {
  if (o == Py_None) return call.fresh(sizes, dtype);
  const at::Tensor& t = as_tensor(o, dtype, -1, call.device);
  if (t.sizes() != sizes) not_regular();
  return t;
}
PyObject* wrapped(PyObject* given, const at::Tensor& t) { return given == Py_None ? THPVariable_Wrap(t) : Py_NewRef(given); }
PyObject* both_of(PyObject* a, PyObject* b) {  // takes both references, which may be null with a Python error set
  PyObject* const r = a && b ? PyTuple_Pack(2, a, b) : nullptr;
  Py_XDECREF(a);
  Py_XDECREF(b);
  return r;
}

// q, k, positions, freqs, interleaved, inverse, scale, out, stream
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return regular_or_none(n, 9, [&]() -> PyObject* {
    const Call call(a[8]);
    const Heads q(a[0], call);
    const bool has_k = a[1] != Py_None;
    const std::optional<Heads> k = has_k ? std::optional<Heads>(std::in_place, a[1], call) : std::nullopt;
    const c10::ScalarType dtype = q.t.scalar_type();
    lba_rotary_how how = {};
    how.type = float_type(dtype);
    if (has_k && (k->t.scalar_type() != dtype || k->t.size(0) != q.t.size(0) || k->t.size(2) != q.t.size(2))) not_regular();
    if (Py_TYPE(a[2]) != (PyTypeObject*)THPVariableClass) not_regular();
    const c10::ScalarType pt = THPVariable_Unpack(a[2]).scalar_type();
    if (pt != at::kInt && pt != at::kLong) not_regular();
    const at::Tensor &pos = as_tensor(a[2], pt, -1, call.device), &freqs = as_tensor(a[3], at::kDouble, -1, call.device);
    if (pos.numel() != q.t.size(0)) not_regular();
    how.heads = as_size(q.t.size(1));
    how.kv_heads = has_k ? as_size(k->t.size(1)) : 0;
    how.dim = as_size(q.t.size(2));
    how.rotary_dim = as_size(2 * freqs.numel());
    how.interleaved = as_bool(a[4]);
    how.inverse = as_bool(a[5]);
    how.wide_positions = pt == at::kLong;
    how.scale = (float)as_real(a[6]);
    how.tokens = q.t.size(0);
    how.positions = pos.data_ptr();
    how.freqs = (const double*)freqs.data_ptr();
    PyObject *go = Py_None, *gk = Py_None;
    if (a[7] != Py_None) {
      if (!PyTuple_CheckExact(a[7]) || PyTuple_GET_SIZE(a[7]) != 2) not_regular();
      go = PyTuple_GET_ITEM(a[7], 0);
      gk = PyTuple_GET_ITEM(a[7], 1);
    }
    const at::Tensor qo = go == Py_None ? call.fresh(q.t.sizes(), dtype) : Heads(go, call).t;
    const at::Tensor ko = !has_k ? at::Tensor() : gk == Py_None ? call.fresh(k->t.sizes(), dtype) : Heads(gk, call).t;
    if (qo.scalar_type() != dtype || qo.sizes() != q.t.sizes() || (has_k && (ko.scalar_type() != dtype || ko.sizes() != k->t.sizes()))) not_regular();
    const lba_strides none = {0, 0}, qo_at = {qo.stride(0), qo.stride(1)}, ko_at = has_k ? lba_strides{ko.stride(0), ko.stride(1)} : none;
    const lba_strides k_at = has_k ? k->at : none;
    const void* const pk = has_k ? k->data : nullptr;
    void *const po = qo.data_ptr(), *const pko = has_k ? ko.data_ptr() : nullptr;
    const int status = without_gil([&] { return lba_rotary(q.data, q.at, pk, k_at, &how, po, qo_at, pko, ko_at, call.stream); });
    if (status != 0) return PyLong_FromLong(status);
    return both_of(wrapped(go, qo), has_k ? wrapped(gk, ko) : Py_NewRef(Py_None));
  });
}

// what both passes share
struct Attention {
  Heads q, k, v;
  lba_attention_how how = {};
  Attention(const Call& call, PyObject* qo, PyObject* ko, PyObject* vo, PyObject* cu_q, PyObject* cu_k, PyObject* causal, PyObject* scale)
      : q(qo, call), k(ko, call), v(vo, call) {
    const c10::ScalarType dtype = q.t.scalar_type();
    how.type = half_type(dtype);
    if (k.t.scalar_type() != dtype || v.t.scalar_type() != dtype || k.t.sizes() != v.t.sizes() || k.t.size(2) != q.t.size(2) ||
        (cu_q == Py_None) != (cu_k == Py_None))
      not_regular();
    how.sequences = 1;
    if (cu_q != Py_None) {
      const at::Tensor& t = as_tensor(cu_q, at::kInt, -1, call.device);
      if (t.numel() < 1) not_regular();
      how.sequences = as_size(t.numel() - 1);
      how.cu_q = (const int32_t*)t.data_ptr();
      how.cu_k = as_ints(cu_k, t.numel(), call.device);
    }
    how.heads = as_size(q.t.size(1));
    how.kv_heads = as_size(k.t.size(1));
    how.dim = as_size(q.t.size(2));
    how.causal = as_bool(causal);
    how.scale = (float)(scale == Py_None ? std::pow((double)how.dim, -0.5) : as_real(scale));
    how.q_rows = q.t.size(0);
    how.k_rows = k.t.size(0);
    how.q_at = q.at;
    how.k_at = k.at;
    how.v_at = v.at;
  }
};
// an attention's output: of the inputs' type, or codes
struct Output {
  at::Tensor out;
  int type, flags = 0;
  const float* scale = nullptr;
  Output(const Call& call, at::IntArrayRef sizes, c10::ScalarType dtype, PyObject* out_dtype, PyObject* out_scale, PyObject* prod_fmt, PyObject* given) {
    c10::ScalarType t = out_dtype == Py_None ? dtype : as_dtype(out_dtype);
    if (given != Py_None) {
      if (Py_TYPE(given) != (PyTypeObject*)THPVariableClass) not_regular();
      t = THPVariable_Unpack(given).scalar_type();
    }
    if (t != dtype && t != at::kByte) not_regular();
    type = t == at::kByte ? (int)LBA_TYPE_CODES : float_type(t);
    if (t == at::kByte) {
      const at::Tensor& s = as_tensor(out_scale, at::kFloat, -1, call.device);
      if (s.numel() != 1) not_regular();
      scale = (const float*)s.data_ptr();
      if (prod_fmt != Py_None) flags = as_format(prod_fmt).flags & LBA_FLAG_INPUT_M4E3;
    }
    out = given_or_fresh(given, call, sizes, t);
  }
};

// q, k, v, cu_q, cu_k, causal, scale, out_dtype, out_scale, prod_fmt, lse, out, stream
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return regular_or_none(n, 13, [&]() -> PyObject* {
    const Call call(a[12]);
    const Attention x(call, a[0], a[1], a[2], a[3], a[4], a[5], a[6]);
    const Output y(call, x.q.t.sizes(), x.q.t.scalar_type(), a[7], a[8], a[9], a[11]);
    const bool fresh = a[10] == Py_True, wanted = fresh || (a[10] != Py_False && a[10] != Py_None);
    at::Tensor lse;
    if (wanted) lse = given_or_fresh(fresh ? Py_None : a[10], call, {x.q.t.size(1), x.q.t.size(0)}, at::kFloat);
    float* const pl = wanted ? (float*)lse.data_ptr() : nullptr;
    void* const po = y.out.data_ptr();
    const int status =
        without_gil([&] { return lba_attention(x.q.data, x.k.data, x.v.data, &x.how, y.type, y.scale, y.flags, po, pl, call.stream); });
    if (status != 0) return PyLong_FromLong(status);
    PyObject* const out = wrapped(a[11], y.out);
    return wanted ? both_of(out, wrapped(fresh ? Py_None : a[10], lse)) : out;
  });
}

// grad_out, q, k, v, out, lse, cu_q, cu_k, causal, scale, workspace, stream
PyObject* attention_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return regular_or_none(n, 12, [&]() -> PyObject* {
    const Call call(a[11]);
    const Attention x(call, a[1], a[2], a[3], a[6], a[7], a[8], a[9]);
    const c10::ScalarType dtype = x.q.t.scalar_type();
    const at::Tensor &g = as_tensor(a[0], dtype, 3, call.device), &out = as_tensor(a[4], dtype, 3, call.device), &lse = as_tensor(a[5], at::kFloat, 2, call.device);
    if (g.sizes() != x.q.t.sizes() || out.sizes() != x.q.t.sizes() || lse.size(0) != x.q.t.size(1) || lse.size(1) != x.q.t.size(0)) not_regular();
    const at::Tensor ws = a[10] != Py_None ? as_tensor(a[10], at::kByte, -1, call.device)
                                           : call.fresh({(int64_t)lba_attention_backward_workspace_bytes(&x.how)}, at::kByte);
    const at::Tensor gq = call.fresh(x.q.t.sizes(), dtype), gk = call.fresh(x.k.t.sizes(), dtype), gv = call.fresh(x.k.t.sizes(), dtype);
    const void *const pg = g.data_ptr(), *const po = out.data_ptr();
    const float* const pl = (const float*)lse.data_ptr();
    return results(without_gil([&] {
                     return lba_attention_backward(pg, x.q.data, x.k.data, x.v.data, po, pl, &x.how, gq.data_ptr(), gk.data_ptr(), gv.data_ptr(),
                                                   ws.data_ptr(), ws.numel(), call.stream);
                   }), {gq, gk, gv});
  });
}

// a cache [pages][heads][page (dim + dim / 16)] and its block table [sequences][width]
lba_cache as_cache(PyObject* o, PyObject* page, PyObject* table, int64_t sequences, const Call& call) {
  const at::Tensor &t = as_tensor(o, at::kByte, 3, call.device), &b = as_tensor(table, at::kInt, 2, call.device);
  const int64_t p = as_int(page), run = t.size(2);
  if (b.size(0) != sequences || p < 1 || p > INT_MAX || run % (17 * p) || run * 16 / (17 * p) % 32) not_regular();
  lba_cache c = {};
  c.pages = t.data_ptr();
  c.page_count = t.size(0);
  c.kv_heads = as_size(t.size(1));
  c.dim = as_size(run * 16 / (17 * p));
  c.page = (int)p;
  c.sequences = as_size(sequences);
  c.table_width = as_size(b.size(1));
  c.table = (const int32_t*)b.data_ptr();
  return c;
}

// k, v, cache, page, table, start, cu, stream
PyObject* cache_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return regular_or_none(n, 8, [&]() -> PyObject* {
    const Call call(a[7]);
    const Heads k(a[0], call), v(a[1], call);
    const at::Tensor& start = as_tensor(a[5], at::kInt, -1, call.device);
    const lba_cache c = as_cache(a[2], a[3], a[4], start.numel(), call);
    if (k.t.scalar_type() != v.t.scalar_type() || k.t.sizes() != v.t.sizes() || k.t.size(1) != c.kv_heads || k.t.size(2) != c.dim) not_regular();
    const int type = float_type(k.t.scalar_type());
    const int32_t* const cu = as_ints(a[6], start.numel() + 1, call.device);
    const int status = without_gil([&] {
      return lba_cache_append(&c, k.data, k.at, v.data, v.at, type, k.t.size(0), (const int32_t*)start.data_ptr(), cu, call.stream);
    });
    return status != 0 ? PyLong_FromLong(status) : Py_NewRef(a[2]);
  });
}

// cache, page, table, start, cu, tokens, dtype, out, stream
PyObject* cache_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return regular_or_none(n, 9, [&]() -> PyObject* {
    const Call call(a[8]);
    const at::Tensor& start = as_tensor(a[3], at::kInt, -1, call.device);
    const lba_cache c = as_cache(a[0], a[1], a[2], start.numel(), call);
    const int32_t* const cu = as_ints(a[4], start.numel() + 1, call.device);
    const int64_t tokens = as_int(a[5]);
    const c10::ScalarType dtype = as_dtype(a[6]);
    const int type = float_type(dtype);
    if (tokens < 0 || a[7] != Py_None) not_regular();
    const at::Tensor k = call.fresh({tokens, c.kv_heads, c.dim}, dtype), v = call.fresh({tokens, c.kv_heads, c.dim}, dtype);
    return results(without_gil([&] {
                     return lba_cache_read(&c, (const int32_t*)start.data_ptr(), cu, tokens, type, k.data_ptr(), v.data_ptr(), call.stream);
                   }), {k, v});
  });
}

// q, cache, page, table, lengths, scale, out_dtype, out_scale, prod_fmt, workspace, out, stream
PyObject* cache_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return regular_or_none(n, 12, [&]() -> PyObject* {
    const Call call(a[11]);
    const Heads q(a[0], call);
    const int type = half_type(q.t.scalar_type()), heads = as_size(q.t.size(1));
    const lba_cache c = as_cache(a[1], a[2], a[3], q.t.size(0), call);
    if (q.t.size(2) != c.dim || a[4] == Py_None) not_regular();
    const int32_t* const lengths = as_ints(a[4], q.t.size(0), call.device);
    const float scale = (float)(a[5] == Py_None ? std::pow((double)c.dim, -0.5) : as_real(a[5]));
    const Output y(call, q.t.sizes(), q.t.scalar_type(), a[6], a[7], a[8], a[10]);
    const at::Tensor ws = a[9] != Py_None ? as_tensor(a[9], at::kByte, -1, call.device)
                                          : call.fresh({(int64_t)lba_cache_attention_workspace_bytes(&c, heads)}, at::kByte);
    void* const po = y.out.data_ptr();
    const int status = without_gil([&] {
      return lba_cache_attention(q.data, q.at, type, heads, &c, lengths, scale, y.type, y.scale, y.flags, po, ws.data_ptr(), ws.numel(), call.stream);
    });
    return status != 0 ? PyLong_FromLong(status) : wrapped(a[10], y.out);
  });
}

PyObject* init_module(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 2) {
    PyErr_SetString(PyExc_TypeError, "init takes the format class and the parameter class");
    return nullptr;
  }
  static const char* const names[5] = {"man_bits", "exp_bits", "bias", "rounding", "flags"};
  for (int i = 0; i < 5; ++i)
    if (!g_field[i] && !(g_field[i] = PyUnicode_InternFromString(names[i]))) return nullptr;
  Py_XSETREF(g_format_type, Py_NewRef(a[0]));
  Py_XSETREF(g_parameter_type, Py_NewRef(a[1]));
  Py_RETURN_NONE;
}

PyMethodDef kMethods[] = {
    {"init", (PyCFunction)(void (*)(void))init_module, METH_FASTCALL, "the format class whose instances are read by attribute, and the parameter class"},
    {"gemm", (PyCFunction)(void (*)(void))gemm, METH_FASTCALL, nullptr},
    {"gemm_batched", (PyCFunction)(void (*)(void))gemm_batched, METH_FASTCALL, nullptr},
    {"conv2d", (PyCFunction)(void (*)(void))conv2d, METH_FASTCALL, nullptr},
    {"linear", (PyCFunction)(void (*)(void))linear, METH_FASTCALL, nullptr},
    {"gated", (PyCFunction)(void (*)(void))gated, METH_FASTCALL, nullptr},
    {"linear_backward", (PyCFunction)(void (*)(void))linear_backward, METH_FASTCALL, nullptr},
    {"gated_backward", (PyCFunction)(void (*)(void))gated_backward, METH_FASTCALL, nullptr},
    {"rotary", (PyCFunction)(void (*)(void))rotary, METH_FASTCALL, nullptr},
    {"attention", (PyCFunction)(void (*)(void))attention, METH_FASTCALL, nullptr},
    {"attention_backward", (PyCFunction)(void (*)(void))attention_backward, METH_FASTCALL, nullptr},
    {"cache_append", (PyCFunction)(void (*)(void))cache_append, METH_FASTCALL, nullptr},
    {"cache_read", (PyCFunction)(void (*)(void))cache_read, METH_FASTCALL, nullptr},
    {"cache_attention", (PyCFunction)(void (*)(void))cache_attention, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "lba_torch", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_lba_torch() {
  PyObject* const m = PyModule_Create(&kModule);
  if (m && PyModule_AddStringConstant(m, "built_for", LBA_TORCH_TAG) != 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
