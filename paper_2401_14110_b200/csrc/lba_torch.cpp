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
