"""Thin binding of ``liblba.so`` (C ABI declared in ``include/lba.h``), through ctypes.

The forward entry points hand a regular call (plain contiguous tensors of the current device, its current stream) to
``lba_torch.so``, which makes the same checks and the same C call in 4 us of host time instead of 10 to 12; everything else, and
every error, takes the ctypes path.  So do all calls, after one warning, where that module is missing or was built for another
torch or interpreter.

Argument marshalling only: PyTorch supplies device memory and the current stream; every step of
the computation runs in the CUDA kernels behind the C entry points.  There is no fallback: if the
library is missing, or a call returns an error, an exception is raised.
"""
import contextlib
import ctypes as C
import importlib.util
import os
import warnings

import torch

from .build import torch_tag
from .formats import FLAG_INPUT_M4E3, LbaFormat, ORDER_CHUNKED, PAPER_CHUNK

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblba.so")
TORCH_LIB_PATH = os.path.join(_HERE, "lba_torch.so")

EXPORTS = ["lba_gemm", "lba_gemm_batched", "lba_linear", "lba_gated", "lba_linear_backward", "lba_gated_backward", "lba_backward_workspace_bytes", "lba_gemm_last_overflow", "lba_gemm_ste_mask", "lba_conv2d", "lba_gemm_host_workspace_bytes", "lba_gemm_host",
           "lba_conv2d_host_workspace_bytes", "lba_conv2d_host", "lba_gemm_host_static", "lba_count_nan_codes", "lba_describe_plan", "lba_describe_plan_batched",
           "lba_set_tile_override", "lba_set_wait_override", "lba_status_string", "lba_last_cuda_error", "lba_version"]


class LbaError(RuntimeError):
    def __init__(self, status, text, cuda_error=0):
        super().__init__(f"liblba status {status}: {text}" + (f" (cudaError {cuda_error})" if cuda_error else ""))
        self.status = status
        self.cuda_error = cuda_error


class _Fmt(C.Structure):
    _fields_ = [("man_bits", C.c_int32), ("exp_bits", C.c_int32), ("bias", C.c_int32), ("rounding", C.c_int32),
                ("flags", C.c_int32)]


class _Layer(C.Structure):
    _fields_ = [("activation", C.c_int32), ("out_type", C.c_int32), ("out_scale", C.c_void_p), ("preact", C.c_void_p),
                ("residual", C.c_void_p), ("preact_type", C.c_int32), ("residual_type", C.c_int32), ("dropout", C.c_double),
                ("rng", C.c_void_p)]


class _Backward(C.Structure):
    _fields_ = [("activation", C.c_int32), ("grad_type", C.c_int32), ("out_type", C.c_int32), ("preact_type", C.c_int32),
                ("preact", C.c_void_p), ("dropout", C.c_double), ("rng", C.c_void_p), ("input_flags", C.c_int32)]


_lib = None
_native = None  # lba_torch.so, or None where it cannot be used


def _load_native():
    """lba_torch.so, or None with a warning: every call then takes the ctypes path, which needs nothing but the library."""
    try:
        spec = importlib.util.spec_from_file_location("lba_torch", TORCH_LIB_PATH)
        native = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(native)
        if native.built_for != torch_tag():
            raise ImportError(f"built for {native.built_for!r}, this is {torch_tag()!r}")
        native.init(LbaFormat, torch.nn.Parameter)
        return native
    except (ImportError, OSError, AttributeError, TypeError) as e:
        warnings.warn(f"{TORCH_LIB_PATH} cannot be used, calls go through ctypes (6 to 8 us more of host time each); build it with "
                      f"`python -m paper_2401_14110_b200.build`: {e}", RuntimeWarning, stacklevel=3)
        return None


def load_library():
    """Load liblba.so from the package directory; raises if it has not been built."""
    global _lib, _native
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2401_14110_b200.build` "
                           "(there is no CPU or PyTorch fallback)")
    lib = C.CDLL(LIB_PATH)
    lib.lba_status_string.restype = C.c_char_p
    lib.lba_status_string.argtypes = [C.c_int]
    lib.lba_gemm_host_workspace_bytes.restype = C.c_size_t
    lib.lba_gemm_host_workspace_bytes.argtypes = [C.c_int64, C.c_int64, C.c_int64, C.c_int, C.c_int, C.c_int]
    lib.lba_conv2d_host_workspace_bytes.restype = C.c_size_t
    lib.lba_conv2d_host_workspace_bytes.argtypes = [C.c_int] * 14
    gemm_args = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_int, C.c_void_p, C.c_int64, C.c_int64,
                 C.c_int64, C.POINTER(_Fmt), C.POINTER(_Fmt), C.c_int, C.c_int, C.c_void_p]
    lib.lba_gemm.argtypes = gemm_args + [C.c_void_p]
    lib.lba_gemm_host.argtypes = gemm_args + [C.c_void_p, C.c_size_t, C.c_void_p]
    lib.lba_gemm_last_overflow.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.POINTER(_Fmt),
                                           C.POINTER(_Fmt), C.c_void_p, C.c_void_p]
    lib.lba_gemm_ste_mask.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.POINTER(_Fmt),
                                      C.POINTER(_Fmt), C.c_int, C.c_int, C.c_int, C.c_float, C.c_float, C.c_void_p,
                                      C.c_void_p, C.c_void_p]
    lib.lba_gemm_batched.argtypes = gemm_args[:7] + [C.c_int64] * 7 + gemm_args[10:] + [C.c_void_p]
    lib.lba_gemm_host_static.argtypes = gemm_args + [C.c_void_p]
    lib.lba_linear.argtypes = gemm_args[:14] + [C.POINTER(_Layer), C.c_void_p, C.c_void_p]
    lib.lba_gated.argtypes = [C.c_void_p] * 4 + [C.c_int, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p] + \
        [C.c_int64] * 3 + gemm_args[10:14] + [C.POINTER(_Layer), C.c_void_p, C.c_void_p]
    lib.lba_backward_workspace_bytes.restype = C.c_size_t
    lib.lba_backward_workspace_bytes.argtypes = [C.c_int] + [C.c_int64] * 3 + [C.c_int, C.c_int, C.POINTER(_Backward), C.c_int]
    lib.lba_linear_backward.argtypes = gemm_args[:2] + [C.c_void_p] + gemm_args[2:6] + [C.c_int64] * 3 + [C.POINTER(_Backward)] + \
        [C.c_void_p] * 4 + [C.c_size_t, C.c_void_p]
    lib.lba_gated_backward.argtypes = [C.c_void_p] * 5 + [C.c_int, C.c_void_p, C.c_void_p, C.c_int] + [C.c_int64] * 3 + \
        [C.POINTER(_Backward)] + [C.c_void_p] * 6 + [C.c_size_t, C.c_void_p]
    conv_args = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_int, C.c_void_p] + [C.c_int] * 11 + \
        [C.POINTER(_Fmt), C.POINTER(_Fmt), C.c_int, C.c_int, C.c_void_p]
    lib.lba_conv2d.argtypes = conv_args + [C.c_void_p]
    lib.lba_conv2d_host.argtypes = conv_args + [C.c_void_p, C.c_size_t, C.c_void_p]
    lib.lba_count_nan_codes.argtypes = [C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
    lib.lba_describe_plan.argtypes = [C.c_int64, C.c_int64, C.c_int64, C.POINTER(_Fmt), C.POINTER(_Fmt), C.c_int,
                                      C.c_int, C.c_int, C.c_int, C.c_char_p, C.c_size_t]
    lib.lba_describe_plan_batched.argtypes = [C.c_int64] + lib.lba_describe_plan.argtypes
    for name in EXPORTS:
        getattr(lib, name)
    _native = _load_native()
    _lib = lib
    return lib


def _done(result):
    """What a native call returned: the output, or the library's status where it is not 0."""
    if result.__class__ is int:
        _check(result)
    return result


def _check(status):
    if status:
        lib = load_library()
        raise LbaError(status, lib.lba_status_string(status).decode(), lib.lba_last_cuda_error())


def _fmt(f):
    t = f.as_tuple() if isinstance(f, LbaFormat) else tuple(f)
    return _Fmt(*[int(v) for v in t])


_fmt_refs = {}   # five Python integers -> pointer to their C struct, which the library only reads


def _fmt_ref(f):
    """Pointer to the format's C struct (building it anew took a fifth of a small call's 17 to 21 us on the host).  Only tuples
    of Python integers are kept: the fields may also be arrays or tensors of one element, which do not hash by value."""
    t = f.as_tuple() if isinstance(f, LbaFormat) else tuple(f)
    try:
        ref = _fmt_refs.get(t)
    except TypeError:
        ref = None
    if ref is None:
        t = tuple(int(v) for v in t)
        ref = _fmt_refs.get(t)
        if ref is None:
            if len(_fmt_refs) >= 256:
                _fmt_refs.clear()
            ref = _fmt_refs[t] = C.byref(_Fmt(*t))
    return ref


def _stream(stream):
    if stream is None:  # the current device's current stream, without the wrapper object
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _torch_stream(stream, device):
    """An explicit stream as PyTorch knows it (handles 0 and 1: the default stream)."""
    if isinstance(stream, torch.cuda.Stream):
        return stream
    handle = _stream(stream)
    return torch.cuda.default_stream(device) if handle in (0, 1) else torch.cuda.ExternalStream(handle, device)


def _empty(shape, dtype, device, stream, returned=True):
    """torch.empty for a kernel on ``stream``.  Memory belongs to the stream that it is allocated on: from the current one's, a kernel
    elsewhere could be given what work that is still queued here reads.  What is returned is used here too, which the allocator is told."""
    if stream is None or device.type != "cuda":
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(_torch_stream(stream, device)):
        t = torch.empty(shape, dtype=dtype, device=device)
    if returned:
        t.record_stream(torch.cuda.current_stream(device))
    return t


def _dev(t, dtype, name):
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise TypeError(f"{name} must be a contiguous CUDA tensor of dtype {dtype}")
    return t.data_ptr()


def _host(t, dtype, name):
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and not t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise TypeError(f"{name} must be a contiguous CPU tensor of dtype {dtype}")
    return t.data_ptr()


def conv_out_hw(H, W, KH, KW, stride, pad):
    return (H + 2 * pad[0] - KH) // stride[0] + 1, (W + 2 * pad[1] - KW) // stride[1] + 1


def lba_gemm(A, B, scale_a, scale_b, bias, prod_fmt, acc_fmt, order=ORDER_CHUNKED, chunk=PAPER_CHUNK, out=None,
             stream=None):
    """out[M][N] (float32, CUDA) for A [M][K], B [N][K] E4M3 bytes on the GPU.  See ``lba_gemm`` in lba.h."""
    lib = load_library()
    done = _native and _native.gemm(A, B, scale_a, scale_b, bias, prod_fmt, acc_fmt, order, chunk, out, stream)
    if done is not None:
        return _done(done)
    M, K = A.shape
    N, K2 = B.shape
    if K != K2:
        raise ValueError("A and B disagree on K")
    if out is None:
        out = _empty((M, N), torch.float32, A.device, stream)
    pf, af = _fmt_ref(prod_fmt), _fmt_ref(acc_fmt)
    _check(lib.lba_gemm(_dev(A, torch.uint8, "A"), _dev(B, torch.uint8, "B"), _dev(scale_a, torch.float32, "scale_a"),
                        scale_a.numel(), _dev(scale_b, torch.float32, "scale_b"), scale_b.numel(),
                        _dev(bias, torch.float32, "bias"), M, N, K, pf, af, order, chunk,
                        _dev(out, torch.float32, "out"), _stream(stream)))
    return out


def lba_gemm_batched(A, B, scale_a, scale_b, bias, prod_fmt, acc_fmt, order=ORDER_CHUNKED, chunk=PAPER_CHUNK, out=None,
                     stream=None):
    """out[Z][M][N] for A [Z][M][K] and B [Z][N][K] (or [N][K], shared by all Z problems).  See lba.h."""
    lib = load_library()
    done = _native and _native.gemm_batched(A, B, scale_a, scale_b, bias, prod_fmt, acc_fmt, order, chunk, out, stream)
    if done is not None:
        return _done(done)
    Z, M, K = A.shape
    if B.dim() == 2:
        N, K2 = B.shape
        stride_b = 0
    else:
        Zb, N, K2 = B.shape
        if Zb != Z:
            raise ValueError("A and B disagree on the batch size")
        stride_b = N * K
    if K != K2:
        raise ValueError("A and B disagree on K")
    if out is None:
        out = _empty((Z, M, N), torch.float32, A.device, stream)
    pf, af = _fmt_ref(prod_fmt), _fmt_ref(acc_fmt)
    _check(lib.lba_gemm_batched(_dev(A, torch.uint8, "A"), _dev(B, torch.uint8, "B"),
                                _dev(scale_a, torch.float32, "scale_a"), scale_a.numel(),
                                _dev(scale_b, torch.float32, "scale_b"), scale_b.numel(),
                                _dev(bias, torch.float32, "bias"), Z, M, N, K, M * K, stride_b, M * N, pf,
                                af, order, chunk, _dev(out, torch.float32, "out"), _stream(stream)))
    return out


_FLOAT_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_OUT_TYPES = {**_FLOAT_TYPES, torch.uint8: 3}
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}


def _activation(name):
    if name not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {', '.join(ACTIVATIONS)}, not {name!r}")
    return ACTIVATIONS[name]


def _typed(t, name):
    """(data pointer, type number) of a contiguous CUDA tensor of 32- or 16-bit floats; (None, 0) for None."""
    if t is None:
        return None, 0
    if not (isinstance(t, torch.Tensor) and t.dtype in _FLOAT_TYPES):
        raise TypeError(f"{name} must be a float32, bfloat16 or float16 CUDA tensor")
    return _dev(t, t.dtype, name), _FLOAT_TYPES[t.dtype]


def _shaped(t, shape, name):
    if t is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    return t


def _same_device(first, *others):
    if any(t is not None and t.device != first.device for t in others) or (first.is_cuda and first.device.index != torch.cuda.current_device()):
        raise ValueError("all tensors of a call must be on the current CUDA device")


def _scale(t, name):
    """(pointer, length) of a tensor of scales"""
    ptr = _dev(t, torch.float32, name)
    if ptr is None:
        raise TypeError(f"{name} must be a contiguous CUDA tensor of dtype torch.float32")
    return ptr, t.numel()


def _rng(rng, dropout):
    if not dropout:
        return None
    ptr = _dev(rng, torch.int64, "rng")
    if ptr is None or rng.numel() != 2:
        raise TypeError("rng must be a CUDA tensor of two int64 values (seed, offset) where dropout is not 0")
    return ptr


def _layer(out_shape, pre_shape, device, stream, activation, out_dtype, out_scale, preact, out, residual=None, dropout=0.0, rng=None):
    """The C struct of a layer's epilogue, and the output and pre-activation tensors that it points to."""
    if out is None:
        if out_dtype not in _OUT_TYPES:
            raise TypeError("out_dtype must be torch.float32, bfloat16, float16, or uint8 for codes")
        out = _empty(out_shape, out_dtype, device, stream)
    elif out.dtype not in _OUT_TYPES:
        raise TypeError("out must be a float32, bfloat16, float16 or (codes) uint8 CUDA tensor")
    _shaped(out, out_shape, "out")
    if isinstance(preact, torch.dtype):
        if preact not in _FLOAT_TYPES:
            raise TypeError("preact must be torch.float32, bfloat16 or float16, a tensor of these, or None")
        preact = _empty(pre_shape, preact, device, stream)
    pre, pre_type = _typed(_shaped(preact, pre_shape, "preact"), "preact")
    res, res_type = _typed(_shaped(residual, out_shape, "residual"), "residual")
    codes = out.dtype == torch.uint8
    if codes and (out_scale is None or out_scale.numel() != 1):
        raise TypeError("codes need out_scale, a CUDA tensor of one float32 value")
    layer = _Layer(_activation(activation), _OUT_TYPES[out.dtype], _dev(out_scale, torch.float32, "out_scale") if codes else None, pre, res,
                   pre_type, res_type, float(dropout), _rng(rng, dropout))
    return layer, out, preact


def lba_linear(A, B, scale_a, scale_b, bias, prod_fmt, acc_fmt, order=ORDER_CHUNKED, chunk=PAPER_CHUNK, activation="none",
               residual=None, dropout=0.0, rng=None, out_dtype=torch.float32, out_scale=None, preact=None, out=None, stream=None):
    """A linear layer: out[M][N] = round(drop(act(lba_gemm(A, B, ...))) + residual), in one kernel.  See ``lba_linear`` in lba.h.

    ``activation``: "none", "relu", "gelu", "gelu_tanh" or "silu".  ``out_dtype``: float32, bfloat16, float16, or uint8 for codes
    of the operands' own format, the output divided by ``out_scale`` (a tensor of one value).  ``dropout``: probability of
    dropping an element, with ``rng`` an int64 CUDA tensor (seed, offset).  ``preact``: a float dtype, or a tensor to write: the
    pre-activations that ``lba_linear_backward`` takes; the call then returns (out, preact)."""
    lib = load_library()
    done = _native and _native.linear(A, B, scale_a, scale_b, bias, prod_fmt, acc_fmt, order, chunk, activation, residual, dropout, rng, out_dtype,
                                      out_scale, preact, out, stream)
    if done is not None:
        return _done(done)
    M, K = A.shape
    N, K2 = B.shape
    if K != K2:
        raise ValueError("A and B disagree on K")
    _same_device(A, B, scale_a, scale_b, bias, residual, rng if dropout else None, out_scale, out, None if isinstance(preact, torch.dtype) else preact)
    layer, out, pre = _layer((M, N), (M, N), A.device, stream, activation, out_dtype, out_scale, preact, out, residual, dropout, rng)
    sa, sa_len = _scale(scale_a, "scale_a")
    sb, sb_len = _scale(scale_b, "scale_b")
    _check(lib.lba_linear(_dev(A, torch.uint8, "A"), _dev(B, torch.uint8, "B"), sa, sa_len, sb, sb_len,
                          _dev(_shaped(bias, (N,), "bias"), torch.float32, "bias"), M, N, K, _fmt_ref(prod_fmt), _fmt_ref(acc_fmt), order, chunk,
                          C.byref(layer), _dev(out, out.dtype, "out"), _stream(stream)))
    return out if pre is None else (out, pre)


def lba_gated(A, B_gate, B_up, scale_a, scale_gate, scale_up, bias_gate, bias_up, prod_fmt, acc_fmt, order=ORDER_CHUNKED,
              chunk=PAPER_CHUNK, activation="silu", out_dtype=torch.float32, out_scale=None, preact=None, out=None, stream=None):
    """A gated feed-forward layer: out[M][N] = round(act(gate) * up) for the two projections gate = lba_gemm(A, B_gate, ...) and
    up = lba_gemm(A, B_up, ...), in one kernel.  See ``lba_gated`` in lba.h.

    ``preact``: a float dtype, or a tensor to write, [2][M][N]: both projections, as ``lba_gated_backward`` takes them; the call
    then returns (out, preact).  The other arguments are those of ``lba_linear``."""
    lib = load_library()
    done = _native and _native.gated(A, B_gate, B_up, scale_a, scale_gate, scale_up, bias_gate, bias_up, prod_fmt, acc_fmt, order, chunk, activation,
                                     out_dtype, out_scale, preact, out, stream)
    if done is not None:
        return _done(done)
    M, K = A.shape
    N, K2 = B_gate.shape
    if K != K2 or tuple(B_up.shape) != (N, K):
        raise ValueError("A, B_gate and B_up disagree on K, or the two projections on N")
    _same_device(A, B_gate, B_up, scale_a, scale_gate, scale_up, bias_gate, bias_up, out_scale, out, None if isinstance(preact, torch.dtype) else preact)
    layer, out, pre = _layer((M, N), (2, M, N), A.device, stream, activation, out_dtype, out_scale, preact, out)
    sa, sa_len = _scale(scale_a, "scale_a")
    sg, sg_len = _scale(scale_gate, "scale_gate")
    su, su_len = _scale(scale_up, "scale_up")
    if sg_len != su_len:
        raise ValueError("scale_gate and scale_up must have the same length")
    _check(lib.lba_gated(_dev(A, torch.uint8, "A"), _dev(B_gate, torch.uint8, "B_gate"), _dev(B_up, torch.uint8, "B_up"), sa, sa_len, sg, su,
                         sg_len, _dev(_shaped(bias_gate, (N,), "bias_gate"), torch.float32, "bias_gate"),
                         _dev(_shaped(bias_up, (N,), "bias_up"), torch.float32, "bias_up"), M, N, K, _fmt_ref(prod_fmt), _fmt_ref(acc_fmt), order,
                         chunk, C.byref(layer), _dev(out, out.dtype, "out"), _stream(stream)))
    return out if pre is None else (out, pre)


def _backward(gated, grad_out, shape, K, scale_a_len, scale_b_len, prod_fmt, preact, activation, dropout, rng, grad_dtype, needs, workspace,
              device, stream):
    """What both backward passes share: the C struct, the type of the gradients and the workspace."""
    lib = load_library()
    g, g_type = _typed(_shaped(grad_out, shape, "grad_out"), "grad_out")
    if g is None:
        raise TypeError("grad_out must be a float32, bfloat16 or float16 CUDA tensor")
    pre, pre_type = _typed(_shaped(preact, (2, *shape) if gated else shape, "preact"), "preact")
    grad_dtype = grad_out.dtype if grad_dtype is None else grad_dtype
    if grad_dtype not in _FLOAT_TYPES:
        raise TypeError("grad_dtype must be torch.float32, bfloat16 or float16")
    flags = (prod_fmt.flags if isinstance(prod_fmt, LbaFormat) else int(tuple(prod_fmt)[4])) & FLAG_INPUT_M4E3
    how = _Backward(_activation(activation), g_type, _FLOAT_TYPES[grad_dtype], pre_type, pre, float(dropout), _rng(rng, dropout), flags)
    need = lib.lba_backward_workspace_bytes(gated, shape[0], shape[1], K, scale_a_len, scale_b_len, C.byref(how),
                                            sum(1 << i for i, n in enumerate(needs) if n))
    if workspace is None:
        workspace = _empty(need, torch.uint8, device, stream, returned=False)
    return how, g, grad_dtype, workspace


def lba_linear_backward(grad_out, A, B, scale_a, scale_b, prod_fmt, preact=None, activation="none", dropout=0.0, rng=None, grad_dtype=None,
                        needs=(True, True, True), workspace=None, stream=None):
    """(grad_a [M][K], grad_b [N][K], grad_bias [N]) of ``lba_linear`` under the straight-through estimator, None where ``needs`` says
    so.  See ``lba_linear_backward`` in lba.h.

    ``preact`` is what the forward call kept; ``activation``, ``dropout`` and ``rng`` are the forward call's (``rng`` holding the
    same two values), and so is ``prod_fmt``, which says what the operands' bytes are.  ``grad_dtype``: of grad_a and grad_b,
    grad_out's if None; grad_bias is float32.  ``workspace``: a CUDA uint8 tensor of ``backward_workspace_bytes``, or None."""
    lib = load_library()
    done = _native and _native.linear_backward(grad_out, A, B, scale_a, scale_b, prod_fmt, preact, activation, dropout, rng, grad_dtype, needs,
                                               workspace, stream)
    if done is not None:
        return _done(done)
    M, K = A.shape
    N, K2 = B.shape
    if K != K2:
        raise ValueError("A and B disagree on K")
    _same_device(A, B, scale_a, scale_b, grad_out, preact, rng if dropout else None, workspace)
    sa, sa_len = _scale(scale_a, "scale_a")
    sb, sb_len = _scale(scale_b, "scale_b")
    how, g, dtype, ws = _backward(0, grad_out, (M, N), K, sa_len, sb_len, prod_fmt, preact, activation, dropout, rng, grad_dtype, needs,
                                  workspace, A.device, stream)
    ga = _empty((M, K), dtype, A.device, stream) if needs[0] else None
    gb = _empty((N, K), dtype, A.device, stream) if needs[1] else None
    gc = _empty((N,), torch.float32, A.device, stream) if needs[2] else None
    _check(lib.lba_linear_backward(g, _dev(A, torch.uint8, "A"), _dev(B, torch.uint8, "B"), sa, sa_len, sb, sb_len, M, N, K,
                                              C.byref(how), _typed(ga, "grad_a")[0], _typed(gb, "grad_b")[0],
                                              _dev(gc, torch.float32, "grad_bias"), _dev(ws, torch.uint8, "workspace"), ws.numel(),
                                              _stream(stream)))
    return ga, gb, gc


def lba_gated_backward(grad_out, A, B_gate, B_up, scale_a, scale_gate, scale_up, prod_fmt, preact, activation="silu", grad_dtype=None,
                       needs=(True, True, True), workspace=None, stream=None):
    """(grad_a, grad_gate, grad_up, grad_bias_gate, grad_bias_up) of ``lba_gated``; ``preact`` is the [2][M][N] that the forward call
    kept, the other arguments are those of ``lba_linear_backward``.  See ``lba_gated_backward`` in lba.h."""
    lib = load_library()
    done = _native and _native.gated_backward(grad_out, A, B_gate, B_up, scale_a, scale_gate, scale_up, prod_fmt, preact, activation, grad_dtype,
                                              needs, workspace, stream)
    if done is not None:
        return _done(done)
    M, K = A.shape
    N, K2 = B_gate.shape
    if K != K2 or tuple(B_up.shape) != (N, K):
        raise ValueError("A, B_gate and B_up disagree on K, or the two projections on N")
    _same_device(A, B_gate, B_up, scale_a, scale_gate, scale_up, grad_out, preact, workspace)
    sa, sa_len = _scale(scale_a, "scale_a")
    sg, sg_len = _scale(scale_gate, "scale_gate")
    su, su_len = _scale(scale_up, "scale_up")
    if sg_len != su_len:
        raise ValueError("scale_gate and scale_up must have the same length")
    how, g, dtype, ws = _backward(1, grad_out, (M, N), K, sa_len, sg_len, prod_fmt, preact, activation, 0.0, None, grad_dtype, needs, workspace,
                                  A.device, stream)
    ga = _empty((M, K), dtype, A.device, stream) if needs[0] else None
    gg, gu = (_empty((N, K), dtype, A.device, stream) if needs[1] else None for _ in range(2))
    cg, cu = (_empty((N,), torch.float32, A.device, stream) if needs[2] else None for _ in range(2))
    _check(lib.lba_gated_backward(g, _dev(A, torch.uint8, "A"), _dev(B_gate, torch.uint8, "B_gate"), _dev(B_up, torch.uint8, "B_up"),
                                             sa, sa_len, sg, su, sg_len, M, N, K, C.byref(how), _typed(ga, "grad_a")[0],
                                             _typed(gg, "grad_gate")[0], _typed(gu, "grad_up")[0], _dev(cg, torch.float32, "grad_bias_gate"),
                                             _dev(cu, torch.float32, "grad_bias_up"), _dev(ws, torch.uint8, "workspace"), ws.numel(),
                                             _stream(stream)))
    return ga, gg, gu, cg, cu


def backward_workspace_bytes(M, N, K, scale_a_len, scale_b_len, grad_dtype, activation="none", gated=False, grad_out_dtype=None,
                             needs=(True, True, True)):
    """Bytes of workspace of a backward call with gradients of ``grad_dtype``."""
    how = _Backward(_activation(activation), _FLOAT_TYPES[grad_out_dtype or grad_dtype], _FLOAT_TYPES[grad_dtype], 0, None, 0.0, None, 0)
    return load_library().lba_backward_workspace_bytes(int(gated), M, N, K, scale_a_len, scale_b_len, C.byref(how),
                                                       sum(1 << i for i, n in enumerate(needs) if n))


def lba_gemm_last_overflow(A, B, prod_fmt, acc_fmt, out=None, stream=None):
    """int32 [M][N]: index of the last sequential step at which Q_acc overflowed, -1 if none.  See lba.h."""
    lib = load_library()
    M, K = A.shape
    N, K2 = B.shape
    if K != K2:
        raise ValueError("A and B disagree on K")
    if out is None:
        out = _empty((M, N), torch.int32, A.device, stream)
    pf, af = _fmt_ref(prod_fmt), _fmt_ref(acc_fmt)
    _check(lib.lba_gemm_last_overflow(_dev(A, torch.uint8, "A"), _dev(B, torch.uint8, "B"), M, N, K, pf,
                                      af, _dev(out, torch.int32, "last"), _stream(stream)))
    return out


STE_OF, STE_DIFF = 1, 2


def lba_gemm_ste_mask(A, B, prod_fmt, acc_fmt, order=ORDER_CHUNKED, chunk=PAPER_CHUNK, ste=STE_OF, eps1=0.0, eps2=0.0,
                      mask1=None, mask2=None, stream=None):
    """(mask1 int32 [M][ceil(K/32)][N], mask2 int32 [M][ceil(ceil(K/chunk)/32)][N] or None): one STE bit per FMAq
    step, as 32-bit words (torch has no unsigned 32-bit arithmetic; the bit patterns are what counts).  See lba.h."""
    lib = load_library()
    M, K = A.shape
    N, K2 = B.shape
    if K != K2:
        raise ValueError("A and B disagree on K")
    if mask1 is None:
        mask1 = _empty((M, (K + 31) // 32, N), torch.int32, A.device, stream)
    if order != ORDER_CHUNKED:
        mask2 = None
    elif mask2 is None:
        mask2 = _empty((M, ((K + chunk - 1) // max(chunk, 1) + 31) // 32, N), torch.int32, A.device, stream)
    pf, af = _fmt_ref(prod_fmt), _fmt_ref(acc_fmt)
    _check(lib.lba_gemm_ste_mask(_dev(A, torch.uint8, "A"), _dev(B, torch.uint8, "B"), M, N, K, pf, af,
                                 order, chunk, ste, C.c_float(eps1), C.c_float(eps2), _dev(mask1, torch.int32, "mask1"),
                                 None if mask2 is None else _dev(mask2, torch.int32, "mask2"), _stream(stream)))
    return mask1, mask2


def lba_conv2d(x, w, scale_x, scale_w, bias, stride, pad, prod_fmt, acc_fmt, order=ORDER_CHUNKED, chunk=PAPER_CHUNK,
               out=None, stream=None):
    """out [B][Hout][Wout][Cout] for x [B][H][W][Cin], w [Cout][KH][KW][Cin] E4M3 bytes.  See lba.h."""
    lib = load_library()
    done = _native and _native.conv2d(x, w, scale_x, scale_w, bias, stride, pad, prod_fmt, acc_fmt, order, chunk, out, stream)
    if done is not None:
        return _done(done)
    B, H, W, Cin = x.shape
    Cout, KH, KW, Cin2 = w.shape
    if Cin != Cin2:
        raise ValueError("x and w disagree on C_in")
    Hout, Wout = conv_out_hw(H, W, KH, KW, stride, pad)
    if out is None:
        out = _empty((B, max(Hout, 0), max(Wout, 0), Cout), torch.float32, x.device, stream)
    pf, af = _fmt_ref(prod_fmt), _fmt_ref(acc_fmt)
    _check(lib.lba_conv2d(_dev(x, torch.uint8, "x"), _dev(w, torch.uint8, "w"), _dev(scale_x, torch.float32, "scale_x"),
                          scale_x.numel(), _dev(scale_w, torch.float32, "scale_w"), scale_w.numel(),
                          _dev(bias, torch.float32, "bias"), B, H, W, Cin, Cout, KH, KW, stride[0], stride[1], pad[0],
                          pad[1], pf, af, order, chunk, _dev(out, torch.float32, "out"),
                          _stream(stream)))
    return out


def gemm_host_workspace_bytes(M, N, K, scale_a_len, scale_b_len, has_bias):
    return load_library().lba_gemm_host_workspace_bytes(M, N, K, scale_a_len, scale_b_len, int(has_bias))


def lba_gemm_host(A, B, scale_a, scale_b, bias, prod_fmt, acc_fmt, order, chunk, out, workspace, stream=None):
    """Host-buffer variant: CPU tensors in (pinned recommended), CPU ``out``; ``workspace`` is a CUDA uint8 tensor."""
    lib = load_library()
    M, K = A.shape
    N, _ = B.shape
    pf, af = _fmt_ref(prod_fmt), _fmt_ref(acc_fmt)
    _check(lib.lba_gemm_host(_host(A, torch.uint8, "A"), _host(B, torch.uint8, "B"),
                             _host(scale_a, torch.float32, "scale_a"), scale_a.numel(),
                             _host(scale_b, torch.float32, "scale_b"), scale_b.numel(),
                             _host(bias, torch.float32, "bias"), M, N, K, pf, af, order, chunk,
                             _host(out, torch.float32, "out"), _dev(workspace, torch.uint8, "workspace"),
                             workspace.numel(), _stream(stream)))
    return out


STATIC_WORKSPACE_BYTES = 8 << 20   # LBA_STATIC_WORKSPACE_BYTES in lba.h


def lba_gemm_host_static(A, B, scale_a, scale_b, bias, prod_fmt, acc_fmt, order, chunk, out, stream=None):
    """``lba_gemm_host`` for callers that cannot allocate device memory: CPU tensors in, CPU ``out``, and the
    device workspace is an 8 MiB array built into the library (shared by all calls on a device, so calls must
    not overlap on the GPU).  Larger problems raise ``LbaError`` with status -8.  No tensor is created here."""
    lib = load_library()
    M, K = A.shape
    N, _ = B.shape
    pf, af = _fmt_ref(prod_fmt), _fmt_ref(acc_fmt)
    _check(lib.lba_gemm_host_static(_host(A, torch.uint8, "A"), _host(B, torch.uint8, "B"),
                                    _host(scale_a, torch.float32, "scale_a"), scale_a.numel(),
                                    _host(scale_b, torch.float32, "scale_b"), scale_b.numel(),
                                    _host(bias, torch.float32, "bias"), M, N, K, pf, af, order,
                                    chunk, _host(out, torch.float32, "out"), _stream(stream)))
    return out


def conv2d_host_workspace_bytes(B, H, W, Cin, Cout, KH, KW, stride, pad, scale_x_len, scale_w_len, has_bias):
    return load_library().lba_conv2d_host_workspace_bytes(B, H, W, Cin, Cout, KH, KW, stride[0], stride[1], pad[0],
                                                          pad[1], scale_x_len, scale_w_len, int(has_bias))


def lba_conv2d_host(x, w, scale_x, scale_w, bias, stride, pad, prod_fmt, acc_fmt, order, chunk, out, workspace,
                    stream=None):
    lib = load_library()
    B, H, W, Cin = x.shape
    Cout, KH, KW, _ = w.shape
    pf, af = _fmt_ref(prod_fmt), _fmt_ref(acc_fmt)
    _check(lib.lba_conv2d_host(_host(x, torch.uint8, "x"), _host(w, torch.uint8, "w"),
                               _host(scale_x, torch.float32, "scale_x"), scale_x.numel(),
                               _host(scale_w, torch.float32, "scale_w"), scale_w.numel(),
                               _host(bias, torch.float32, "bias"), B, H, W, Cin, Cout, KH, KW, stride[0], stride[1],
                               pad[0], pad[1], pf, af, order, chunk,
                               _host(out, torch.float32, "out"), _dev(workspace, torch.uint8, "workspace"),
                               workspace.numel(), _stream(stream)))
    return out


def count_nan_codes(codes, stream=None):
    """Number of E4M3 NaN codes (0x7F, 0xFF) in a CUDA uint8 tensor (synchronises)."""
    lib = load_library()
    data = _dev(codes, torch.uint8, "codes")
    with contextlib.nullcontext() if stream is None else torch.cuda.stream(_torch_stream(stream, codes.device)):
        count = torch.zeros(1, dtype=torch.int64, device=codes.device)
        _check(lib.lba_count_nan_codes(data, codes.numel(), C.c_void_p(count.data_ptr()), _stream(stream)))
        return int(count.item())


def set_tile_override(tile):
    """Force the CTA tile (0..3, 5 = cluster pair) or restore the automatic choice (-1).  A testing hook: process-wide.
    Speed only; results are unchanged."""
    _check(load_library().lba_set_tile_override(int(tile)))


def set_wait_override(which):
    """Let waits inside the layers' backward products run out at once (1 to 3, see lba.h), or restore them (0).  A testing hook: process-wide."""
    _check(load_library().lba_set_wait_override(int(which)))


def describe_plan(M, N, K, prod_fmt, acc_fmt, order=ORDER_CHUNKED, chunk=PAPER_CHUNK, is_conv=False, vec_ok=True, batch=1):
    """Text description of the kernel variant a call would run (``batch`` problems for ``lba_gemm_batched``); raises
    LbaError for rejected arguments."""
    lib = load_library()
    buf = C.create_string_buffer(256)
    pf, af = _fmt_ref(prod_fmt), _fmt_ref(acc_fmt)
    _check(lib.lba_describe_plan_batched(batch, M, N, K, pf, af, order, chunk, int(is_conv), int(vec_ok),
                                         buf, 256))
    return buf.value.decode()
