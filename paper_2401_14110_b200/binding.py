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
import math
import os
import warnings

import torch

from .build import torch_tag
from .formats import FLAG_INPUT_M4E3, LbaFormat, ORDER_CHUNKED, PAPER_CHUNK

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblba.so")
TORCH_LIB_PATH = os.path.join(_HERE, "lba_torch.so")

EXPORTS = ["lba_rotary", "lba_attention", "lba_attention_backward", "lba_attention_backward_workspace_bytes", "lba_cache_append", "lba_cache_read",
           "lba_cache_attention", "lba_cache_attention_workspace_bytes", "lba_gemm", "lba_gemm_batched", "lba_linear", "lba_gated", "lba_linear_backward", "lba_gated_backward", "lba_backward_workspace_bytes", "lba_gemm_last_overflow", "lba_gemm_ste_mask", "lba_conv2d", "lba_gemm_host_workspace_bytes", "lba_gemm_host",
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


class _Strides(C.Structure):
    _fields_ = [("token", C.c_int64), ("head", C.c_int64)]


class _Rotary(C.Structure):
    _fields_ = [("type", C.c_int32), ("heads", C.c_int32), ("kv_heads", C.c_int32), ("dim", C.c_int32), ("rotary_dim", C.c_int32),
                ("interleaved", C.c_int32), ("inverse", C.c_int32), ("wide_positions", C.c_int32), ("scale", C.c_float), ("tokens", C.c_int64),
                ("positions", C.c_void_p), ("freqs", C.c_void_p)]


class _Attention(C.Structure):
    _fields_ = [("type", C.c_int32), ("heads", C.c_int32), ("kv_heads", C.c_int32), ("dim", C.c_int32), ("causal", C.c_int32),
                ("sequences", C.c_int32), ("scale", C.c_float), ("q_rows", C.c_int64), ("k_rows", C.c_int64), ("cu_q", C.c_void_p),
                ("cu_k", C.c_void_p), ("q_at", _Strides), ("k_at", _Strides), ("v_at", _Strides)]


class _Cache(C.Structure):
    _fields_ = [("pages", C.c_void_p), ("page_count", C.c_int64), ("kv_heads", C.c_int32), ("dim", C.c_int32), ("page", C.c_int32),
                ("sequences", C.c_int32), ("table_width", C.c_int32), ("table", C.c_void_p)]


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
    lib.lba_rotary.argtypes = [C.c_void_p, _Strides, C.c_void_p, _Strides, C.POINTER(_Rotary), C.c_void_p, _Strides, C.c_void_p, _Strides, C.c_void_p]
    lib.lba_attention.argtypes = [C.c_void_p] * 3 + [C.POINTER(_Attention), C.c_int, C.c_void_p, C.c_int] + [C.c_void_p] * 3
    lib.lba_attention_backward_workspace_bytes.restype = C.c_size_t
    lib.lba_attention_backward_workspace_bytes.argtypes = [C.POINTER(_Attention)]
    lib.lba_attention_backward.argtypes = [C.c_void_p] * 6 + [C.POINTER(_Attention)] + [C.c_void_p] * 4 + [C.c_size_t, C.c_void_p]
    lib.lba_cache_append.argtypes = [C.POINTER(_Cache), C.c_void_p, _Strides, C.c_void_p, _Strides, C.c_int, C.c_int64] + [C.c_void_p] * 3
    lib.lba_cache_read.argtypes = [C.POINTER(_Cache), C.c_void_p, C.c_void_p, C.c_int64, C.c_int] + [C.c_void_p] * 3
    lib.lba_cache_attention_workspace_bytes.restype = C.c_size_t
    lib.lba_cache_attention_workspace_bytes.argtypes = [C.POINTER(_Cache), C.c_int]
    lib.lba_cache_attention.argtypes = [C.c_void_p, _Strides, C.c_int, C.c_int, C.POINTER(_Cache), C.c_void_p, C.c_float, C.c_int, C.c_void_p, C.c_int] + \
        [C.c_void_p] * 2 + [C.c_size_t, C.c_void_p]
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


def rotary_frequencies(rotary_dim, base=10000.0, scaling="none", factor=1.0, original_length=8192, low=1.0, high=4.0, device="cuda"):
    """float64 frequencies of a head's rotary_dim / 2 pairs for ``lba_rotary``, base^(-2 i / rotary_dim), and for texts longer than a
    model was trained on (``factor`` times):

    ``"linear"``: all divided by ``factor``.  ``"base"``: the base is raised so that the slowest pair is divided by ``factor``.  ``"ramp"``:
    pairs that turn fewer than ``low`` times within ``original_length`` tokens are divided by ``factor``, those that turn more than ``high``
    times are kept, and those between are blended linearly in their number of turns."""
    if rotary_dim < 2 or rotary_dim % 2 or not factor > 0 or not base > 0:
        raise ValueError("rotary_dim must be even and at least 2, factor and base above 0")
    n = rotary_dim // 2
    if scaling == "base" and n > 1:
        base = base * factor ** (rotary_dim / (rotary_dim - 2))
    f = base ** (-torch.arange(n, dtype=torch.float64) / n)
    if scaling == "linear":
        f = f / factor
    elif scaling == "ramp":
        if not high > low:
            raise ValueError("high must be above low")
        keep = ((original_length * f / (2 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
        f = keep * f + (1 - keep) * f / factor
    elif scaling not in ("none", "base"):
        raise ValueError(f"scaling must be none, linear, base or ramp, not {scaling!r}")
    return f.to(device)


def _heads(t, name, dtypes=None):
    """(pointer, strides, type number) of a CUDA tensor [rows][heads][dim] whose heads' values are contiguous; rows and heads may be apart"""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == 3 and t.dtype in (dtypes or _FLOAT_TYPES)):
        raise TypeError(f"{name} must be a CUDA tensor [rows][heads][dim] of " + ("bfloat16 or float16" if dtypes else "float32, bfloat16 or float16"))
    if t.shape[2] > 1 and t.stride(2) != 1:
        raise ValueError(f"the values of a head of {name} must be contiguous")
    return t.data_ptr(), _Strides(t.stride(0), t.stride(1)), _FLOAT_TYPES[t.dtype]


_HALF_TYPES = (torch.bfloat16, torch.float16)
_NO_STRIDES = _Strides(0, 0)


def _int32(t, n, name):
    """pointer of a contiguous CUDA int32 tensor of n values (None: NULL)"""
    if t is not None and t.numel() != n:
        raise ValueError(f"{name} must hold {n} values, not {t.numel()}")
    return _dev(t, torch.int32, name)


def lba_rotary(q, k, positions, freqs, interleaved=False, inverse=False, scale=1.0, out=None, stream=None):
    """(q, k) with their pairs turned by positions x frequencies: see ``lba_rotary`` in lba.h.

    ``q`` [T][heads][dim], ``k`` [T][kv_heads][dim] or None: slices of a projection's output will do.  ``positions``: int32 or int64, [T];
    ``freqs``: float64, half the values that turn (``rotary_frequencies``).  ``inverse``: the opposite way, which is the gradient's.
    ``scale``: multiplies what turns.  ``out``: a pair of tensors, which may be ``q`` and ``k`` themselves."""
    lib = load_library()
    done = _native and _native.rotary(q, k, positions, freqs, interleaved, inverse, scale, out, stream)
    if done is not None:
        return _done(done)
    qo, ko = (None, None) if out is None else out
    _same_device(q, k, positions, freqs, qo, ko)
    pq, q_at, dtype = _heads(q, "q")
    if k is not None and (k.dtype != q.dtype or k.dim() != 3 or k.shape[0] != q.shape[0] or k.shape[2] != q.shape[2]):
        raise ValueError("k must have q's type, tokens and dim")
    pk, k_at, _ = (None, _NO_STRIDES, 0) if k is None else _heads(k, "k")
    if positions.dtype not in (torch.int32, torch.int64) or positions.numel() != q.shape[0]:
        raise TypeError("positions must be an int32 or int64 CUDA tensor with a value for each token")
    how = _Rotary(dtype, q.shape[1], 0 if k is None else k.shape[1], q.shape[2], 2 * freqs.numel(), int(interleaved), int(inverse),
                  int(positions.dtype == torch.int64), float(scale), q.shape[0], _dev(positions, positions.dtype, "positions"),
                  _dev(freqs, torch.float64, "freqs"))
    if qo is None:
        qo = _empty(q.shape, q.dtype, q.device, stream)
    if k is not None and ko is None:
        ko = _empty(k.shape, k.dtype, k.device, stream)
    for t, like, name in ((qo, q, "out[0]"), (ko, k, "out[1]")):
        if like is not None and (t.dtype != like.dtype or t.shape != like.shape):
            raise ValueError(f"{name} must have the shape and type of what it is of")
    po, qo_at, _ = _heads(qo, "out[0]")
    pko, ko_at, _ = (None, _NO_STRIDES, 0) if k is None else _heads(ko, "out[1]")
    _check(lib.lba_rotary(pq, q_at, pk, k_at, C.byref(how), po, qo_at, pko, ko_at, _stream(stream)))
    return qo, (None if k is None else ko)


def _attention(q, k, v, cu_q, cu_k, causal, scale):
    """the C struct of an attention call, and its tensors' pointers"""
    pq, q_at, dtype = _heads(q, "q", _HALF_TYPES)
    pk, k_at, kt = _heads(k, "k", _HALF_TYPES)
    pv, v_at, vt = _heads(v, "v", _HALF_TYPES)
    if kt != dtype or vt != dtype or k.shape != v.shape or k.shape[2] != q.shape[2]:
        raise ValueError("q, k and v must have one type and dim, k and v one shape")
    if (cu_q is None) != (cu_k is None):
        raise ValueError("cu_q and cu_k come together")
    n = 1 if cu_q is None else cu_q.numel() - 1
    if n < 0:
        raise ValueError("cu_q holds one value more than there are sequences")
    how = _Attention(dtype, q.shape[1], k.shape[1], q.shape[2], int(causal), n, float(q.shape[2] ** -0.5 if scale is None else scale), q.shape[0],
                     k.shape[0], _int32(cu_q, n + 1, "cu_q"), _int32(cu_k, n + 1, "cu_k"), q_at, k_at, v_at)
    return how, pq, pk, pv


def _attention_out(shape, dtype, device, stream, out_dtype, out_scale, prod_fmt, out):
    """(out, its type, scale pointer, flags) of an attention's output: the inputs' type, or codes"""
    if out is None:
        out = _empty(shape, dtype if out_dtype is None else out_dtype, device, stream)
    _shaped(out, shape, "out")
    if out.dtype not in (dtype, torch.uint8):
        raise TypeError("out must have the inputs' type, or be uint8 for codes")
    codes = out.dtype == torch.uint8
    if codes and (out_scale is None or out_scale.numel() != 1):
        raise TypeError("codes need out_scale, a CUDA tensor of one float32 value")
    flags = 0
    if codes and prod_fmt is not None:
        flags = (prod_fmt.flags if isinstance(prod_fmt, LbaFormat) else int(tuple(prod_fmt)[4])) & FLAG_INPUT_M4E3
    return out, _OUT_TYPES[out.dtype], _dev(out_scale, torch.float32, "out_scale") if codes else None, flags


def lba_attention(q, k, v, cu_q=None, cu_k=None, causal=True, scale=None, out_dtype=None, out_scale=None, prod_fmt=None, lse=False, out=None,
                  stream=None):
    """Attention of packed sequences over whole prompts: out [Tq][heads][dim].  See ``lba_attention`` in lba.h.

    ``q`` [Tq][heads][dim], ``k`` and ``v`` [Tk][kv_heads][dim], bfloat16 or float16; slices of a projection's output will do.  ``cu_q``,
    ``cu_k``: int32 [sequences + 1], where each sequence's rows begin (None: one sequence of all rows).  ``scale``: dim^-1/2 if None.
    ``out_dtype``: uint8 for codes of out / ``out_scale`` in the byte format that ``prod_fmt`` names (E4M3 if None), as the next
    ``lba_linear`` takes them.  ``lse``: True, or a float32 tensor [heads][Tq] to write: the call then returns (out, lse), which
    ``lba_attention_backward`` takes.  Rows that no sequence holds are left as they were."""
    lib = load_library()
    done = _native and _native.attention(q, k, v, cu_q, cu_k, causal, scale, out_dtype, out_scale, prod_fmt, lse, out, stream)
    if done is not None:
        return _done(done)
    sums = lse if isinstance(lse, torch.Tensor) else None
    _same_device(q, k, v, cu_q, cu_k, out_scale, out, sums)
    how, pq, pk, pv = _attention(q, k, v, cu_q, cu_k, causal, scale)
    out, out_type, ps, flags = _attention_out(tuple(q.shape), q.dtype, q.device, stream, out_dtype, out_scale, prod_fmt, out)
    if lse is True:
        sums = _empty((q.shape[1], q.shape[0]), torch.float32, q.device, stream)
    _check(lib.lba_attention(pq, pk, pv, C.byref(how), out_type, ps, flags, _dev(out, out.dtype, "out"),
                             _dev(_shaped(sums, (q.shape[1], q.shape[0]), "lse"), torch.float32, "lse"), _stream(stream)))
    return out if sums is None else (out, sums)


def lba_attention_backward(grad_out, q, k, v, out, lse, cu_q=None, cu_k=None, causal=True, scale=None, workspace=None, stream=None):
    """(grad_q, grad_k, grad_v) of ``lba_attention``, whose ``out`` (of the inputs' type) and ``lse`` these are; contiguous, of q's type.
    See ``lba_attention_backward`` in lba.h.  ``workspace``: a CUDA uint8 tensor of ``attention_backward_workspace_bytes``, or None."""
    lib = load_library()
    done = _native and _native.attention_backward(grad_out, q, k, v, out, lse, cu_q, cu_k, causal, scale, workspace, stream)
    if done is not None:
        return _done(done)
    _same_device(q, k, v, grad_out, out, lse, cu_q, cu_k, workspace)
    how, pq, pk, pv = _attention(q, k, v, cu_q, cu_k, causal, scale)
    for t, name in ((grad_out, "grad_out"), (out, "out")):
        _dev(_shaped(t, tuple(q.shape), name), q.dtype, name)
    _shaped(lse, (q.shape[1], q.shape[0]), "lse")
    if workspace is None:
        workspace = _empty(lib.lba_attention_backward_workspace_bytes(C.byref(how)), torch.uint8, q.device, stream, returned=False)
    gq = _empty(tuple(q.shape), q.dtype, q.device, stream)
    gk, gv = (_empty(tuple(k.shape), q.dtype, q.device, stream) for _ in range(2))
    _check(lib.lba_attention_backward(grad_out.data_ptr(), pq, pk, pv, out.data_ptr(), _dev(lse, torch.float32, "lse"), C.byref(how), gq.data_ptr(),
                                      gk.data_ptr(), gv.data_ptr(), _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream)))
    return gq, gk, gv


def attention_backward_workspace_bytes(q, k, v, cu_q=None, cu_k=None, causal=True, scale=None):
    """Bytes of workspace of a ``lba_attention_backward`` call with these arguments."""
    return load_library().lba_attention_backward_workspace_bytes(C.byref(_attention(q, k, v, cu_q, cu_k, causal, scale)[0]))


def cache_shape(pages, kv_heads, page, dim):
    """Shape of the uint8 tensor that holds a cache of ``pages`` pages of ``page`` tokens."""
    return pages, kv_heads, page * (dim + dim // 16)


def _cache(cache, page, table, sequences):
    """the C struct of a cache [pages][kv_heads][page (dim + dim / 16)] and its block table [sequences][width]"""
    if not isinstance(cache, torch.Tensor) or cache.dim() != 3 or not isinstance(table, torch.Tensor) or table.dim() != 2:
        raise TypeError("cache must be a uint8 CUDA tensor of cache_shape(...), table an int32 one [sequences][pages of a sequence]")
    if table.shape[0] != sequences:
        raise ValueError(f"table must have a row for each of the {sequences} sequences")
    page, run = int(page), cache.shape[2]
    if page < 1 or run % (17 * page) or run * 16 // (17 * page) % 32:
        raise ValueError("the cache's last size must be page (dim + dim / 16), dim a multiple of 32")
    return _Cache(_dev(cache, torch.uint8, "cache"), cache.shape[0], cache.shape[1], run * 16 // (17 * page), page, sequences, table.shape[1],
                  _dev(table, torch.int32, "table"))


def lba_cache_append(k, v, cache, page, table, start, cu=None, stream=None):
    """Rounds new keys and values [T][kv_heads][dim] to 4 bits and stores them: row i of sequence b (row cu[b] + i of k and v; ``cu`` None: one row a
    sequence) becomes token start[b] + i.  See ``lba_cache_append`` in lba.h.  Returns ``cache``.

    ``cache``: uint8 of ``cache_shape(...)``; ``page``: tokens of a page; ``table``: int32 [sequences][pages of a sequence], numbers of
    pages; ``start``: int32 [sequences]; ``cu``: int32 [sequences + 1]."""
    lib = load_library()
    done = _native and _native.cache_append(k, v, cache, page, table, start, cu, stream)
    if done is not None:
        return _done(done)
    _same_device(cache, k, v, table, start, cu)
    n = start.numel()
    how = _cache(cache, page, table, n)
    pk, k_at, kt = _heads(k, "k")
    pv, v_at, vt = _heads(v, "v")
    if kt != vt or k.shape != v.shape or tuple(k.shape[1:]) != (how.kv_heads, how.dim):
        raise ValueError("k and v must be [tokens][kv_heads][dim] of the cache's heads and dim, of one type")
    _check(lib.lba_cache_append(C.byref(how), pk, k_at, pv, v_at, kt, k.shape[0], _int32(start, n, "start"), _int32(cu, n + 1, "cu"), _stream(stream)))
    return cache


def lba_cache_read(cache, page, table, start, cu, tokens, dtype=torch.bfloat16, out=None, stream=None):
    """(k, v) [tokens][kv_heads][dim] as numbers again: row cu[b] + i is token start[b] + i of sequence b.  See ``lba_cache_read`` in lba.h.

    ``tokens``: rows of the outputs, as cu's last value says; ``dtype``: float32, bfloat16 or float16; ``out``: a pair of tensors to write."""
    lib = load_library()
    done = _native and _native.cache_read(cache, page, table, start, cu, tokens, dtype, out, stream)
    if done is not None:
        return _done(done)
    k, v = (None, None) if out is None else out
    _same_device(cache, table, start, cu, k, v)
    n = start.numel()
    how = _cache(cache, page, table, n)
    shape = (int(tokens), how.kv_heads, how.dim)
    if dtype not in _FLOAT_TYPES:
        raise TypeError("dtype must be torch.float32, bfloat16 or float16")
    k, v = (_empty(shape, dtype, cache.device, stream) if t is None else _shaped(t, shape, "out") for t in (k, v))
    pk, kt = _typed(k, "out[0]")
    pv, vt = _typed(v, "out[1]")
    if kt != vt:
        raise ValueError("both outputs must have one type")
    _check(lib.lba_cache_read(C.byref(how), _int32(start, n, "start"), _int32(cu, n + 1, "cu"), shape[0], kt, pk, pv, _stream(stream)))
    return k, v


def lba_cache_attention(q, cache, page, table, lengths, scale=None, out_dtype=None, out_scale=None, prod_fmt=None, workspace=None, out=None, stream=None):
    """Attention of one new token of each sequence over its cached ones: out [sequences][heads][dim] for q of that shape.  See
    ``lba_cache_attention`` in lba.h.

    ``lengths``: int32 [sequences], tokens in the cache, the new one's among them.  ``out_dtype``, ``out_scale`` and ``prod_fmt`` are those of
    ``lba_attention``; ``workspace``: a CUDA uint8 tensor of ``cache_attention_workspace_bytes``, or None."""
    lib = load_library()
    done = _native and _native.cache_attention(q, cache, page, table, lengths, scale, out_dtype, out_scale, prod_fmt, workspace, out, stream)
    if done is not None:
        return _done(done)
    _same_device(q, cache, table, lengths, out_scale, workspace, out)
    pq, q_at, dtype = _heads(q, "q", _HALF_TYPES)
    n = q.shape[0]
    how = _cache(cache, page, table, n)
    if q.shape[2] != how.dim:
        raise ValueError(f"q must have the cache's dim, {how.dim}")
    out, out_type, ps, flags = _attention_out(tuple(q.shape), q.dtype, q.device, stream, out_dtype, out_scale, prod_fmt, out)
    if workspace is None:
        workspace = _empty(lib.lba_cache_attention_workspace_bytes(C.byref(how), q.shape[1]), torch.uint8, q.device, stream, returned=False)
    _check(lib.lba_cache_attention(pq, q_at, dtype, q.shape[1], C.byref(how), _int32(lengths, n, "lengths"),
                                   float(how.dim ** -0.5 if scale is None else scale), out_type, ps, flags, _dev(out, out.dtype, "out"),
                                   _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream)))
    return out


def cache_attention_workspace_bytes(cache, page, table, heads):
    """Bytes of workspace of a ``lba_cache_attention`` call on this cache and table."""
    return load_library().lba_cache_attention_workspace_bytes(C.byref(_cache(cache, page, table, table.shape[0])), heads)


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
