"""Layers without a GPU: the reference's generator against published vectors, and calls that are refused on the host."""
import ctypes as C

import pytest
import torch

from helpers.layer_ref import philox4x32
from paper_2401_14110_b200 import binding as lba
from paper_2401_14110_b200 import code_domain_formats, ORDER_CHUNKED as CHK

PROD, ACC = code_domain_formats(7, 4)
FAKE = C.c_void_p(256)
ONES = 0xFFFFFFFF


@pytest.mark.parametrize("counter,key,want", [   # the generator's published known answers
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((ONES,) * 4, (ONES,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_generator_known_answers(counter, key, want):
    assert tuple(philox4x32(counter, key)) == want


def _linear(M=4, N=4, K=16, layer=None, out=FAKE, a=FAKE, b=FAKE, sa_len=1, sb_len=1, prod=PROD, acc=ACC):
    lib = lba.load_library()
    ref = None if layer is None else C.byref(layer)
    return lib.lba_linear(a, b, FAKE, sa_len, FAKE, sb_len, None, M, N, K, C.byref(lba._fmt(prod)), C.byref(lba._fmt(acc)), CHK, 16, ref, out, None)


def _gated(M=4, N=4, K=16, layer=None, out=FAKE, up=FAKE, bias_gate=None, bias_up=None, sb_len=1):
    lib = lba.load_library()
    ref = None if layer is None else C.byref(layer)
    return lib.lba_gated(FAKE, FAKE, up, FAKE, 1, FAKE, FAKE, sb_len, bias_gate, bias_up, M, N, K, C.byref(lba._fmt(PROD)), C.byref(lba._fmt(ACC)),
                         CHK, 16, ref, out, None)


def _with(**kw):
    layer = lba._Layer()
    for k, v in kw.items():
        setattr(layer, k, v)
    return layer


@pytest.mark.parametrize("kw,status", [
    (dict(activation=5), -9), (dict(activation=-1), -9), (dict(out_type=4), -9), (dict(out_type=-1), -9),
    (dict(residual=256, residual_type=3), -9), (dict(preact=256, preact_type=3), -9),
    (dict(dropout=1.0, rng=256), -9), (dict(dropout=-0.1, rng=256), -9), (dict(dropout=float("nan"), rng=256), -9),
    (dict(dropout=1 - 2.0 ** -40, rng=256), -9),
    (dict(dropout=0.5), -1), (dict(out_type=3), -1),
])
def test_refused_layers(kw, status):
    assert _linear(layer=_with(**kw)) == status
    if "dropout" not in kw and "residual" not in kw:
        assert _gated(layer=_with(**kw)) == status


def test_refused_arguments():
    assert _linear(M=-1) == -2 and _linear(K=1 << 31) == -2 and _linear(sa_len=3) == -5 and _linear(sb_len=3) == -5
    assert _linear(out=None) == -1 and _linear(a=None) == -1 and _linear(b=None) == -1
    assert _linear(prod=(0, 4, 8, 0, 1)) == -3
    assert _linear(M=1 << 33, layer=_with(dropout=0.5, rng=256)) == -2       # a row's number is one word of the counter
    assert _gated(N=1 << 62) == -2 and _gated(sb_len=3) == -5 and _gated(up=None) == -1 and _gated(out=None) == -1
    assert _gated(bias_gate=FAKE) == -1 and _gated(bias_up=FAKE) == -1       # both biases or neither
    assert _gated(layer=_with(residual=256)) == -9 and _gated(layer=_with(dropout=0.5, rng=256)) == -9
    assert lba.load_library().lba_status_string(-9) != b"unknown status"


def test_empty_shapes_enqueue_nothing():
    assert _linear(M=0) == 0 and _linear(N=0) == 0 and _gated(M=0) == 0 and _gated(N=0) == 0


def test_binding_refuses_on_the_host():
    a, b = torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(8, 16, dtype=torch.uint8)
    s = torch.ones(1)
    with pytest.raises(TypeError):
        lba.lba_linear(a, b, s, s, None, PROD, ACC)                                        # not on a GPU
    with pytest.raises(ValueError):
        lba.lba_linear(a, b[:, :8], s, s, None, PROD, ACC)
    with pytest.raises(ValueError):
        lba.lba_linear(a, b, s, s, None, PROD, ACC, activation="tanh")
    with pytest.raises(TypeError):
        lba.lba_linear(a, b, s, s, None, PROD, ACC, out_dtype=torch.float64)
    with pytest.raises(TypeError):
        lba.lba_linear(a, b, s, s, None, PROD, ACC, out_dtype=torch.uint8)                 # codes without a scale
    with pytest.raises(TypeError):
        lba.lba_linear(a, b, s, s, None, PROD, ACC, preact=torch.int32)
    with pytest.raises(ValueError):
        lba.lba_linear(a, b, s, s, None, PROD, ACC, residual=torch.zeros(4, 4))
    with pytest.raises(TypeError):
        lba.lba_linear(a, b, s, s, None, PROD, ACC, dropout=0.5)                           # no generator
    with pytest.raises(ValueError):
        lba.lba_gated(a, b, b[:4], s, s, s, None, None, PROD, ACC)
    with pytest.raises(ValueError):
        lba.lba_gated(a, b, b, s, s, s, None, None, PROD, ACC, preact=torch.zeros(4, 8))


def _how(**kw):
    h = lba._Backward()
    h.activation, h.preact = 2, 256
    for k, v in kw.items():
        setattr(h, k, v)
    return h


def _backward(M=4, N=4, K=16, how=None, grad=FAKE, a=FAKE, ws=FAKE, ws_bytes=1 << 30, sa_len=1, sb_len=1, sa=FAKE):
    return lba.load_library().lba_linear_backward(grad, a, FAKE, sa, sa_len, FAKE, sb_len, M, N, K, None if how is None else C.byref(how), FAKE, FAKE,
                                                  FAKE, ws, ws_bytes, None)


def _gated_backward(how, grads=(256, 256), biases=(256, 256), up=FAKE):
    return lba.load_library().lba_gated_backward(FAKE, FAKE, FAKE, up, FAKE, 1, FAKE, FAKE, 1, 4, 4, 16, C.byref(how), FAKE, *grads, *biases, FAKE,
                                                 1 << 30, None)


@pytest.mark.parametrize("kw,status", [
    (dict(activation=5), -9), (dict(grad_type=3), -9), (dict(out_type=3), -9), (dict(preact_type=3), -9), (dict(input_flags=1), -9),
    (dict(dropout=1.0, rng=256), -9), (dict(dropout=0.5), -1), (dict(preact=None), -1),
])
def test_refused_backward_options(kw, status):
    assert _backward(how=_how(**kw)) == status


def test_refused_backward_arguments():
    h = _how()
    assert _backward(how=None) == -1 and _backward(how=h, grad=None) == -1 and _backward(how=h, a=None) == -1 and _backward(how=h, sa=None) == -1
    assert _backward(M=-1, how=h) == -2 and _backward(N=1 << 30, how=h) == -2 and _backward(M=1 << 31, how=h) == -2
    assert _backward(how=h, sa_len=3) == -5 and _backward(how=h, sb_len=3) == -5
    assert _backward(M=100, how=h, ws=None) == -7 and _backward(M=100, how=h, ws=C.c_void_p(128)) == -7 and _backward(M=100, how=h, ws_bytes=256) == -7
    assert _gated_backward(_how(dropout=0.5, rng=256)) == -9 and _gated_backward(_how(preact=None)) == -1
    assert _gated_backward(h, grads=(256, None)) == -1 and _gated_backward(h, biases=(None, 256)) == -1 and _gated_backward(h, up=None) == -1


def test_backward_workspace_grows_with_what_is_asked():
    size = lambda **k: lba.backward_workspace_bytes(1000, 50, 70, 1, k.pop("sb", 1), k.pop("dtype", torch.bfloat16), activation="gelu", **k)  # noqa: E731
    full = size()
    assert 0 < size(needs=(False, False, True)) < size(needs=(True, False, False)) < full
    assert size(sb=50) == full and size(dtype=torch.float16) > full and size(gated=True) > full
    assert lba.backward_workspace_bytes(16, 50, 70, 1, 1, torch.bfloat16, activation="gelu") == 0  # few rows need none
    assert size(needs=(False, False, False)) == 0 and lba.backward_workspace_bytes(0, 50, 70, 1, 1, torch.bfloat16) == 0
