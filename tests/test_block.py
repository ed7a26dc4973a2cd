"""What stands between a block's linear layers, without a GPU: calls that are refused on the host, frequencies, and the cache's layout."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from helpers.block_ref import cache_values, nearest4, row_bytes
from paper_2401_14110_b200 import binding as lba

FAKE = C.c_void_p(4096)
AT = lba._Strides(64, 64)


def _rotary(q=FAKE, k=FAKE, out=FAKE, k_out=FAKE, **kw):
    how = lba._Rotary(type=1, heads=2, kv_heads=1, dim=64, rotary_dim=64, scale=1.0, tokens=3, positions=4096, freqs=4096)
    for name, v in kw.items():
        setattr(how, name, v)
    return lba.load_library().lba_rotary(q, AT, k, AT, C.byref(how), out, AT, k_out, AT, None)


@pytest.mark.parametrize("kw,status", [
    (dict(type=3), -9), (dict(type=-1), -9), (dict(scale=math.inf), -9), (dict(scale=math.nan), -9),
    (dict(heads=0), -2), (dict(kv_heads=-1), -2), (dict(heads=65000, kv_heads=600), -2), (dict(dim=63, rotary_dim=62), -2), (dict(dim=1026, rotary_dim=64), -2),
    (dict(rotary_dim=66), -2), (dict(rotary_dim=63), -2), (dict(rotary_dim=0), -2), (dict(tokens=-1), -2), (dict(tokens=1 << 31), -2),
    (dict(q=None), -1), (dict(k=None), -1), (dict(out=None), -1), (dict(k_out=None), -1), (dict(positions=None), -1), (dict(freqs=None), -1),
    (dict(tokens=0, q=None, out=None, positions=None), 0),
])
def test_refused_rotary_calls(kw, status):
    assert _rotary(**kw) == status


def _attention_how(**kw):
    how = lba._Attention(type=1, heads=4, kv_heads=2, dim=64, causal=1, sequences=2, scale=0.125, q_rows=100, k_rows=100, cu_q=4096, cu_k=4096,
                         q_at=lba._Strides(256, 64), k_at=lba._Strides(128, 64), v_at=lba._Strides(128, 64))
    for name, v in kw.items():
        setattr(how, name, v)
    return how


def _attention(q=FAKE, k=FAKE, v=FAKE, out=FAKE, out_type=1, out_scale=None, flags=0, how=None, **kw):
    return lba.load_library().lba_attention(q, k, v, C.byref(how or _attention_how(**kw)), out_type, out_scale, flags, out, None, None)


def _gradients(g=FAKE, q=FAKE, k=FAKE, v=FAKE, out=FAKE, lse=FAKE, gq=FAKE, gk=FAKE, gv=FAKE, ws=FAKE, size=1 << 30, **kw):
    return lba.load_library().lba_attention_backward(g, q, k, v, out, lse, C.byref(_attention_how(**kw)), gq, gk, gv, ws, size, None)


SHAPES = [
    (dict(type=0), -9), (dict(type=3), -9), (dict(scale=0.0), -9), (dict(scale=-1.0), -9), (dict(scale=math.nan), -9), (dict(scale=math.inf), -9),
    (dict(heads=3), -2), (dict(heads=0), -2), (dict(kv_heads=0), -2), (dict(dim=0), -2), (dict(dim=12), -2), (dict(dim=136), -2), (dict(q_rows=-1), -2),
    (dict(k_rows=-1), -2), (dict(q_rows=(1 << 31) - 1000), -2), (dict(sequences=-1), -2), (dict(cu_q=None), -2), (dict(cu_k=None), -2),
    (dict(q_at=lba._Strides(260, 64)), -10), (dict(k_at=lba._Strides(128, 4)), -10), (dict(v_at=lba._Strides(0, 64)), -10),
    (dict(q_at=lba._Strides(1 << 40, 64)), -10),
]


@pytest.mark.parametrize("kw,status", SHAPES)
def test_refused_attention_shapes_in_both_directions(kw, status):
    assert _attention(**kw) == status and _gradients(**kw) == status
    assert lba.load_library().lba_attention_backward_workspace_bytes(C.byref(_attention_how(**kw))) == 0


def test_refused_attention_arguments():
    odd = C.c_void_p(4104)
    assert _attention(out_type=0) == -9 and _attention(out_type=2) == -9 and _attention(flags=1) == -9
    assert _attention(out_type=3) == -1 and _attention(q=None) == -1 and _attention(k=None) == -1 and _attention(v=None) == -1 and _attention(out=None) == -1
    assert _attention(q=odd) == -10 and _attention(v=odd) == -10 and _attention(out=odd) == -10
    assert lba.load_library().lba_attention(FAKE, FAKE, FAKE, None, 1, None, 0, FAKE, None, None) == -1
    assert _attention(q_rows=0, q=None, out=None) == 0 and _attention(sequences=0) == 0
    for name in ("g", "q", "k", "v", "out", "lse", "gq", "gk", "gv"):
        assert _gradients(**{name: None}) == -1
    assert _gradients(gk=odd) == -10 and _gradients(ws=None) == -7 and _gradients(ws=C.c_void_p(4096 + 16)) == -7 and _gradients(size=256) == -7


def _cache(**kw):
    c = lba._Cache(pages=4096, page_count=10, kv_heads=2, dim=64, page=16, sequences=3, table_width=5, table=4096)
    for name, v in kw.items():
        setattr(c, name, v)
    return c


def _decode(q=FAKE, type=1, heads=4, lengths=FAKE, scale=0.1, out_type=1, out_scale=None, flags=0, out=FAKE, ws=FAKE, size=1 << 30, **kw):
    return lba.load_library().lba_cache_attention(q, AT, type, heads, C.byref(_cache(**kw)), lengths, scale, out_type, out_scale, flags, out, ws, size, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dim=48), -2), (dict(dim=0), -2), (dict(dim=160), -2), (dict(page=8), -2), (dict(page=24), -2), (dict(page=2048), -2), (dict(kv_heads=0), -2),
    (dict(kv_heads=4096), -2), (dict(sequences=-1), -2), (dict(sequences=65536), -2), (dict(table_width=-1), -2), (dict(table_width=1 << 28), -2),
    (dict(page_count=1 << 31), -2), (dict(page_count=-1), -2), (dict(pages=4104), -10),
])
def test_refused_caches(kw, status):
    lib, c = lba.load_library(), _cache(**kw)
    assert _decode(**kw) == status
    assert lib.lba_cache_append(C.byref(c), FAKE, AT, FAKE, AT, 1, 3, FAKE, FAKE, None) == status
    assert lib.lba_cache_read(C.byref(c), FAKE, FAKE, 3, 1, FAKE, FAKE, None) == status
    assert lib.lba_cache_attention_workspace_bytes(C.byref(c), 4) == 0


def test_refused_cache_arguments():
    lib, c = lba.load_library(), _cache()
    append = lambda k=FAKE, v=FAKE, t=1, n=3, start=FAKE, c=c: lib.lba_cache_append(C.byref(c), k, AT, v, AT, t, n, start, FAKE, None)  # noqa: E731
    assert append(k=None) == -1 and append(v=None) == -1 and append(start=None) == -1 and append(t=3) == -9 and append(n=-1) == -2 and append(n=0, k=None) == 0
    assert append(c=_cache(pages=None)) == -1 and append(c=_cache(table=None)) == -1 and append(c=_cache(sequences=0), k=None) == 0
    assert _decode(type=0) == -9 and _decode(out_type=2) == -9 and _decode(scale=math.nan) == -9 and _decode(flags=2) == -9
    assert _decode(heads=3) == -2 and _decode(heads=0) == -2 and _decode(q=None) == -1 and _decode(lengths=None) == -1 and _decode(out=None) == -1
    assert _decode(out_type=3) == -1 and _decode(ws=None) == -7 and _decode(size=0) == -7 and _decode(ws=C.c_void_p(4096 + 128)) == -7
    assert _decode(sequences=0) == 0
    # 2^31 units of 64 tokens and more
    assert _decode(sequences=65535, table_width=1 << 24, page=64, kv_heads=4, heads=4) == -2


@pytest.mark.parametrize("scale", [0.0, -0.1, math.inf, math.nan])
def test_refused_scales_of_cache_attention(scale):
    assert _decode(scale=scale) == -9


def test_binding_refuses_what_is_no_cuda_tensor():
    x, n = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    cache, table = torch.zeros(lba.cache_shape(3, 2, 16, 64), dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.int32)
    for call in (lambda: lba.lba_rotary(x, x, n, torch.ones(32, dtype=torch.float64)), lambda: lba.lba_attention(x, x, x),
                 lambda: lba.lba_attention_backward(x, x, x, x, x, torch.zeros(2, 4)), lambda: lba.lba_cache_append(x, x, cache, 16, table, n),
                 lambda: lba.lba_cache_read(cache, 16, table, n, None, 4), lambda: lba.lba_cache_attention(x, cache, 16, table, n)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        lba._cache(cache, 24, table, 4)
    with pytest.raises(ValueError):
        lba._cache(cache, 16, table, 5)


def test_frequencies():
    f = lba.rotary_frequencies(8, device="cpu")
    assert f.dtype == torch.float64 and torch.allclose(f, torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=torch.float64), rtol=1e-12)
    assert torch.equal(lba.rotary_frequencies(8, scaling="linear", factor=4.0, device="cpu"), f / 4)
    raised = lba.rotary_frequencies(8, scaling="base", factor=4.0, device="cpu")
    assert raised[0] == 1 and abs(raised[-1] / f[-1] - 0.25) < 1e-12
    ramp = lba.rotary_frequencies(64, scaling="ramp", factor=8.0, original_length=8192, device="cpu")
    plain, turns = lba.rotary_frequencies(64, device="cpu"), 8192 * lba.rotary_frequencies(64, device="cpu") / (2 * math.pi)
    assert torch.equal(ramp[turns >= 4], plain[turns >= 4]) and torch.allclose(ramp[turns <= 1], plain[turns <= 1] / 8, rtol=1e-15)
    assert ((ramp <= plain) & (ramp >= plain / 8)).all()
    assert lba.rotary_frequencies(2, scaling="base", factor=2.0, device="cpu").tolist() == [1.0]
    for kw in (dict(rotary_dim=7), dict(rotary_dim=0), dict(rotary_dim=8, factor=0.0), dict(rotary_dim=8, scaling="other"), dict(rotary_dim=8, scaling="ramp", low=4.0)):
        with pytest.raises(ValueError):
            lba.rotary_frequencies(device="cpu", **kw)


def test_reference_of_the_cache_by_hand():
    """6 is 6 x 1; with 6.5 the power of two is 2: 6.5 / 2 = 3.25 is nearest to 3; ties go to the even code"""
    x = np.zeros((1, 32))
    x[0, :3] = 6.0, 2.5, -0.25
    assert nearest4(x)[0, :3].tolist() == [6.0, 2.0, 0.0]
    x[0, :5] = 6.5, 1.0, 3.0, 5.0, 7.0
    assert nearest4(x)[0, :5].tolist() == [6.0, 1.0, 3.0, 4.0, 8.0]


def test_layout_of_a_row():
    codes = list(range(16)) * 4
    cache = torch.zeros(lba.cache_shape(1, 1, 16, 64), dtype=torch.uint8)
    n = 16 * 64 // 2
    cache[0, 0, 5 * 32:6 * 32], cache[0, 0, n + 5 * 32:n + 6 * 32] = (torch.tensor(row_bytes(codes, key), dtype=torch.uint8) for key in (True, False))
    cache[0, 0, 2 * n:] = 127
    k, v = cache_values(cache, 16, 64)
    want = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64).repeat(4)
    assert torch.equal(k[0, 0, 5], want) and torch.equal(v[0, 0, 5], want) and (k[0, 0, 4] == 0).all()
