"""Gradients of attention on the GPU against the formulas in 64 bits and against differences."""
import math

import pytest
import torch

from helpers.block_ref import attention, close
from paper_2401_14110_b200 import binding as lba

pytestmark = pytest.mark.gpu


def _randn(*shape, seed=0, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(dtype)


def _cu(lengths, first=0):
    return torch.tensor([first] + [first + sum(lengths[:i + 1]) for i in range(len(lengths))], dtype=torch.int32, device="cuda")


def _check(q, k, v, cu_q, cu_k, causal, scale=None, size=1.0):
    g = (_randn(*q.shape, seed=77) * size).to(q.dtype)
    out, lse = lba.lba_attention(q, k, v, cu_q, cu_k, causal=causal, scale=scale, lse=True)
    got = lba.lba_attention_backward(g, q, k, v, out, lse, cu_q, cu_k, causal=causal, scale=scale)
    want = attention(q, k, v, cu_q, cu_k, causal, q.shape[2] ** -0.5 if scale is None else scale, grad=g, out16=out)
    for name, t, like in zip(("grad_q", "grad_k", "grad_v"), got, (q, k, v)):
        assert t.dtype == q.dtype and t.shape == like.shape and t.is_contiguous()
        close(t, want[name], want[name + "_bound"])
    return (g, q, k, v, out, lse), got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [8, 24, 64, 72, 80, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_head_sizes_and_groups(dim, causal, dtype):
    T, H, G = 300, 6, 2
    _check(_randn(T, H, dim, dtype=dtype), _randn(T, G, dim, seed=1, dtype=dtype), _randn(T, G, dim, seed=2, dtype=dtype), None, None, causal)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("T", [1, 2, 63, 64, 65, 127, 128, 129, 256, 257, 511, 1025])
def test_lengths(T, causal):
    _check(_randn(T, 2, 64), _randn(T, 2, 64, seed=1), _randn(T, 2, 64, seed=2), None, None, causal)


@pytest.mark.parametrize("causal", [False, True])
def test_packed_sequences_of_every_kind(causal):
    lq = [1, 0, 200, 128, 5, 0, 300, 17, 256, 0]
    lk = [1, 7, 200, 64, 500, 0, 0, 300, 255, 0]
    _check(_randn(sum(lq), 4, 128), _randn(sum(lk), 2, 128, seed=1), _randn(sum(lk), 2, 128, seed=2), _cu(lq), _cu(lk), causal)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim,heads,kv_heads", [(64, 12, 12), (128, 16, 2), (56, 6, 1)])
@pytest.mark.parametrize("causal", [False, True])
def test_short_sequences_are_off_by_the_results_rounding(dim, heads, kv_heads, causal, dtype):
    """A result's own rounding, uniform within half a step u, is 0.43 u of the norm (0.58 u over a mantissa's root mean square of 1.35 to 1.5).  Weights
    and slopes in two pieces add 2^-8 of that, outputs of 16 bits in delta a tenth or two; of one piece each they would make it 0.6 u."""
    lengths = [256, 8, 100, 30, 129, 200]
    T, cu = sum(lengths), _cu(lengths)
    q, k, v = _randn(T, heads, dim, dtype=dtype), _randn(T, kv_heads, dim, seed=1, dtype=dtype), _randn(T, kv_heads, dim, seed=2, dtype=dtype)
    (g, _, _, _, out, _), got = _check(q, k, v, cu, cu, causal)
    want = attention(q, k, v, cu, cu, causal, dim ** -0.5, grad=g, out16=out)
    for name, t in zip(("grad_q", "grad_k", "grad_v"), got):
        assert (t.double() - want[name]).norm() <= 0.5 * torch.finfo(dtype).eps / 2 * want[name].norm(), name


def test_groups_with_many_cut_tiles():
    lengths = [130, 70, 190]
    _check(_randn(390, 12, 64), _randn(390, 1, 64, seed=1), _randn(390, 1, 64, seed=2), _cu(lengths), _cu(lengths), True)


@pytest.mark.parametrize("size", [1e-6, 1e-3, 1.0, 500.0])
def test_small_and_large_gradients_of_binary16(size):
    """the common power of two keeps ds inside binary16: what a gradient is worth does not depend on its size, but for its own type's steps"""
    t = torch.float16
    _check(_randn(400, 2, 64, dtype=t), _randn(400, 2, 64, seed=1, dtype=t), _randn(400, 2, 64, seed=2, dtype=t), None, None, True, size=size)


@pytest.mark.parametrize("scale", [1e-4, 1.0, 10.0])
def test_scales(scale):
    _check(_randn(300, 2, 64), _randn(300, 2, 64, seed=1), _randn(300, 2, 64, seed=2), None, None, True, scale=scale)


def test_rows_of_no_sequence_get_zero_and_are_not_read():
    T, first, lengths = 200, 11, [50, 60]
    x = [_randn(T, h, 64, seed=s) for s, h in enumerate((4, 2, 2, 4))]
    for t in x:
        t[:first], t[first + 110:] = math.nan, math.inf
    q, k, v, g = x
    cu = _cu(lengths, first)
    out, lse = lba.lba_attention(q, k, v, cu, cu, lse=True, out=torch.full_like(q, math.nan))
    got = lba.lba_attention_backward(g, q, k, v, out, lse, cu, cu)
    inside = slice(first, first + 110)
    clean = [t[inside].contiguous() for t in x]
    want = attention(*clean[:3], _cu(lengths), _cu(lengths), True, 0.125, grad=clean[3], out16=out)
    outside = torch.ones(T, dtype=torch.bool, device="cuda")
    outside[inside] = False
    for name, t in zip(("grad_q", "grad_k", "grad_v"), got):
        close(t[inside], want[name], want[name + "_bound"])
        assert (t[outside] == 0).all()


@pytest.mark.parametrize("causal", [False, True])
def test_a_neighbours_values_do_not_leak(causal):
    lengths = [100, 60, 75]
    x = [_randn(235, h, 64, seed=s) for s, h in enumerate((2, 1, 1, 2))]
    cu = _cu(lengths)

    def run(q, k, v, g):
        out, lse = lba.lba_attention(q, k, v, cu, cu, causal=causal, lse=True)
        return lba.lba_attention_backward(g, q, k, v, out, lse, cu, cu, causal=causal)
    clean = run(*x)
    bad = [t.clone() for t in x]
    for t in bad:
        t[100:160] = math.nan
    for a, b in zip(run(*bad), clean):
        assert torch.equal(a[:100], b[:100]) and torch.equal(a[160:], b[160:])


def test_hidden_keys_do_not_count():
    """keys and values that are not finite spoil the rows that see them, and no earlier ones"""
    q, k, v, g = (_randn(200, h, 64, seed=s) for s, h in enumerate((2, 1, 1, 2)))

    def grad_q(k, v):
        out, lse = lba.lba_attention(q, k, v, lse=True)
        return lba.lba_attention_backward(g, q, k, v, out, lse)[0]
    clean = grad_q(k, v)
    for which in range(2):
        kv = [k.clone(), v.clone()]
        kv[which][150, 0, 3] = math.nan
        got = grad_q(*kv)
        assert torch.equal(got[:150], clean[:150]) and torch.isnan(got[150:]).any(-1).all()


def test_strides_of_projections():
    T, H, G, D = 150, 6, 2, 64
    x = _randn(T, H + 2 * G, D)
    _check(x[:, :H], x[:, H:H + G], x[:, H + G:], None, None, True)


def test_against_differences():
    """a step along a direction changes <out, g> by the gradient's product with it, up to the third derivative: 64-bit form and kernel side by side"""
    q, k, v = (_randn(40, 2, 16, seed=s, dtype=torch.float16) for s in range(3))
    (g, *_), got = _check(q, k, v, None, None, True)
    for i, (t, grad) in enumerate(zip((q, k, v), got)):
        d = _randn(*t.shape, seed=20 + i, dtype=torch.float32).double()

        def value(e):
            x = [a.double() for a in (q, k, v)]
            x[i] = x[i] + e * d
            s = torch.einsum("ihd,jhd->hij", x[0], x[1]) / 4
            s = s.masked_fill(torch.ones(40, 40, dtype=torch.bool, device="cuda").triu(1), -math.inf)
            return (torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), x[2]) * g.double()).sum()
        slope = (value(1e-5) - value(-1e-5)) / 2e-5
        # gradients are off by some 2^-10 of their terms each, independently: 1280 terms, ten of their standard deviations
        assert abs(slope - (grad.double() * d).sum()) <= 10 * 2.0 ** -10 * (grad.double() * d).norm() + 1e-6 * abs(slope) + 1e-2


def test_repeats_streams_and_graphs():
    lengths = [100, 300, 57]
    T, cu = sum(lengths), _cu(lengths)
    args, want = _check(_randn(T, 4, 128), _randn(T, 2, 128, seed=1), _randn(T, 2, 128, seed=2), cu, cu, True)
    for _ in range(3):
        for a, b in zip(lba.lba_attention_backward(*args, cu, cu), want):
            assert torch.equal(a, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = lba.lba_attention_backward(*args, cu, cu, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = lba.lba_attention_backward(*args, cu, cu)
    args[0].copy_(_randn(T, 4, 128, seed=31))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, lba.lba_attention_backward(*args, cu, cu)))


def test_empty():
    q, e = _randn(5, 2, 64), _randn(0, 2, 64)
    out, lse = lba.lba_attention(q, e, e, lse=True, causal=False)
    gq, gk, gv = lba.lba_attention_backward(q, q, e, e, out, lse, causal=False)
    assert (gq == 0).all() and gk.numel() == 0
    out, lse = lba.lba_attention(e, q, q, lse=True)
    gq, gk, gv = lba.lba_attention_backward(e, e, q, q, out, lse)
    assert (gk == 0).all() and (gv == 0).all()
