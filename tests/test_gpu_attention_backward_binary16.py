"""Gradients of attention of binary16 inputs: what a sequence, a row or a key gets does not depend on the size of what it does not go with."""
import math

import pytest
import torch

from helpers.block_ref import attention, close
from paper_2401_14110_b200 import binding as lba

pytestmark = pytest.mark.gpu
NAMES = ("grad_q", "grad_k", "grad_v")


def _randn(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda").half()


def _cu(lengths):
    return torch.tensor([sum(lengths[:i]) for i in range(len(lengths) + 1)], dtype=torch.int32, device="cuda")


def _inputs(Tq, Tk, H=2, G=1, D=64, size=2.0 ** -14):
    return [_randn(Tq, H, D), _randn(Tk, G, D, seed=1), _randn(Tk, G, D, seed=2), (_randn(Tq, H, D, seed=3).float() * size).half()]


def _run(x, cu_q=None, cu_k=None, causal=True):
    q, k, v, g = x
    out, lse = lba.lba_attention(q, k, v, cu_q, cu_k, causal=causal, lse=True)
    return lba.lba_attention_backward(g, q, k, v, out, lse, cu_q, cu_k, causal=causal), out


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("what", ["nan", "inf", "large"])
def test_neighbours_do_not_matter(what, causal, D):
    """the sequences beside one that is not finite, or has gradients and values 2^24 times theirs, get what they get beside an ordinary one"""
    lq, lk = [100, 60, 400], [130, 60, 400]
    cu_q, cu_k = _cu(lq), _cu(lk)
    x = _inputs(sum(lq), sum(lk), D=D, size=2.0 ** -19)
    clean, out = _run(x, cu_q, cu_k, causal)
    want = attention(*x[:3], cu_q, cu_k, causal, D ** -0.5, grad=x[3], out16=out)
    mid_q, mid_k = slice(100, 160), slice(130, 190)
    bad = [t.clone() for t in x]
    for i, t in enumerate(bad):
        at = mid_k if i in (1, 2) else mid_q
        if what != "large":
            t[at] = math.nan if what == "nan" else math.inf
    if what == "large":
        bad[2][mid_k] *= 2.0 ** 10
        bad[3][mid_q] = (bad[3][mid_q].float() * 2.0 ** 24).half()
    got, _ = _run(bad, cu_q, cu_k, causal)
    for a, b, name, mid in zip(got, clean, NAMES, (mid_q, mid_k, mid_k)):
        keep = torch.ones(a.shape[0], dtype=torch.bool, device="cuda")
        keep[mid] = False
        assert torch.equal(a[keep], b[keep]), name
        close(b[keep], want[name][keep], want[name + "_bound"][keep])


def test_keys_without_queries_do_not_matter():
    lq, lk = [150, 0, 70], [150, 40, 70]
    x = _inputs(220, 260, size=2.0 ** -19)
    clean, _ = _run(x, _cu(lq), _cu(lk))
    x[1][150:190], x[2][150:190] = math.nan, math.inf
    got, _ = _run(x, _cu(lq), _cu(lk))
    assert torch.equal(got[0], clean[0])
    for a, b in zip(got[1:], clean[1:]):
        assert torch.equal(a[:150], b[:150]) and torch.equal(a[190:], b[190:]) and (a[150:190] == 0).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_hidden_values_do_not_matter(bad):
    x = _inputs(400, 400, size=2.0 ** -19)
    x[2][7, 0, 9] = 5.0   # the largest
    clean, _ = _run(x)
    x[2][300, 0, 3] = bad
    got, _ = _run(x)
    assert torch.equal(got[0][:300], clean[0][:300]) and not torch.isfinite(got[0][300:].float()).all(-1).any()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ratio", [10, 24])
@pytest.mark.parametrize("where", [0, 150, 399])
def test_a_row_with_a_large_gradient(where, ratio, D):
    """The other rows' grad_q, and what keys that only later rows see get: the keys of later blocks of 128, from row 384 on here, and all keys where the
    row is the last one and they get most from it"""
    x = _inputs(400, 400, D=D, size=2.0 ** -19)
    x[3][where] = (x[3][where].float() * 2.0 ** ratio).half()
    got, out = _run(x)
    want = attention(*x[:3], None, None, True, D ** -0.5, grad=x[3], out16=out)
    close(got[0], want["grad_q"], want["grad_q_bound"])
    close(got[2], want["grad_v"], want["grad_v_bound"])
    later = slice((where // 128 + 1) * 128 if ratio > 10 else 0, None)
    if where < 384:
        close(got[1][later], want["grad_k"][later], want["grad_k_bound"][later])


def test_a_large_value_that_a_row_does_not_see():
    x = _inputs(400, 400, size=2.0 ** -19)
    x[2][399, 0] *= 2.0 ** 12
    got, out = _run(x)
    want = attention(*x[:3], None, None, True, 0.125, grad=x[3], out16=out)
    close(got[0][:384], want["grad_q"][:384], want["grad_q_bound"][:384])


def test_a_captured_call_follows_new_sizes():
    """what the powers of two are chosen from is formed anew by each replay"""
    lengths = [100, 300, 57]
    cu = _cu(lengths)
    x = _inputs(457, 457, H=4, G=2, size=2.0 ** -10)
    q, k, v, g = x
    out, lse = lba.lba_attention(q, k, v, cu, cu, lse=True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = lba.lba_attention_backward(g, q, k, v, out, lse, cu, cu)
    for size in (2.0 ** -20, 2.0 ** 4, 2.0 ** -16):
        g.copy_(_randn(457, 4, 64, seed=31).float() * size)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, lba.lba_attention_backward(g, q, k, v, out, lse, cu, cu)))
        want = attention(q, k, v, cu, cu, True, 0.125, grad=g, out16=out)
        for name, t in zip(NAMES, got):
            close(t, want[name], want[name + "_bound"])


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n", [1, 100, 129, 300])
def test_bits_do_not_depend_on_neighbours(n, causal):
    """a sequence alone and among others whose gradients and values are far larger"""
    x = _inputs(n, n, H=4, G=2, size=2.0 ** -19)
    alone, _ = _run(x, _cu([n]), _cu([n]), causal)
    for before, behind in ((0, 40), (77, 200), (130, 0)):
        others = [t * 8 for t in _inputs(before + behind, before + behind, H=4, G=2, size=1.0)]
        cu = _cu([before, n, behind])
        got, _ = _run([torch.cat([o[:before], t, o[before:]]) for o, t in zip(others, x)], cu, cu, causal)
        assert all(torch.equal(a, b[before:before + n]) for a, b in zip(alone, got))
