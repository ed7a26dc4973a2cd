"""Linear and gated layers: the contraction bit for bit, everything after it against 64 bits.  Needs a B200."""
import threading

import numpy as np
import pytest
import torch

from helpers.layer_ref import ACT_ERR, ACTS, act, half_step, keep_mask
from oracle import lba_oracle as orc
from paper_2401_14110_b200 import binding as lba
from paper_2401_14110_b200 import synth
from paper_2401_14110_b200 import (LbaFormat, fixed_point_format, code_domain_formats, m4e3_input_formats, M7E4_PAPER, ORDER_SEQUENTIAL as SEQ,
                                   ORDER_CHUNKED as CHK)

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

FORMATS = {
    "m7e4": code_domain_formats(7, 4),
    "m7e4_paper": M7E4_PAPER,                                         # Q_prod saturates
    "m5e6": code_domain_formats(5, 6),                                # Q_prod cuts
    "m2e5": code_domain_formats(2, 5),                                # more than A's scales carry
    "m8e6": code_domain_formats(8, 6),                                # product and sum fused
    "m7e4_rne": code_domain_formats(7, 4, rounding=1),                # through bfloat16 in chunks of 16
    "m10e6_rne": code_domain_formats(10, 6, rounding=1),
    "m12e5_rne": code_domain_formats(12, 5, rounding=1),              # generic kernel
    "wide_rne": (LbaFormat(23, 8, 127, 1), LbaFormat(23, 8, 127, 1)),
    "m4e3_bytes": m4e3_input_formats(7, 4),
    "fixed": (fixed_point_format(16, 2), fixed_point_format(18, 2)),
    "fixed_wrap": (fixed_point_format(12, 0, True), fixed_point_format(14, 0, True)),
}


def bits(t):
    return t.detach().cpu().contiguous().view(torch.int32)


def inputs(M, N, K, seed, prod, copies=1):
    """A, B ... as codes of the call's format with scales, per tensor and per channel"""
    m4e3 = bool(prod.flags & 4)
    a = synth.gaussian((M, K), seed)
    A, sa = (synth.quantise_m4e3_per_tensor if m4e3 else synth.quantise_per_tensor)(a) if M * K else (a.to(torch.uint8), torch.ones(1))
    out = [A.to(DEV), sa.to(DEV)]
    for i in range(copies):
        b = synth.gaussian((N, K), seed + 1 + i, std=max(K, 1) ** -0.5)
        B, sb = (synth.quantise_m4e3_per_tensor if m4e3 else synth.quantise_per_tensor)(b) if N * K else (b.to(torch.uint8), torch.ones(1))
        out += [B.to(DEV), (sb * torch.linspace(0.5, 1.5, N)).to(DEV), torch.linspace(-0.5, 0.5, N).to(DEV)]
    return out


SHAPES = [(1, 1, 1), (1, 17, 16), (1, 250, 333), (3, 5, 33), (16, 16, 32), (37, 70, 96), (130, 67, 161), (5, 6, 0)]


@pytest.mark.parametrize("order,chunk", [(CHK, 16), (SEQ, 16), (CHK, 32), (CHK, 5)])
@pytest.mark.parametrize("name", list(FORMATS))
def test_contraction_is_that_of_the_gemm(name, order, chunk):
    prod, acc = FORMATS[name]
    for M, N, K in SHAPES:
        A, sa, B, sb, bias, B2, sb2, bias2 = inputs(M, N, K, 11 * M + N, prod, 2)
        z = lba.lba_gemm(A, B, sa, sb, bias, prod, acc, order, chunk)
        v = lba.lba_gemm(A, B2, sa, sb2, bias2, prod, acc, order, chunk)
        out, pre = lba.lba_linear(A, B, sa, sb, bias, prod, acc, order, chunk, preact=torch.float32)
        assert torch.equal(bits(out), bits(z)) and torch.equal(bits(pre), bits(z)), (M, N, K)
        out, pre = lba.lba_gated(A, B, B2, sa, sb, sb2, bias, bias2, prod, acc, order, chunk, "none", preact=torch.float32)
        assert torch.equal(bits(pre[0]), bits(z)) and torch.equal(bits(pre[1]), bits(v)), (M, N, K)
        assert torch.equal(bits(out), bits(z * v)), (M, N, K)


@pytest.mark.parametrize("order,tiles", [(CHK, (0, 1, 2, 3, 5, 6, 7)), (SEQ, (0, 1, 2, 3, 10))])
@pytest.mark.parametrize("name", ["m7e4", "m5e6", "m7e4_rne", "m10e6_rne"])
def test_every_tile(name, order, tiles):
    prod, acc = FORMATS[name]
    for M, N, K in [(150, 139, 176), (33, 140, 95)]:
        A, sa, B, sb, bias, B2, sb2, bias2 = inputs(M, N, K, M, prod, 2)
        n = lambda t: t.cpu().numpy()  # noqa: E731
        z = torch.from_numpy(orc.gemm(n(A), n(B), n(sa), n(sb), n(bias), prod.as_tuple(), acc.as_tuple(), order, 16))
        v = torch.from_numpy(orc.gemm(n(A), n(B2), n(sa), n(sb2), n(bias2), prod.as_tuple(), acc.as_tuple(), order, 16))
        try:
            for t in tiles:
                lba.set_tile_override(t)
                got = lba.lba_linear(A, B, sa, sb, bias, prod, acc, order, 16)
                assert torch.equal(bits(got), bits(z)), (t, M, N, K)
                _, pre = lba.lba_gated(A, B, B2, sa, sb, sb2, bias, bias2, prod, acc, order, 16, preact=torch.float32)
                assert torch.equal(bits(pre), bits(torch.stack([z, v]))), (t, M, N, K)
        finally:
            lba.set_tile_override(-1)


@pytest.mark.parametrize("name", ["m7e4", "m7e4_paper", "m5e6", "m2e5", "m8e6", "m7e4_rne", "m10e6_rne", "m4e3_bytes"])
def test_few_rows(name):
    # the kernel for few rows against the tiles, bit for bit: several rounds of 512 k and trips around its rings, ragged ends of
    # columns and rounds, one pair of columns and many; Gaussian operands, and codes whose sums saturate in both hierarchies
    prod, acc = FORMATS[name]
    for M, N, K in [(1, 1, 32), (1, 2, 512), (2, 3, 528), (1, 40, 5120), (3, 601, 1040), (5, 2048, 1536), (8, 77, 2064), (16, 330, 4096), (15, 4500, 544),
                    (1, 9000, 1024), (16, 2, 16384), (17, 64, 512)]:
        for wild in (False, True):
            A, sa, B, sb, bias, B2, sb2, bias2 = inputs(M, N, K, 3 * M + N + K, prod, 2)
            if wild:
                A, B = (synth.random_codes(t.shape, 5 + i).to(DEV) for i, t in enumerate((A, B)))
            z = lba.lba_gemm(A, B, sa, sb, bias, prod, acc)
            v = lba.lba_gemm(A, B2, sa, sb2, bias2, prod, acc)
            got = lba.lba_linear(A, B, sa, sb, bias, prod, acc)
            assert torch.equal(bits(got), bits(z)), (M, N, K, wild)
            out, pre = lba.lba_gated(A, B, B2, sa, sb, sb2, bias, bias2, prod, acc, activation="none", preact=torch.float32)
            assert torch.equal(bits(pre), bits(torch.stack([z, v]))) and torch.equal(bits(out), bits(z * v)), (M, N, K, wild)


def check(got, want, err, scale=None, m4e3=False):
    """got: a layer's output; want: what it should hold, in 64 bits, off by at most err before its last rounding"""
    if got.dtype == torch.uint8:
        top, kind = (synth.M4E3_MAX, "m4e3") if m4e3 else (synth.E4M3_MAX, "e4m3")
        q = (want / scale).clamp(-top, top)
        got = (synth.m4e3_decode if m4e3 else synth.e4m3_decode)(got.cpu()).double()
        tol = half_step(kind, q) + err / scale + q.abs() * 2.0 ** -24   # (the division rounds)
        assert bool(((got - q).abs() <= tol).all())
    else:
        tol = half_step(got.dtype, want.abs() + err) + err
        assert bool(((got.cpu().double() - want).abs() <= tol).all()), float(((got.cpu().double() - want).abs() / tol).max())


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16, torch.float16, torch.uint8])
@pytest.mark.parametrize("name", ACTS)
def test_linear_epilogue(name, out_dtype):
    for i, (M, N, K) in enumerate([(1, 7, 40), (1, 64, 64), (35, 66, 48), (130, 201, 33), (64, 128, 64)]):
        for fmt in ("m7e4", "m4e3_bytes"):
            prod, acc = FORMATS[fmt]
            A, sa, B, sb, bias = inputs(M, N, K, 100 + i, prod)
            p = (0.0, 0.1, 0.5)[i % 3]
            res = [None, torch.float32, torch.bfloat16, torch.float16][(i + 1) % 4]
            res = None if res is None else synth.gaussian((M, N), 7).to(res).to(DEV)
            rng = torch.tensor([(5 << 33) + 12345 * i, (3 << 40) + i], device=DEV)
            z = lba.lba_gemm(A, B, sa, sb, bias, prod, acc).cpu().double()
            scale = torch.tensor([1.5 / 448], device=DEV)
            pre_dtype = [torch.bfloat16, torch.float32, torch.float16][i % 3]
            got, pre = lba.lba_linear(A, B, sa, sb, bias, prod, acc, activation=name, residual=res, dropout=p, rng=rng if p else None,
                                      out_dtype=out_dtype, out_scale=scale, preact=pre_dtype)
            assert torch.equal(pre.cpu(), z.float().to(pre_dtype))
            want, err = act(z, name), z.abs() * (0 if name in ("none", "relu") else ACT_ERR)
            if p:
                keep = keep_mask(M, N, p, *rng.tolist())
                assert 0 < int(keep.sum()) or M * N < 10
                want = torch.where(keep, want / (1 - p), torch.zeros_like(want))
                err = err / (1 - p) + want.abs() * 2.0 ** -23     # the factor's rounding and the product's
            if res is not None:
                want = want + res.cpu().double()
                err = err + (want.abs() + err) * 2.0 ** -24
            check(got, want, err, float(scale), fmt == "m4e3_bytes")


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16, torch.float16, torch.uint8])
@pytest.mark.parametrize("name", ACTS)
def test_gated_epilogue(name, out_dtype):
    for i, (M, N, K) in enumerate([(1, 7, 40), (1, 64, 64), (35, 66, 48), (130, 101, 33), (64, 128, 64)]):
        for fmt in ("m7e4", "m4e3_bytes"):
            prod, acc = FORMATS[fmt]
            A, sa, B, sb, bias, B2, sb2, bias2 = inputs(M, N, K, 200 + i, prod, 2)
            bias, bias2 = (bias, bias2) if i % 2 else (None, None)
            z = lba.lba_gemm(A, B, sa, sb, bias, prod, acc).cpu().double()
            v = lba.lba_gemm(A, B2, sa, sb2, bias2, prod, acc).cpu().double()
            scale = torch.tensor([1.5 / 448], device=DEV)
            pre_dtype = [torch.bfloat16, torch.float32, torch.float16][i % 3]
            got, pre = lba.lba_gated(A, B, B2, sa, sb, sb2, bias, bias2, prod, acc, activation=name, out_dtype=out_dtype, out_scale=scale,
                                     preact=pre_dtype)
            assert torch.equal(pre.cpu(), torch.stack([z, v]).float().to(pre_dtype))
            want = act(z, name) * v
            err = (z * v).abs() * (0 if name in ("none", "relu") else ACT_ERR) + want.abs() * 2.0 ** -23
            check(got, want, err, float(scale), fmt == "m4e3_bytes")


def test_codes_at_every_border():
    # values on, next to and between the borders of every code, saturation, signs and infinities, through the residual of a layer of K = 0
    for m4e3 in (False, True):
        prod, acc = FORMATS["m4e3_bytes" if m4e3 else "m7e4"]
        codes = torch.tensor([c for c in range(128) if m4e3 or c != 127], dtype=torch.uint8)
        v = (synth.m4e3_decode if m4e3 else synth.e4m3_decode)(codes).sort().values
        mid = (v[1:] + v[:-1]) / 2
        near = torch.cat([v, mid, torch.nextafter(mid, mid * 2), torch.nextafter(mid, mid * 0), v[-1:] * 1.03, v[-1:] * 100, torch.tensor([float("inf"), 1e-30])])
        near = torch.cat([near, -near])[None].contiguous()
        N = near.shape[1]
        A, B = torch.zeros(1, 0, dtype=torch.uint8, device=DEV), torch.zeros(N, 0, dtype=torch.uint8, device=DEV)
        one = torch.ones(1, device=DEV)
        got = lba.lba_linear(A, B, one, one, None, prod, acc, residual=near.to(DEV), out_dtype=torch.uint8, out_scale=one).cpu()
        if m4e3:
            grid = torch.cat([v, -v])
            gotv = synth.m4e3_decode(got).double()
            x = near.double().clamp(-248, 248)
            best = (x[0][:, None] - grid.double()[None]).abs().min(dim=1).values
            assert torch.equal((gotv[0] - x[0]).abs(), best)
            tie = torch.isin(near[0].abs(), mid)
            assert bool(((got[0][tie] & 1) == 0).all())
        else:
            assert torch.equal(got & 0x7F, synth.e4m3_encode(near) & 0x7F) and torch.equal(synth.e4m3_decode(got), synth.e4m3_decode(synth.e4m3_encode(near)))


def test_special_values_pass_and_dropped_ones_do_not():
    prod, acc = FORMATS["m7e4"]
    A, sa, B, sb, _ = inputs(4, 8, 16, 3, prod)
    bias = torch.tensor([float("nan"), float("inf"), -float("inf"), 0, 1e38, -1e38, 100, -100], device=DEV)
    for name in ACTS:
        got = lba.lba_linear(A, B, sa, sb, bias, prod, acc, activation=name).cpu()
        z = lba.lba_gemm(A, B, sa, sb, bias, prod, acc).cpu()
        want = act(z.float().double(), name).float()
        assert torch.equal(torch.isnan(got[:, 0]), torch.isnan(want[:, 0])) and bool((got[:, 1] == float("inf")).all())
        assert torch.allclose(got[:, 3:], want[:, 3:], rtol=1e-5, atol=1e-5) and not bool(torch.isnan(got[:, 3:]).any()), name
    rng = torch.tensor([1, 2], device=DEV)
    got = lba.lba_linear(A, B, sa, sb, bias, prod, acc, dropout=0.5, rng=rng).cpu()
    assert bool((got[~keep_mask(4, 8, 0.5, 1, 2)] == 0).all())


def test_columns_behind_the_last_and_the_residual_in_place():
    prod, acc = FORMATS["m7e4"]
    A, sa, B, sb, bias = inputs(9, 13, 48, 5, prod)
    store = torch.full((9 * 13 + 64,), 7.0, dtype=torch.bfloat16, device=DEV)
    out = store[:9 * 13].view(9, 13)
    r = synth.gaussian((9, 13), 8).to(torch.bfloat16).to(DEV)
    want = lba.lba_linear(A, B, sa, sb, bias, prod, acc, residual=r, out_dtype=torch.bfloat16)
    out.copy_(r)
    assert lba.lba_linear(A, B, sa, sb, bias, prod, acc, residual=out, out=out) is out
    assert torch.equal(out, want) and bool((store[9 * 13:] == 7).all())
    odd = store[1:1 + 9 * 13].view(9, 13)   # an output that no vector store can reach
    lba.lba_linear(A, B, sa, sb, bias, prod, acc, residual=r, out=odd)
    assert torch.equal(odd, want)


def test_streams_and_graphs():
    prod, acc = FORMATS["m7e4"]
    A, sa, B, sb, bias = inputs(64, 64, 64, 6, prod)
    rng = torch.tensor([9, 0], device=DEV)
    side = torch.cuda.Stream()
    out = torch.empty(64, 64, device=DEV)
    side.wait_stream(torch.cuda.current_stream())
    lba.lba_linear(A, B, sa, sb, bias, prod, acc, dropout=0.25, rng=rng, out=out, stream=side)
    side.synchronize()
    first = out.clone()
    assert torch.equal(first == 0, ~keep_mask(64, 64, 0.25, 9, 0).to(DEV))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lba.lba_linear(A, B, sa, sb, bias, prod, acc, dropout=0.25, rng=rng, out=out)
    for offset in (0, 5):
        rng[1] = offset
        g.replay()
        assert torch.equal((out == 0).cpu(), ~keep_mask(64, 64, 0.25, 9, offset))
    assert not torch.equal(out, first)


def test_calls_of_several_threads():
    # launches of different sizes and kernels from threads with streams of their own
    prod, acc = FORMATS["m7e4"]
    sizes = [(1, 700, 256), (7, 90, 1040), (12, 2000, 64), (40, 200, 512), (3, 64, 4096)]
    data = [inputs(M, N, K, 20 + i, prod) for i, (M, N, K) in enumerate(sizes)]
    grads = [synth.gaussian((M, N), i).to(torch.bfloat16).to(DEV) for i, (M, N, _) in enumerate(sizes)]

    def calls(i, stream=None):
        A, sa, B, sb, bias = data[i]
        y = lba.lba_linear(A, B, sa, sb, bias, prod, acc, activation="gelu", stream=stream)
        return (y, *lba.lba_linear_backward(grads[i], A, B, sa, sb, prod, y, "gelu", stream=stream))

    want = [calls(i) for i in range(len(sizes))]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(100):
                    got = calls(i)
                stream.synchronize()
                wrong.extend((i, j) for j, (x, y) in enumerate(zip(got, want[i])) if not torch.equal(x, y))
        except Exception as e:  # noqa: BLE001
            wrong.append((i, e))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(sizes))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_two_layers_in_a_row_as_a_network_uses_them():
    # codes -> gated layer -> codes -> down projection + residual: the codes go from kernel to kernel
    prod, acc = FORMATS["m7e4"]
    A, sa, B, sb, _, B2, sb2, _ = inputs(20, 96, 64, 7, prod, 2)
    _, _, D, sd, bias = inputs(20, 64, 96, 8, prod)
    res = synth.gaussian((20, 64), 9).to(torch.bfloat16).to(DEV)
    scale = torch.tensor([0.01], device=DEV)
    h = lba.lba_gated(A, B, B2, sa, sb, sb2, None, None, prod, acc, out_dtype=torch.uint8, out_scale=scale)
    out = lba.lba_linear(h, D, scale, sd, bias, prod, acc, residual=res, out_dtype=torch.bfloat16)
    f = lba.lba_gated(A, B, B2, sa, sb, sb2, None, None, prod, acc)
    assert torch.equal(synth.e4m3_encode(f / scale) & 0x7F, h & 0x7F)
    want = lba.lba_gemm(h, D, scale, sd, bias, prod, acc) + res.float()
    assert torch.equal(out, want.to(torch.bfloat16))


def test_native_calls_are_those_of_the_ctypes_path(monkeypatch):
    prod, acc = FORMATS["m7e4"]
    A, sa, B, sb, bias, B2, sb2, bias2 = inputs(20, 40, 64, 12, prod, 2)
    g, rng, scale = synth.gaussian((20, 40), 1).to(DEV), torch.tensor([3, 4], device=DEV), torch.tensor([0.1], device=DEV)
    pre, buf = torch.empty(2, 20, 40, device=DEV), torch.empty(20, 40, dtype=torch.bfloat16, device=DEV)

    def calls():
        yield lba.lba_linear(A, B, sa, sb, bias, prod, acc)
        yield from lba.lba_linear(A, B, sa, sb, bias, prod, acc, SEQ, 16, "gelu", g, 0.5, rng, torch.uint8, scale, torch.float16)
        yield lba.lba_linear(A, B, sa, sb, torch.nn.Parameter(bias), prod.as_tuple(), acc.as_tuple(), out=buf).clone()
        yield lba.lba_gated(A, B, B2, sa, sb, sb2, None, None, prod, acc, out_dtype=torch.bfloat16)
        yield from (t.clone() for t in lba.lba_gated(A, B, B2, sa, sb, sb2, bias, bias2, prod, acc, activation="gelu_tanh", preact=pre, out=buf))
        yield from lba.lba_linear_backward(g, A, B, sa, sb, prod, pre[0], "silu", 0.5, rng, torch.bfloat16)
        yield from (t for t in lba.lba_linear_backward(g, A, B, sa, sb, prod, needs=(False, True, False)) if t is not None)
        yield from lba.lba_gated_backward(g, A, B, B2, sa, sb, sb2, prod, pre)

    assert lba._native
    count = [0]
    native = lba._native

    class Counting:
        def __getattr__(self, name):
            def call(*args):
                r = getattr(native, name)(*args)
                count[0] += r is not None
                return r
            return call
    monkeypatch.setattr(lba, "_native", Counting())
    first = list(calls())
    assert count[0] == 8                      # every one of them is regular
    monkeypatch.setattr(lba, "_native", None)
    assert all(torch.equal(x, y) for x, y in zip(first, list(calls()), strict=True))


def test_what_is_refused_with_tensors_on_the_gpu():
    prod, acc = FORMATS["m7e4"]
    A, sa, B, sb, bias = inputs(4, 8, 16, 13, prod)
    for kw in [dict(out=torch.empty(4, 9, device=DEV)), dict(residual=torch.empty(8, 4, device=DEV)), dict(preact=torch.empty(4, 9, device=DEV)),
               dict(activation="swish"), dict(out=torch.empty(4, 8))]:
        with pytest.raises((ValueError, TypeError)):
            lba.lba_linear(A, B, sa, sb, bias, prod, acc, **kw)
    for kw in [dict(out=torch.empty(8, 4, device=DEV).t()), dict(residual=torch.empty(8, 4, device=DEV).t()), dict(dropout=0.5),
               dict(dropout=0.5, rng=torch.zeros(3, dtype=torch.int64, device=DEV)), dict(out_dtype=torch.uint8), dict(out_dtype=torch.float64)]:
        with pytest.raises(TypeError):
            lba.lba_linear(A, B, sa, sb, bias, prod, acc, **kw)
    for p in (1.0, -0.5):
        with pytest.raises(lba.LbaError):
            lba.lba_linear(A, B, sa, sb, bias, prod, acc, dropout=p, rng=torch.zeros(2, dtype=torch.int64, device=DEV))
    with pytest.raises(ValueError):
        lba.lba_linear(A, B, sa, sb, bias[:7], prod, acc)
    with pytest.raises(lba.LbaError):
        lba.lba_linear(A, B, sa, sb[:7], bias, prod, acc)
    with pytest.raises(lba.LbaError):
        lba.lba_gated(A, B, B, sa, sb, sb, bias, None, prod, acc)
