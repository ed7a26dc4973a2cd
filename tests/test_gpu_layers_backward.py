"""Backward pass of the linear and gated layers against 64 bits and against differences.  Needs a B200."""
import pytest
import torch

from helpers.layer_ref import ACTS, SLOPE_ERR, ACT_ERR, act, half_step, keep_mask, piece_err, slope
from paper_2401_14110_b200 import binding as lba
from paper_2401_14110_b200 import synth
from paper_2401_14110_b200 import LbaFormat, code_domain_formats, m4e3_input_formats

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PROD, ACC = code_domain_formats(7, 4)
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def case(M, N, K, seed, halves=1, m4e3=False, per_row=False, per_col=True):
    quantise = synth.quantise_m4e3_per_tensor if m4e3 else synth.quantise_per_tensor
    some = lambda *s: quantise(synth.gaussian(s, seed + len(out))) if min(s) else (torch.zeros(s, dtype=torch.uint8), torch.ones(1))  # noqa: E731
    out = []
    A, sa = some(M, K)
    out = [A.to(DEV), (sa * torch.linspace(0.5, 1.5, M) if per_row else sa).to(DEV)]
    for _ in range(halves):
        B, sb = some(N, K)
        out += [B.to(DEV), (sb * torch.linspace(1.5, 0.5, N) if per_col else sb).to(DEV)]
    return out


def dense(codes, scale, m4e3=False):
    return (synth.m4e3_decode if m4e3 else synth.e4m3_decode)(codes.cpu()).double() * scale.cpu().double().reshape(-1, 1)


def close(got, dz, slack, w, contract, what):
    """got against sum dz w: dz is off by `slack` and by its pieces, each of the sum's additions by 2^-23 of what it has summed"""
    want, mass = contract(dz, w), contract(dz.abs(), w.abs())
    length = dz.shape[1] if contract is rows else dz.shape[0]
    tol = piece_err(got.dtype) * mass + contract(slack, w.abs()) + (length / 16 * 3 + 18) * 2.0 ** -23 * mass
    tol = tol + half_step(got.dtype, want.abs() + tol) + 1e-300
    bad = ((got.cpu().double() - want).abs() / tol).max() if want.numel() else 0.0
    assert float(bad) <= 1, (what, float(bad))


def rows(dz, w):
    return dz @ w


def cols(dz, w):
    return dz.T @ w


def check_bias(got, dz, slack):
    tol = slack.sum(0) + (dz.shape[0] + 8) * 2.0 ** -24 * dz.abs().sum(0) + 1e-300
    assert bool(((got.cpu().double() - dz.sum(0)).abs() <= tol).all())


SHAPES = [(1, 1, 1), (1, 130, 65), (2, 16, 16), (33, 40, 72), (64, 64, 64), (129, 257, 130), (300, 65, 511), (70, 520, 264),
          (5, 1040, 48), (16, 300, 515), (17, 140, 1030), (32, 129, 144), (31, 1100, 70), (49, 260, 527),
          (50, 70, 1200)]


@pytest.mark.parametrize("out", [F32, BF16, F16])
@pytest.mark.parametrize("name", ACTS)
def test_linear_against_64_bits(name, out):
    for i, (M, N, K) in enumerate(SHAPES):
        m4e3, per_row, per_col = i % 3 == 2, i % 4 == 3, i % 2 == 0
        prod = (m4e3_input_formats(7, 4) if m4e3 else (PROD, ACC))[0]
        A, sa, B, sb = case(M, N, K, 10 * i, 1, m4e3, per_row, per_col)
        g = synth.gaussian((M, N), 500 + i).to([F32, BF16, F16][(i + len(name)) % 3])
        z = synth.gaussian((M, N), 600 + i, 2.0).to([BF16, F32, F16][i % 3])
        p = (0.0, 0.3)[i % 2]
        rng = torch.tensor([77 + i, 1 << 35], device=DEV)
        ga, gb, gc = lba.lba_linear_backward(g.to(DEV), A, B, sa, sb, prod, None if name == "none" else z.to(DEV), name, p, rng if p else None, out)
        gd = g.double()
        if p:
            gd = torch.where(keep_mask(M, N, p, *rng.tolist()), gd / (1 - p), torch.zeros_like(gd))
        dz = gd * slope(z, name)
        slack = gd.abs() * (SLOPE_ERR if name not in ("none", "relu") else 0) + dz.abs() * 2.0 ** -21   # scales and factors: below 8 roundings
        close(ga, dz, slack, dense(B, sb, m4e3), rows, (M, N, K, "a"))
        close(gb, dz, slack, dense(A, sa, m4e3), cols, (M, N, K, "b"))
        check_bias(gc, dz, slack)


@pytest.mark.parametrize("out", [F32, BF16, F16])
@pytest.mark.parametrize("name", ACTS)
def test_gated_against_64_bits(name, out):
    for i, (M, N, K) in enumerate(SHAPES):
        m4e3, per_row, per_col = i % 3 == 2, i % 4 == 3, i % 2 == 0
        prod = (m4e3_input_formats(7, 4) if m4e3 else (PROD, ACC))[0]
        A, sa, B, sb, B2, sb2 = case(M, N, K, 10 * i, 2, m4e3, per_row, per_col)
        g = synth.gaussian((M, N), 500 + i).to([F32, BF16, F16][(i + len(name)) % 3])
        pre = synth.gaussian((2, M, N), 600 + i, 2.0).to([BF16, F32, F16][i % 3])
        ga, g1, g2, c1, c2 = lba.lba_gated_backward(g.to(DEV), A, B, B2, sa, sb, sb2, prod, pre.to(DEV), name, out)
        gd, z, v = g.double(), pre[0].double(), pre[1].double()
        d1, d2 = gd * v * slope(z, name), gd * act(z, name)
        smooth = name not in ("none", "relu")
        s1 = (gd * v).abs() * (SLOPE_ERR if smooth else 0) + d1.abs() * 2.0 ** -21
        s2 = (gd * z).abs() * (ACT_ERR if smooth else 0) + d2.abs() * 2.0 ** -21
        close(ga, torch.cat([d1, d2], 1), torch.cat([s1, s2], 1), torch.cat([dense(B, sb, m4e3), dense(B2, sb2, m4e3)]), rows, (M, N, K, "a"))
        close(g1, d1, s1, dense(A, sa, m4e3), cols, (M, N, K, "gate"))
        close(g2, d2, s2, dense(A, sa, m4e3), cols, (M, N, K, "up"))
        check_bias(c1, d1, s1)
        check_bias(c2, d2, s2)


@pytest.mark.parametrize("M,N,K", [(1500, 700, 1000), (5000, 256, 260), (260, 4000, 300), (2, 3000, 1100), (20, 9000, 64), (3, 20000, 48)])
def test_many_tiles(M, N, K):
    # several tiles per multiprocessor, long sums of either product
    A, sa, B, sb, B2, sb2 = case(M, N, K, M, 2)
    g = synth.gaussian((M, N), 1)
    pre = synth.gaussian((2, M, N), 2)
    for out in (BF16, F32):
        ga, g1, g2, c1, c2 = lba.lba_gated_backward(g.to(DEV), A, B, B2, sa, sb, sb2, PROD, pre.to(DEV), "silu", out)
        d1, d2 = g.double() * pre[1].double() * slope(pre[0], "silu"), g.double() * act(pre[0], "silu")
        s1, s2 = (g * pre[1]).abs().double() * SLOPE_ERR + d1.abs() * 2.0 ** -21, (g * pre[0]).abs().double() * ACT_ERR + d2.abs() * 2.0 ** -21
        close(ga, torch.cat([d1, d2], 1), torch.cat([s1, s2], 1), torch.cat([dense(B, sb), dense(B2, sb2)]), rows, "a")
        close(g1, d1, s1, dense(A, sa), cols, "gate")
        close(g2, d2, s2, dense(A, sa), cols, "up")
        check_bias(c1, d1, s1)
        check_bias(c2, d2, s2)


def test_exact_where_nothing_rounds():
    # small whole numbers: every product and sum is exact, in each type and with either scale layout
    for M, N, K in [(130, 140, 150), (65, 64, 300)]:
        A, B = synth.small_integer_codes((M, K), 1).to(DEV), synth.small_integer_codes((N, K), 2).to(DEV)
        g = torch.randint(-2, 3, (M, N), generator=torch.Generator().manual_seed(3)).float()
        for sa, sb in [(torch.tensor([0.5]), torch.tensor([2.0])), (torch.full((M,), 0.5), torch.full((N,), 2.0))]:
            for dt in (F32, BF16, F16):
                ga, gb, gc = lba.lba_linear_backward(g.to(dt).to(DEV), A, B, sa.to(DEV), sb.to(DEV), PROD, grad_dtype=F32)
                assert torch.equal(ga.cpu().double(), g.double() @ dense(B, sb)) and torch.equal(gb.cpu().double(), g.double().T @ dense(A, sa))
                assert torch.equal(gc.cpu(), g.sum(0))


def test_repeats_give_the_same_bits_and_subsets_the_same_values():
    # a subset divides the work differently, so sums may be formed in another order: one more rounding of the result's type, and of
    # binary32 sums that the tests above bound
    A, sa, B, sb, B2, sb2 = case(200, 72, 136, 4, 2)
    g, pre = synth.gaussian((200, 72), 1).to(BF16).to(DEV), synth.gaussian((2, 200, 72), 2).to(DEV)
    one = torch.ones(1, device=DEV)
    calls = [(lambda needs: lba.lba_gated_backward(g, A, B, B2, sa, sb, sb2, PROD, pre, needs=needs), [(0,), (1, 2), (3, 4)]),
             (lambda needs: lba.lba_linear_backward(g, A, B, one, one, PROD, pre[0], "gelu", needs=needs), [(0,), (1,), (2,)])]
    for call, part in calls:
        full = call((True,) * 3)
        assert all(torch.equal(x, y) for x, y in zip(call((True,) * 3), full))
        for mask in range(8):
            needs = tuple(bool(mask >> i & 1) for i in range(3))
            got = call(needs)
            for i, need in enumerate(needs):
                for j in part[i]:
                    if not need:
                        assert got[j] is None
                    else:
                        assert bool(((got[j] - full[j]).abs() <= 2.0 ** -7 * full[j].abs() + 2.0 ** -16 * full[j].abs().max()).all())


def test_any_alignment():
    # tensors that begin at any element give what their aligned copies give, up to the order of sums
    def shifted(t, by):
        room = torch.empty(t.numel() + by, dtype=t.dtype, device=DEV)
        room[by:] = t.reshape(-1)
        return room[by:].view(t.shape)

    for M, N, K in [(5, 136, 80), (70, 136, 80), (20, 64, 1040)]:
        A, sa, B, sb, B2, sb2 = case(M, N, K, 8, 2, per_row=True)
        g, pre = synth.gaussian((M, N), 1).to(BF16).to(DEV), synth.gaussian((2, M, N), 2).to(DEV)
        for by in (1, 3):
            s = [shifted(t, by) for t in (g, A, B, B2, sa, sb, sb2, pre)]
            got = lba.lba_gated_backward(*s[:7], PROD, s[7], "gelu", F32)
            want = lba.lba_gated_backward(g, A, B, B2, sa, sb, sb2, PROD, pre, "gelu", F32)
            for x, y in zip(got, want):
                assert bool(((x - y).abs() <= 2.0 ** -16 * y.abs().max()).all())
            got = lba.lba_linear_backward(s[0], s[1], s[2], s[4], s[5], PROD, s[7][1], "silu", grad_dtype=F16)
            want = lba.lba_linear_backward(g, A, B, sa, sb, PROD, pre[1], "silu", grad_dtype=F16)
            for x, y in zip(got, want):
                assert bool(((x - y).abs() <= 2.0 ** -10 * y.abs() + 2.0 ** -14 * y.abs().max()).all())


def test_empty_sums_are_zero():
    one = torch.ones(1, device=DEV)
    for M, N, K in [(0, 24, 32), (24, 0, 32), (24, 32, 0)]:
        A, B = torch.zeros(M, K, dtype=torch.uint8, device=DEV), torch.zeros(N, K, dtype=torch.uint8, device=DEV)
        g = torch.ones(M, N, device=DEV)
        ga, gb, gc = lba.lba_linear_backward(g, A, B, one, one, PROD)
        assert ga.shape == (M, K) and gb.shape == (N, K) and not bool(ga.any()) and not bool(gb.any())
        assert torch.equal(gc, torch.full((N,), float(M), device=DEV))


@pytest.mark.parametrize("out", [F32, BF16, F16])
def test_scales_of_empty_rows(out):
    # rows and channels of zeros are quantised to the smallest normal scale; 2^-90 is as far from 1 as a user's may be, and scales of 0 stand
    # for rows of zeros.  The codes' gradients do not depend on their own scales, however small
    M, N, K = 70, 136, 96
    A, sa, B, sb, B2, sb2 = case(M, N, K, 6, 2, per_row=True)
    tiny = torch.finfo(F32).tiny
    for s, codes, stride in ((sa, A, 9), (sb, B, 7), (sb2, B2, 5)):
        s[::stride], s[1::2 * stride], s[2::2 * stride], s[3::4 * stride] = tiny, 0.0, 1.2345 * 2.0 ** -90, 1.2345 * 2.0 ** 6
        codes[::stride] = 0
    g = synth.gaussian((M, N), 1, 2.0 ** -8).to(BF16).to(DEV)
    pre = synth.gaussian((2, M, N), 2).to(BF16).to(DEV)
    dz = g.cpu().double()
    for sx in (sa, torch.ones(1, device=DEV)):
        ga, gb, _ = lba.lba_linear_backward(g, A, B, sx, sb, PROD, grad_dtype=out)
        close(ga, dz, dz.abs() * 2.0 ** -21, dense(B, sb), rows, "a")
        close(gb, dz, dz.abs() * 2.0 ** -21, dense(A, sx), cols, "b")
        assert float(gb[::7].float().abs().max()) > 0
    d1, d2 = dz * pre[1].cpu().double() * slope(pre[0].cpu(), "silu"), dz * act(pre[0].cpu(), "silu")
    s1, s2 = (dz * pre[1].cpu().double()).abs() * SLOPE_ERR + d1.abs() * 2.0 ** -21, (dz * pre[0].cpu().double()).abs() * ACT_ERR + d2.abs() * 2.0 ** -21
    for p, q in ((sb, sb2), (torch.full((1,), tiny, device=DEV), torch.full((1,), 0.75, device=DEV))):
        ga, g1, g2, _, _ = lba.lba_gated_backward(g, A, B, B2, sa, p, q, PROD, pre, "silu", out)
        close(ga, torch.cat([d1, d2], 1), torch.cat([s1, s2], 1), torch.cat([dense(B, p), dense(B2, q)]), rows, "a")
        close(g1, d1, s1, dense(A, sa), cols, "gate")
        close(g2, d2, s2, dense(A, sa), cols, "up")


def test_special_values():
    # a NaN or an infinity reaches the sums it belongs to and no other; dropped elements reach none
    A, sa, B, sb = case(64, 64, 64, 5)
    for out in (F32, BF16, F16):
        g = torch.ones(64, 64)
        g[3, 5], g[7, 9] = float("nan"), float("inf")
        ga, gb, gc = (t.cpu() for t in lba.lba_linear_backward(g.to(DEV), A, B, sa, sb, PROD, grad_dtype=out))
        bad = torch.zeros(64, dtype=torch.bool)
        bad[[3, 7]] = True
        assert torch.equal(~torch.isfinite(ga).all(1), bad) and bool(torch.isnan(ga[3]).all())
        bad[:] = False
        bad[[5, 9]] = True
        assert torch.equal(~torch.isfinite(gb).all(1), bad) and torch.equal(~torch.isfinite(gc), bad) and float(gc[9]) == float("inf")
    rng = torch.tensor([3, 4], device=DEV)
    g = torch.where(keep_mask(64, 64, 0.5, 3, 4), torch.ones(64, 64), torch.full((64, 64), float("inf")))
    assert all(bool(torch.isfinite(t).all()) for t in lba.lba_linear_backward(g.to(DEV), A, B, sa, sb, PROD, dropout=0.5, rng=rng))


WIDE = (LbaFormat(23, 8, 127, 1), LbaFormat(23, 8, 127, 1))   # a 24-bit accumulator: the layer is smooth in its scales and biases


@pytest.mark.parametrize("name", ["none", "gelu", "gelu_tanh", "silu"])
def test_against_differences(name):
    # L = sum(r * out).  dL/dbias[n] and, through the scales, sum_k grad_b[n][k] B[n][k] = dL/dscale_b[n] and likewise for scale_a
    M, N, K = 40, 24, 32
    A, sa, B, sb, B2, sb2 = case(M, N, K, 21, 2)
    bias = torch.linspace(-0.3, 0.3, N, device=DEV)
    r = synth.gaussian((M, N), 22).to(DEV)
    rng = torch.tensor([5, 6], device=DEV)
    lin = dict(activation=name, dropout=0.25, rng=rng)

    def loss(kind, sa=sa, sb=sb, bias=bias):
        if kind == "linear":
            out = lba.lba_linear(A, B, sa, sb, bias, *WIDE, **lin)
        else:
            out = lba.lba_gated(A, B, B2, sa, sb, sb2, bias, bias, *WIDE, activation=name)
        return float((r.double() * out.double()).sum())

    for kind in ("linear", "gated"):
        if kind == "linear":
            _, pre = lba.lba_linear(A, B, sa, sb, bias, *WIDE, preact=F32, **lin)
            ga, gb, gc = lba.lba_linear_backward(r, A, B, sa, sb, WIDE[0], pre, **lin)
        else:
            _, pre = lba.lba_gated(A, B, B2, sa, sb, sb2, bias, bias, *WIDE, activation=name, preact=F32)
            ga, gb, _, c1, c2 = lba.lba_gated_backward(r, A, B, B2, sa, sb, sb2, WIDE[0], pre, name)
            gc = c1 + c2   # one bias for both
        scale = float((r.abs() * (pre.abs() if kind == "linear" else pre.abs().sum(0))).sum()) + 1
        h = 2.0 ** -6     # second differences: third derivative times h^2 / 6, below 2^-12 of the terms' mass; values carry 2^-22 of it, over h
        tol = scale * (2.0 ** -12 + 2.0 ** -22 / h)
        for n in (0, 7, N - 1):
            e = torch.zeros(N, device=DEV)
            e[n] = h
            assert abs((loss(kind, bias=bias + e) - loss(kind, bias=bias - e)) / (2 * h) - float(gc[n])) <= tol
            up, down = sb.clone(), sb.clone()
            up[n] *= 1 + h
            down[n] *= 1 - h
            want = float((gb[n].cpu().double() * synth.e4m3_decode(B[n].cpu()).double()).sum()) * float(sb[n])
            assert abs((loss(kind, sb=up) - loss(kind, sb=down)) / (2 * h) - want) <= tol
        want = float((ga.cpu().double() * synth.e4m3_decode(A.cpu()).double()).sum()) * float(sa)
        assert abs((loss(kind, sa=sa * (1 + h)) - loss(kind, sa=sa * (1 - h))) / (2 * h) - want) <= tol


def test_streams_graphs_and_workspaces():
    A, sa, B, sb = case(100, 60, 80, 31)
    g, z = synth.gaussian((100, 60), 1).to(BF16).to(DEV), synth.gaussian((100, 60), 2).to(BF16).to(DEV)
    want = lba.lba_linear_backward(g, A, B, sa, sb, PROD, z, "gelu")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = lba.lba_linear_backward(g, A, B, sa, sb, PROD, z, "gelu", stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    need = lba.backward_workspace_bytes(100, 60, 80, 1, 60, BF16, "gelu")
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device=DEV)   # NaN patterns: nothing of it may be read before it is written
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = lba.lba_linear_backward(g, A, B, sa, sb, PROD, z, "gelu", workspace=ws[:need])
    for _ in range(2):
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert bool((ws[need:] == 0xFF).all())
    g.mul_(2)
    graph.replay()
    assert torch.equal(got[2], want[2] * 2) and torch.equal(got[0], want[0] * 2)
    with pytest.raises(lba.LbaError):
        lba.lba_linear_backward(g, A, B, sa, sb, PROD, z, "gelu", workspace=ws[:need - 256])


def test_a_training_step_of_both_layers():
    # gated layer -> down projection with dropout and residual, forward and backward, against the same step in 64 bits with the
    # contraction's results and the pre-activations taken as they are (the straight-through estimator)
    M, N, K = 96, 160, 64
    A, sa, B, sb, B2, sb2 = case(M, N, K, 41, 2)
    _, _, D, sd = case(M, K, N, 42)
    scale, rng = torch.tensor([0.02], device=DEV), torch.tensor([1, 2], device=DEV)
    h, pre = lba.lba_gated(A, B, B2, sa, sb, sb2, None, None, PROD, ACC, out_dtype=torch.uint8, out_scale=scale, preact=F32)
    res = synth.gaussian((M, K), 43).to(DEV)
    out, pre2 = lba.lba_linear(h, D, scale, sd, None, PROD, ACC, activation="gelu", residual=res, dropout=0.1, rng=rng, preact=F32)
    g = synth.gaussian((M, K), 44).to(DEV)
    gh, gd, gb = lba.lba_linear_backward(g, h, D, scale, sd, PROD, pre2, "gelu", 0.1, rng)
    ga, g1, g2, _, _ = lba.lba_gated_backward(gh, A, B, B2, sa, sb, sb2, PROD, pre, needs=(True, True, False))
    keep = keep_mask(M, K, 0.1, 1, 2)
    dz = torch.where(keep, g.cpu().double() / 0.9, torch.zeros(M, K).double()) * slope(pre2.cpu(), "gelu")
    wh = dz @ dense(D, sd)
    z, v = pre.cpu().double()
    d1, d2 = wh * v * slope(z, "silu"), wh * act(z, "silu")
    for got, want in [(gh, wh), (gd, dz.T @ dense(h, scale)), (gb, dz.sum(0)), (ga, d1 @ dense(B, sb) + d2 @ dense(B2, sb2)),
                      (g1, d1.T @ dense(A, sa)), (g2, d2.T @ dense(A, sa))]:
        assert float((got.cpu().double() - want).norm() / want.norm()) < 2.0 ** -16   # two slopes of 2^-18 and sums of 160 terms
    want = torch.where(keep, act(pre2.cpu(), "gelu") / 0.9, torch.zeros(M, K).double()) + res.cpu().double()
    # the activation's error, 1/0.9 of it after dropout, and three roundings: the factor, its product, the sum (values reach 200)
    tol = pre2.cpu().double().abs() * ACT_ERR / 0.9 + (want.abs() + res.cpu().double().abs()) * 3 * 2.0 ** -24
    assert bool(((out.cpu().double() - want).abs() <= tol).all())
