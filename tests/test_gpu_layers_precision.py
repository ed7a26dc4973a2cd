"""How exactly the layers' backward pass holds dz, and their activations the tails.  Needs a B200."""
import math

import pytest
import torch

from helpers.layer_ref import half_step
from paper_2401_14110_b200 import binding as lba
from paper_2401_14110_b200 import code_domain_formats, synth

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PROD, ACC = code_domain_formats(7, 4)
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16

# A cut to 8 significant bits leaves less than 2^-7 of dz, rounding that to 8 bits 2^-8 of it; a third piece leaves nothing of 24 bits.
PIECES_ERR = {BF16: 2.0 ** -15, F16: 0.0}


def share_off(got, dz, w, sums):
    """the share of elements that are further from sum dz w than PIECES_ERR, the additions and the result's own rounding allow"""
    want, mass = sums(dz, w), sums(dz.abs(), w.abs())
    length = dz.shape[1] if sums is rows else dz.shape[0]
    # scales: dz times a fraction of each, and one of them divided out, 4 roundings of 2^-24; every addition of 16 products 2^-23 of what is summed
    tol = (PIECES_ERR[got.dtype] + 2.0 ** -22 + (length / 16 * 3 + 18) * 2.0 ** -23) * mass
    tol = tol + half_step(got.dtype, want.abs() + tol)
    return float(((got.double() - want).abs() > tol).double().mean())


def rows(dz, w):
    return dz @ w


def cols(dz, w):
    return dz.T @ w


@pytest.mark.parametrize("out", [BF16, F16])
@pytest.mark.parametrize("M,N,K", [(1, 50, 300), (1, 4096, 48), (3, 900, 130), (16, 2048, 64), (40, 70, 96),      # one launch
                                   (3000, 16, 64), (65, 40, 200), (100, 129, 70), (300, 200, 130), (1000, 64, 48), (20, 64, 4200)])
def test_dz_keeps_twice_the_results_bits(M, N, K, out):
    # one rounding of dz to the result's own bits shows in single terms and in sums of any length: at sizes of both kernels
    A, sa = synth.quantise_per_tensor(synth.gaussian((M, K), 1))
    B, sb = synth.quantise_per_tensor(synth.gaussian((N, K), 2))
    sa, sb = sa * torch.linspace(0.5, 1.5, M), sb * torch.linspace(1.5, 0.5, N)
    g = synth.gaussian((M, N), 3)
    x, w, dz = synth.e4m3_decode(A).double() * sa.double()[:, None], synth.e4m3_decode(B).double() * sb.double()[:, None], g.double()
    ga, gb, _ = (t.cpu() for t in lba.lba_linear_backward(g.to(DEV), A.to(DEV), B.to(DEV), sa.to(DEV), sb.to(DEV), PROD, grad_dtype=out))
    assert share_off(ga, dz, w, rows) == 0 and share_off(gb, dz, x, cols) == 0
    if out is BF16:  # the same sums with dz rounded once do not pass
        once = g.to(BF16).double()
        assert max(share_off((once @ w).to(out), dz, w, rows), share_off((once.T @ x).to(out), dz, x, cols)) > 0.05


def test_gelu_keeps_its_tail():
    # z P(z) and its slope are small below -3 and have all the bits of their type there.  Relative error: the sum of eight terms 28 roundings of
    # 2^-24 at most, 1.7e-6, its own fit 2.6e-8 (1 + z^2), t 1.8e-7, the exponential 2.4e-7 and of its argument's three roundings 9e-8 z^2, two
    # products 1.2e-7: below (5 + z^2 / 4) 2^-21.  Slopes: of both terms' magnitudes, with one more product and one more sum.
    z = -torch.cat([torch.linspace(0.01, 12, 4001), torch.linspace(3, 6, 4000)])
    N, z64 = z.numel(), z.double()
    rel = (5 + z64 ** 2 / 4) * 2.0 ** -21
    P, density = 0.5 * torch.special.erfc(-z64 / math.sqrt(2)), torch.exp(-z64 * z64 / 2) / math.sqrt(2 * math.pi)
    one, codes = torch.ones(1, device=DEV), torch.zeros(N, 16, dtype=torch.uint8, device=DEV)
    for out in (F32, BF16):
        got = lba.lba_linear(codes[:1], codes, one, one, z.to(DEV), PROD, ACC, activation="gelu", out_dtype=out).cpu().double()[0]
        want = z64 * P
        assert bool(((got - want).abs() <= want.abs() * rel + half_step(out, want * (1 + rel))).all())
    gated, pre = lba.lba_gated(codes[:1], codes, codes, one, one, one, z.to(DEV), torch.ones(N, device=DEV), PROD, ACC, activation="gelu", preact=F32)
    assert torch.equal(pre[0, 0].cpu(), z) and bool(((gated.cpu().double()[0] - z64 * P).abs() <= (z64 * P).abs() * (rel + 2.0 ** -24) + 2.0 ** -126).all())
    want, mass = P + z64 * density, P + z64.abs() * density
    for needs in ((False, False, True), (True, True, True)):   # two launches, and the one of few rows
        dz = lba.lba_linear_backward(torch.ones(1, N, device=DEV), codes[:1], codes, one, one, PROD, z[None].to(DEV), "gelu", needs=needs)[2]
        assert bool(((dz.cpu().double() - want).abs() <= mass * (rel + 2.0 ** -22) + 2.0 ** -126).all())
