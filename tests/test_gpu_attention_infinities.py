"""Infinities and NaN of grad_out reach what the formula has them reach, and nothing that the mask keeps from their rows."""
import math

import pytest
import torch

from paper_2401_14110_b200 import binding as lba

pytestmark = pytest.mark.gpu


def _randn(*shape, seed=0, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Tq,Tk", [(200, 200), (300, 420), (420, 300)])
@pytest.mark.parametrize("row", [0, 5, 40, 127, 128, 150, 199])
def test_a_row_of_grad_out(row, Tq, Tk, D, dtype):
    H, G = 4, 2
    q, k, v, g = _randn(Tq, H, D, dtype=dtype), _randn(Tk, G, D, seed=1, dtype=dtype), _randn(Tk, G, D, seed=2, dtype=dtype), _randn(Tq, H, D, seed=3, dtype=dtype)
    g[7, 0, 0] = 6.0   # the largest that is finite
    out, lse = lba.lba_attention(q, k, v, lse=True)
    clean = lba.lba_attention_backward(g, q, k, v, out, lse)
    seen = max(0, row + Tk - Tq + 1)   # keys that the row sees
    for bad in (math.inf, -math.inf, math.nan):
        x = g.clone()
        x[row, 1, 3] = bad   # of the first key-value head's group
        gq, gk, gv = lba.lba_attention_backward(x, q, k, v, out, lse)
        others = [i for i in range(Tq) if i != row]
        assert torch.equal(gq[others], clean[0][others]) and torch.equal(gq[row, [0, 2, 3]], clean[0][row, [0, 2, 3]])
        for t, c in ((gk, clean[1]), (gv, clean[2])):
            assert torch.equal(t[seen:], c[seen:]) and torch.equal(t[:, 1], c[:, 1])
        dims = [d for d in range(D) if d != 3]
        assert torch.equal(gv[:seen, 0][:, dims], clean[2][:seen, 0][:, dims])
        if seen:
            assert not torch.isfinite(gq[row, 1].float()).any()
            assert not torch.isfinite(gk[:seen, 0].float()).any()
            one = gv[:seen, 0, 3].float()   # infinite, or NaN where a weight in the operand's type is 0
            assert (torch.isnan(one) | (one == bad)).all()
