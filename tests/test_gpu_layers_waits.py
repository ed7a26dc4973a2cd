"""Waits of the layers' backward products that run out: what was not formed for it is NaN, all else is what it is.  Needs a B200."""
import pytest
import torch

from paper_2401_14110_b200 import binding as lba
from paper_2401_14110_b200 import code_domain_formats, synth

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PROD, ACC = code_domain_formats(7, 4)


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("which", [1, 2, 3])
def test_outputs_are_right_or_nan(which, out):
    # grad_a is two tiles with long sums, which several pairs of CTAs share; grad_b's tiles are whole
    M, N, K = 256, 4096, 512
    A, sa = (t.to(DEV) for t in synth.quantise_per_tensor(synth.gaussian((M, K), 1)))
    B, sb = (t.to(DEV) for t in synth.quantise_per_tensor(synth.gaussian((N, K), 2)))
    g, z = synth.gaussian((M, N), 3).to(DEV), synth.gaussian((M, N), 4).to(DEV)

    def grads():
        return [t.cpu() for t in lba.lba_linear_backward(g, A, B, sa, sb, PROD, z, "silu", grad_dtype=out)]

    want = grads()
    try:
        lba.set_wait_override(which)
        got = grads()
    finally:
        lba.set_wait_override(0)
    lost = [torch.isnan(t) for t in got]
    assert all(torch.equal(x[~n], y[~n]) for x, y, n in zip(got, want, lost))
    assert bool(lost[0].any()) and not bool(lost[2].any())
    if which == 1:
        assert bool(lost[0].all()) and not bool(lost[1].any())
    else:
        assert bool(lost[1].any()) and not bool(lost[1].all())
    assert all(torch.equal(x, y) for x, y in zip(grads(), want))
