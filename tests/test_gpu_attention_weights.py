"""Weights far below their row's largest in prompts of binary16."""
import pytest
import torch

from helpers.block_ref import attention, close
from paper_2401_14110_b200 import binding as lba

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("where", ["first", "last", "middle"])
@pytest.mark.parametrize("T", [300, 8000])
@pytest.mark.parametrize("down", [16, 20, 21])
def test_many_small_weights_beside_a_large_one(down, T, where):
    """One key with a value of 0 has almost all the weight, each other one 2^(0.45 - down) of it: the output is made of those, whose products are as exact as any,
    down to 2^-21 = 2^-(14 + 7) where binary16's normal numbers end"""
    q, k, v = (torch.zeros(t, 1, 64, device="cuda", dtype=torch.float16) for t in (2, T, T))
    q[:, 0, 0] = 1.0
    k[:, 0, 0] = 0.45 - down
    v[:, 0] = torch.rand(T, 64, generator=torch.Generator("cuda").manual_seed(1), device="cuda") + 1.0
    at = {"first": 0, "last": T - 1, "middle": T // 2}[where]
    k[at], v[at] = 0.0, 0.0
    scale = 0.6931471805599453
    out, lse = lba.lba_attention(q, k, v, causal=False, scale=scale, lse=True)
    want = attention(q, k, v, None, None, False, scale)
    close(out, want["out"], want["out_bound"])
    close(lse, want["lse"], want["lse_bound"])
    codes = lba.lba_attention(q, k, v, causal=False, scale=scale, out_dtype=torch.uint8, out_scale=torch.tensor([2.0 ** -20], device="cuda"))
    x = want["out"] * 2.0 ** 20
    close(codes.view(torch.float8_e4m3fn), x.clamp(-448, 448), (2.0 ** -4 * x.abs()).clamp_min(2.0 ** -10) * 1.001 + want["out_bound"] * 2.0 ** 20)
