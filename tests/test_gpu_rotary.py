"""Rotary positions on the GPU against the 64-bit form: layouts, parts of a head, strides, far positions, in place, the gradient."""
import pytest
import torch

from helpers.block_ref import close, rotary
from paper_2401_14110_b200 import binding as lba

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _randn(*shape, seed=0, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,kv,dim,rot", [(1, 1, 1, 2, 2), (1, 32, 8, 128, 128), (7, 3, 1, 96, 40), (33, 5, 5, 80, 80), (300, 4, 2, 64, 6), (1201, 12, 4, 128, 64),
                                                     (5, 2, 0, 256, 128), (9, 1, 1, 1024, 1024)])
def test_against_the_definition(tokens, heads, kv, dim, rot, interleaved, dtype):
    q, k = _randn(tokens, heads, dim, seed=1, dtype=dtype), _randn(tokens, kv, dim, seed=2, dtype=dtype) if kv else None
    pos = torch.randint(0, 200000, (tokens,), generator=torch.Generator("cuda").manual_seed(3), device="cuda")
    f = lba.rotary_frequencies(rot, 10000.0, "ramp", 8.0)
    for inverse, p in ((False, pos), (True, pos.to(torch.int32))):
        got = lba.lba_rotary(q, k, p, f, interleaved=interleaved, inverse=inverse, scale=1.25)
        close(got[0], *rotary(q, pos, f, interleaved, inverse, 1.25))
        if kv:
            close(got[1], *rotary(k, pos, f, interleaved, inverse, 1.25))
        else:
            assert got[1] is None


@pytest.mark.parametrize("offset", [0, 1, 4])
def test_slices_of_a_projection_and_odd_starts(offset):
    T, H, G, D = 37, 6, 2, 64
    flat = _randn(T * (H + 2 * G) * D + 8, dtype=torch.bfloat16)
    x = flat[offset:offset + T * (H + 2 * G) * D].view(T, H + 2 * G, D)
    q, k = x[:, :H], x[:, H:H + G]
    pos, f = torch.arange(T, device="cuda") + 1000, lba.rotary_frequencies(D)
    for inter in (False, True):
        want = [rotary(t, pos, f, inter, False, 1.0) for t in (q, k)]
        got = lba.lba_rotary(q, k, pos, f, interleaved=inter)
        for g, w in zip(got, want):
            close(g, *w)
    before, v = x.clone(), x[:, H + G:].clone()
    lba.lba_rotary(q, k, pos, f, out=(q, k))   # in place: only what turns changes
    close(x[:, :H], *rotary(before[:, :H], pos, f, False, False, 1.0))
    close(x[:, H:H + G], *rotary(before[:, H:H + G], pos, f, False, False, 1.0))
    assert torch.equal(x[:, H + G:], v)


def test_heads_first_and_expanded_inputs():
    q, k = _randn(3, 50, 64).transpose(0, 1), _randn(50, 1, 64).expand(50, 4, 64)
    pos, f = torch.arange(50, device="cuda"), lba.rotary_frequencies(32)
    got = lba.lba_rotary(q, k, pos, f)
    close(got[0], *rotary(q, pos, f, False, False, 1.0))
    close(got[1], *rotary(k, pos, f, False, False, 1.0))


def test_far_positions_keep_their_angles():
    f = lba.rotary_frequencies(64)
    pos = torch.tensor([0, 1, -5, 2 ** 31 - 1, 2 ** 40 + 3], device="cuda")
    q = _randn(5, 2, 64)
    want, bound = rotary(q, pos, f, False, False, 1.0)
    # a product of 2^40 radians in 64 bits is off by 2^-13, in both forms; by 2^-22 at 2^31
    bound = bound + torch.tensor([0, 0, 0, 2.0 ** -21, 2.0 ** -11], device="cuda").double()[:, None, None] * q.abs().amax() * 2
    close(lba.lba_rotary(q, None, pos, f)[0], want, bound)


def test_gradient_against_differences():
    """<rotary(x), g> has the gradient rotary^-1(g); central differences of a linear function are exact but for rounding"""
    x, g = _randn(4, 2, 16), _randn(4, 2, 16, seed=5)
    pos, f = torch.tensor([0, 3, 100, 5000], device="cuda"), lba.rotary_frequencies(12)
    grad = lba.lba_rotary(g, None, pos, f, inverse=True, scale=0.5)[0]
    for i in range(0, x.numel(), 7):
        d = torch.zeros_like(x).view(-1)
        d[i] = 1.0
        d = d.view_as(x)
        diff = ((lba.lba_rotary(x + d, None, pos, f, scale=0.5)[0] - lba.lba_rotary(x - d, None, pos, f, scale=0.5)[0]).double() * g.double()).sum() / 2
        # the two results are off by 2^-21 of |x| + 1 in the two values that differ; the others cancel
        assert abs(diff.item() - (grad.view(-1)[i].item() if i % 16 < 12 else g.view(-1)[i].item())) <= 2.0 ** -20 * (x.abs().max() + 1).item() * g.abs().max().item() * 2


def test_streams_and_graphs():
    q, k = _randn(100, 4, 64, dtype=torch.float16), _randn(100, 2, 64, dtype=torch.float16)
    pos, f = torch.arange(100, device="cuda"), lba.rotary_frequencies(64)
    want = lba.lba_rotary(q, k, pos, f)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = lba.lba_rotary(q, k, pos, f, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = lba.lba_rotary(q, k, pos, f)
    pos += 11
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, lba.lba_rotary(q, k, pos, f)))
