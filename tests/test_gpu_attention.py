"""Attention over prompts on the GPU against the 64-bit form: packed sequences, masks that leave rows empty, head layouts, what a mask hides."""
import math

import pytest
import torch

from helpers.block_ref import HALF, attention, close
from paper_2401_14110_b200 import FLAG_INPUT_M4E3, LbaFormat
from paper_2401_14110_b200 import binding as lba

pytestmark = pytest.mark.gpu


def _randn(*shape, seed=0, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(dtype)


def _cu(lengths, first=0):
    return torch.tensor([first] + [first + sum(lengths[:i + 1]) for i in range(len(lengths))], dtype=torch.int32, device="cuda")


def _check(q, k, v, cu_q, cu_k, causal, scale=None):
    out, lse = lba.lba_attention(q, k, v, cu_q, cu_k, causal=causal, scale=scale, lse=True)
    want = attention(q, k, v, cu_q, cu_k, causal, q.shape[2] ** -0.5 if scale is None else scale)
    inside = ~torch.isnan(want["lse"][0])
    close(out[inside], want["out"][inside], want["out_bound"][inside])
    close(lse[:, inside], want["lse"][:, inside], want["lse_bound"][:, inside])
    return out, lse


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [8, 24, 64, 72, 80, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_head_sizes_and_groups(dim, causal, dtype):
    T, H, G = 300, 6, 2
    _check(_randn(T, H, dim, dtype=dtype), _randn(T, G, dim, seed=1, dtype=dtype), _randn(T, G, dim, seed=2, dtype=dtype), None, None, causal)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("T", [1, 2, 63, 127, 128, 129, 255, 256, 257, 384, 511, 640, 1025])
def test_lengths(T, causal):
    _check(_randn(T, 2, 64), _randn(T, 2, 64, seed=1), _randn(T, 2, 64, seed=2), None, None, causal)


@pytest.mark.parametrize("causal", [False, True])
def test_packed_sequences_of_every_kind(causal):
    lq = [1, 0, 200, 128, 5, 0, 300, 17, 256, 0]
    lk = [1, 7, 200, 64, 500, 0, 0, 300, 255, 0]
    _check(_randn(sum(lq), 4, 128), _randn(sum(lk), 2, 128, seed=1), _randn(sum(lk), 2, 128, seed=2), _cu(lq), _cu(lk), causal)


def test_many_short_sequences():
    lengths = [(i * 37) % 50 for i in range(100)]
    T = sum(lengths)
    _check(_randn(T, 3, 32), _randn(T, 1, 32, seed=1), _randn(T, 1, 32, seed=2), _cu(lengths), _cu(lengths), True)


def test_rows_of_no_sequence_are_left():
    T, first, lengths = 200, 11, [50, 60]
    q, k, v = _randn(T, 2, 64), _randn(T, 2, 64, seed=1), _randn(T, 2, 64, seed=2)
    for t in (q, k, v):   # what lies outside is not looked at
        t[:first], t[first + 110:] = math.nan, math.nan
    cu = _cu(lengths, first)
    out, lse = torch.full_like(q, 7.0), torch.full((2, T), 7.0, device="cuda")
    got = lba.lba_attention(q, k, v, cu, cu, lse=lse, out=out)
    assert got[0] is out and got[1] is lse
    want = attention(q, k, v, cu, cu, True, 0.125)
    inside = slice(first, first + 110)
    close(out[inside], want["out"][inside], want["out_bound"][inside])
    close(lse[:, inside], want["lse"][:, inside], want["lse_bound"][:, inside])
    outside = torch.ones(T, dtype=torch.bool, device="cuda")
    outside[inside] = False
    assert (out[outside] == 7).all() and (lse[:, outside] == 7).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("where", [0, 3, 130, 199, 255, 256, 300])
def test_infinities_and_nan_count_only_where_they_are_seen(where, dtype):
    """A key or value that the causal mask hides changes nothing; rows that see it get what the formula gives"""
    T, H, D = 310, 2, 64
    lengths = [310, 90]
    q, k, v = _randn(400, H, D, dtype=dtype), _randn(400, 1, D, seed=1, dtype=dtype), _randn(400, 1, D, seed=2, dtype=dtype)
    cu = _cu(lengths)
    clean = lba.lba_attention(q, k, v, cu, cu)
    v[where, 0, 5], v[where, 0, 6], v[where, 0, 63] = math.inf, math.nan, -math.inf
    out = lba.lba_attention(q, k, v, cu, cu)
    assert torch.equal(out[:where], clean[:where]) and torch.equal(out[T:], clean[T:])
    seen = out[where:T]
    assert torch.isnan(seen[..., 6]).all()
    for col, sign in ((5, 1), (63, -1)):   # infinite, or NaN where a weight in the operand's type is 0
        assert ((seen[..., col] == sign * math.inf) | torch.isnan(seen[..., col])).all()
    other = [c for c in range(D) if c not in (5, 6, 63)]
    assert torch.equal(seen[..., other], clean[where:T][..., other])
    k[where] = math.nan
    v[where] = 1.0
    out = lba.lba_attention(q, k, v, cu, cu)
    assert torch.equal(out[:where], clean[:where]) and torch.equal(out[T:], clean[T:]) and torch.isnan(out[where:T]).all()


def test_a_neighbours_values_do_not_leak():
    lengths = [100, 60]
    q, k, v = _randn(160, 2, 64), _randn(160, 2, 64, seed=1), _randn(160, 2, 64, seed=2)
    cu = _cu(lengths)
    for causal in (False, True):
        clean = lba.lba_attention(q, k, v, cu, cu, causal=causal)
        bad = [t.clone() for t in (q, k, v)]
        for t in bad:
            t[100:] = math.nan
        assert torch.equal(lba.lba_attention(*bad, cu, cu, causal=causal)[:100], clean[:100])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [16, 64, 72, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_blocks_of_one_and_two_tiles_agree(dim, causal, dtype):
    """Many rows to a sequence, though most are in none, make the blocks twice as long: the same sums in the same order"""
    lq, lk = [1, 0, 200, 128, 5, 0, 300, 17, 256, 0, 257], [1, 7, 200, 64, 500, 0, 0, 300, 255, 0, 700]
    n = sum(lq)
    q, k, v = _randn(n + 24000, 4, dim, dtype=dtype), _randn(sum(lk), 2, dim, seed=1, dtype=dtype), _randn(sum(lk), 2, dim, seed=2, dtype=dtype)
    k[3], v[300, 0, 5], v[1300, 1, 3], v[2000, 0, :8] = math.nan, math.inf, -math.inf, math.nan
    scale = torch.tensor([0.01], device="cuda")
    for kw in ({}, dict(out_dtype=torch.uint8, out_scale=scale)):
        short, lse = lba.lba_attention(q[:n], k, v, _cu(lq), _cu(lk), causal=causal, lse=True, **kw)
        long, lse2 = lba.lba_attention(q, k, v, _cu(lq), _cu(lk), causal=causal, lse=True, **kw)
        assert torch.equal(short.view(torch.uint8), long[:n].view(torch.uint8))
        assert torch.equal(lse.view(torch.int32), lse2[:, :n].contiguous().view(torch.int32))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [40, 64, 104, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_long_blocks(dim, causal, dtype):
    for T in (2177, 2305):  # a last block of one tile and of two
        _check(_randn(T, 2, dim, dtype=dtype), _randn(T - 100, 1, dim, seed=1, dtype=dtype), _randn(T - 100, 1, dim, seed=2, dtype=dtype), None, None, causal)


def test_strides_of_projections():
    T, H, G, D = 150, 6, 2, 64
    x = _randn(T, H + 2 * G, D)
    out, _ = _check(x[:, :H], x[:, H:H + G], x[:, H + G:], None, None, True)
    assert torch.equal(out, lba.lba_attention(*(t.contiguous() for t in (x[:, :H], x[:, H:H + G], x[:, H + G:]))))
    first = _randn(H, T, D)   # heads outermost
    _check(first.transpose(0, 1), x[:, H:H + G], x[:, H + G:], None, None, False)
    one = _randn(T, 1, 136)[:, :, 8:72]
    _check(one, one, one, None, None, True)


@pytest.mark.parametrize("scale", [1e-6, 0.02, 1.0, 20.0])
def test_scales(scale):
    """from almost uniform weights to almost one each: the running maximum jumps"""
    q, k, v = _randn(300, 2, 64), _randn(300, 2, 64, seed=1), _randn(300, 2, 64, seed=2)
    k *= torch.linspace(0.05, 2.0, 300, device="cuda", dtype=torch.bfloat16)[:, None, None]
    _check(q, k, v, None, None, True, scale)
    _check(q, k.flip(0), v, None, None, False, scale)


def test_long_sequence():
    T = 5000
    out, lse = _check(_randn(T, 1, 128), _randn(T, 1, 128, seed=1), _randn(T, 1, 128, seed=2), None, None, True)


@pytest.mark.parametrize("m4e3", [False, True])
@pytest.mark.parametrize("dim", [64, 88])
def test_codes(m4e3, dim):
    """codes are the nearest to out / out_scale: compared with the 16-bit outputs, half a step of those off at most before rounding"""
    q, k, v = _randn(260, 4, dim, dtype=torch.float16), _randn(260, 2, dim, seed=1, dtype=torch.float16), _randn(260, 2, dim, seed=2, dtype=torch.float16)
    s = torch.tensor([2.0 / (248.0 if m4e3 else 448.0)], device="cuda")
    fmt = LbaFormat(7, 4, 0, 0, 1 + (FLAG_INPUT_M4E3 if m4e3 else 0))
    codes = lba.lba_attention(q, k, v, out_dtype=torch.uint8, out_scale=s, prod_fmt=fmt)
    assert codes.dtype == torch.uint8 and codes.shape == q.shape
    if m4e3:
        c = torch.arange(256, device="cuda")
        mag = torch.exp2(((c >> 4) & 7).double()) * (1 + (c & 15).double() / 16)
        held = torch.where((c & 127) == 0, 0.0, torch.where(c >= 128, -mag, mag))[codes.long()]
        top, half, least = 248.0, 2.0 ** -5, 0.53125
    else:
        held, top, half, least = codes.view(torch.float8_e4m3fn).double(), 448.0, 2.0 ** -4, 2.0 ** -10
    want = attention(q, k, v, None, None, True, dim ** -0.5)
    x = want["out"] / s.double()
    close(held, x.clamp(-top, top), (half * x.abs()).clamp_min(least) * 1.001 + want["out_bound"] / s.double() * 1.1)


def test_streams_graphs_and_repeats():
    lengths = [100, 300, 57]
    T = sum(lengths)
    q, k, v, cu = _randn(T, 4, 128), _randn(T, 2, 128, seed=1), _randn(T, 2, 128, seed=2), _cu(lengths)
    want = lba.lba_attention(q, k, v, cu, cu)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = lba.lba_attention(q, k, v, cu, cu, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = lba.lba_attention(q, k, v, cu, cu)
    q.copy_(_randn(T, 4, 128, seed=9))
    cu.copy_(_cu([200, 200, 57]))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, lba.lba_attention(q, k, v, cu, cu))


def test_no_rows_and_no_keys():
    q, e = _randn(5, 2, 64), _randn(0, 2, 64)
    out, lse = lba.lba_attention(q, e, e, lse=True, causal=False)
    assert (out == 0).all() and (lse == -math.inf).all()
    assert lba.lba_attention(e, q, q).shape == (0, 2, 64)
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    lba.lba_attention(q, q, q, none, none)
    torch.cuda.synchronize()
