"""Attention, its gradients and the cache over many sequences: each way of finding a row's sequence, offsets that descend, and neighbours."""
import numpy as np
import pytest
import torch

from helpers import cache_ref
from helpers.block_ref import attention, close, nearest4
from paper_2401_14110_b200 import binding as lba

pytestmark = pytest.mark.gpu


def _randn(*shape, seed=0, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(dtype)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _both_directions(lq, lk, cu_q, cu_k, causal=True, H=2, G=1, D=32, spare=5, dtype=torch.bfloat16):
    Tq, Tk = sum(lq) + spare, sum(lk) + spare
    q, k, v, g = _randn(Tq, H, D, dtype=dtype), _randn(Tk, G, D, seed=1, dtype=dtype), _randn(Tk, G, D, seed=2, dtype=dtype), _randn(Tq, H, D, seed=3, dtype=dtype)
    out, lse = lba.lba_attention(q, k, v, cu_q, cu_k, causal=causal, lse=True, out=torch.full_like(q, 3.0))
    got = lba.lba_attention_backward(g, q, k, v, out, lse, cu_q, cu_k, causal=causal)
    want = attention(q, k, v, cu_q.tolist(), cu_k.tolist(), causal, D ** -0.5, grad=g, out16=out)
    inside = ~torch.isnan(want["lse"][0])
    close(out[inside], want["out"][inside], want["out_bound"][inside])
    close(lse[:, inside], want["lse"][:, inside], want["lse_bound"][:, inside])
    assert (out[~inside] == 3).all()
    for name, t in zip(("grad_q", "grad_k", "grad_v"), got):
        close(t, want[name], want[name + "_bound"])


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("sequences", [31, 32, 33, 127, 128, 129, 300])
def test_attention_and_gradients_of_many_sequences(sequences, causal):
    """empty ones, ones with queries or keys alone and longer ones among them, rows before and behind all of them"""
    rng = np.random.default_rng(sequences)
    lq, lk = rng.integers(0, 12, sequences), rng.integers(0, 20, sequences)
    lq[rng.random(sequences) < 0.2] = 0
    lk[rng.random(sequences) < 0.2] = 0
    lq[[0, -1]], lk[[1, -1]] = 0, 0
    lq[sequences // 2], lk[sequences // 2] = 150, 300
    cu_q, cu_k = (_ints((np.cumsum([0] + list(n)) + 2).tolist()) for n in (lq, lk))
    _both_directions(lq, lk, cu_q, cu_k, causal, dtype=torch.float16 if sequences % 2 else torch.bfloat16)


@pytest.mark.parametrize("many", [0, 40, 200])
@pytest.mark.parametrize("ends_q,ends_k", [([0, 100, 50], [0, 90, 90]), ([0, 100, 50], [0, 100, 30]), ([40, 140, 20, 20], [7, 60, 0, 0]),
                                           ([60, 30, 90], [60, 10, 80]), ([0, 100, -5], [0, 100, 70])])
def test_a_sequence_that_ends_before_it_starts_is_empty(ends_q, ends_k, many):
    """the others are what they are without it, and rows of none get no gradient, however many (here empty) sequences there are"""
    ends_q, ends_k = ends_q + [ends_q[-1]] * many, ends_k + [ends_k[-1]] * many
    _both_directions([140], [140], _ints(ends_q), _ints(ends_k))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("lq,lk", [([5000], [32]), ([5000], [33]), ([2000, 3, 700], [31, 9, 40]), ([4100], [1])])
def test_many_queries_over_few_keys(lq, lk, dtype):
    cu_q, cu_k = (_ints(np.cumsum([0] + n).tolist()) for n in (lq, lk))
    _both_directions(lq, lk, cu_q, cu_k, causal=False, H=3, G=1, D=64, dtype=dtype)


@pytest.mark.parametrize("requests", [127, 128, 129, 400])
def test_cache_attention_of_many_requests(requests):
    """lengths of 0 at the borders of what a warp knows at a time, at the start and at the end"""
    page, G, D, H = 16, 1, 32, 4
    lengths = np.random.default_rng(requests).integers(1, 90, requests)
    for at in (0, 1, 126, 127, 128, 129, 255, 256, 383, 384, requests - 1):
        if at < requests:
            lengths[at] = 0 if at != 126 else 700
    width = -(-700 // page)
    table = torch.arange(requests * width, device="cuda").flip(0).to(torch.int32).view(requests, width)
    cache = torch.zeros(lba.cache_shape(requests * width, G, page, D), dtype=torch.uint8, device="cuda")
    T = int(lengths.sum())
    cu = _ints(np.cumsum([0] + lengths.tolist()).tolist())
    k, v, start = _randn(T, G, D, seed=1), _randn(T, G, D, seed=2), torch.zeros(requests, dtype=torch.int32, device="cuda")
    lba.lba_cache_append(k, v, cache, page, table, start, cu)
    q = _randn(requests, H, D, seed=3)
    close(lba.lba_cache_attention(q, cache, page, table, _ints(lengths.tolist())), *cache_ref.attention(q, cache, page, table, lengths.tolist(), D ** -0.5))


@pytest.mark.parametrize("sequences", [1023, 1024, 1500])
def test_append_and_read_of_many_sequences(sequences):
    page, G, D = 16, 1, 32
    new = np.random.default_rng(sequences).integers(0, 4, sequences)
    new[[0, 511, -1]] = 0
    T = int(new.sum()) + 6
    cu = _ints((np.cumsum([0] + new.tolist()) + 3).tolist())
    start = _ints((np.arange(sequences) % 14).tolist())
    table = torch.randperm(2 * sequences, device="cuda").to(torch.int32).view(sequences, 2)
    cache = torch.full(lba.cache_shape(2 * sequences, G, page, D), 0x5A, dtype=torch.uint8, device="cuda")
    k, v = _randn(T, G, D, seed=1), _randn(T, G, D, seed=2)
    lba.lba_cache_append(k, v, cache, page, table, start, cu)
    out = tuple(torch.full((T, G, D), 9.0, device="cuda") for _ in range(2))
    lba.lba_cache_read(cache, page, table, start, cu, T, torch.float32, out=out)
    for got, x in zip(out, (k, v)):
        want = torch.from_numpy(nearest4(x.double().cpu().numpy())).cuda()
        want[:3], want[T - 3:] = 9.0, 9.0
        close(got, want, 0.0)


@pytest.mark.parametrize("tokens", [20000, 70000])
def test_one_line_in_very_many_parts(tokens):
    """more parts than are joined at a time: 313 units of 64 tokens, and a share of a unit each"""
    page, D = 64, 32
    blocks = -(-tokens // page)
    table = torch.randperm(blocks, device="cuda").to(torch.int32).view(1, blocks)
    cache = torch.zeros(lba.cache_shape(blocks, 1, page, D), dtype=torch.uint8, device="cuda")
    k, v = _randn(tokens, 1, D, seed=1), _randn(tokens, 1, D, seed=2) + 0.25
    k[tokens // 2:] *= 2
    lba.lba_cache_append(k, v, cache, page, table, _ints([0]), _ints([0, tokens]))
    for heads in (1, 12):
        q = _randn(1, heads, D, seed=3)
        close(lba.lba_cache_attention(q, cache, page, table, _ints([tokens])), *cache_ref.attention(q, cache, page, table, [tokens], D ** -0.5))


def _alone_and_packed(call, n, heads, D, dtype):
    """what a call gives of a sequence of n rows alone, and of the same rows with others in front and behind whose scores are far larger"""
    x = [_randn(n, h, D, seed=s, dtype=dtype) for s, h in enumerate(heads)]
    for before, behind in ((0, 40), (77, 200), (130, 0)):
        others = [_randn(before + behind, h, D, seed=9 + i, dtype=dtype) * 8 for i, h in enumerate(heads)]
        packed = [torch.cat([o[:before], t, o[before:]]) for o, t in zip(others, x)]
        got = call(packed, _ints([0, before, before + n, before + n + behind]))
        yield call(x, _ints([0, n])), [t[before:before + n] for t in got]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n", [1, 31, 100, 129, 300])
def test_bits_do_not_depend_on_neighbours(n, causal, dtype):
    def call(x, cu):
        out, lse = lba.lba_attention(*x, cu, cu, causal=causal, lse=True)
        return out, lse.T
    for alone, packed in _alone_and_packed(call, n, (4, 2, 2), 64, dtype):
        assert all(torch.equal(a, b) for a, b in zip(alone, packed))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n", [1, 31, 100, 129, 300])
def test_bits_of_gradients_do_not_depend_on_neighbours(n, causal, dtype=torch.bfloat16):
    def call(x, cu):
        q, k, v, g = x
        out, lse = lba.lba_attention(q, k, v, cu, cu, causal=causal, lse=True)
        return lba.lba_attention_backward(g, q, k, v, out, lse, cu, cu, causal=causal)
    for alone, packed in _alone_and_packed(call, n, (4, 2, 2, 4), 64, dtype):
        assert all(torch.equal(a, b) for a, b in zip(alone, packed))
