"""The 4-bit key-value cache on the GPU: bytes and values against the definition, and the attention that reads it against the 64-bit form."""
import math

import numpy as np
import pytest
import torch

from helpers.block_ref import HALF, LEAST, cache_values, close, nearest4, row_bytes
from paper_2401_14110_b200 import LbaFormat
from paper_2401_14110_b200 import binding as lba

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _randn(*shape, seed=0, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(dtype)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _table(lengths, page, width=None, spare=2, seed=0):
    """(block table with pages in random order, page count)"""
    blocks = [-(-n // page) for n in lengths]
    order = torch.randperm(sum(blocks) + spare, generator=torch.Generator().manual_seed(seed)).tolist()
    width = max(blocks + [1]) if width is None else width
    rows = []
    for b in blocks:
        rows.append([order.pop() for _ in range(b)] + [-1] * (width - b))
    return _ints(rows), sum(blocks) + spare


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [32, 64, 96, 128])
def test_append_writes_the_nearest_values_where_the_layout_says(dim, dtype):
    kv, page, new, start = 2, 16, [1, 0, 37, 5], [0, 3, 11, 60]
    table, pages = _table([a + b for a, b in zip(new, start)], page)
    cu = _ints(np.cumsum([0] + new).tolist())
    k, v = _randn(43, kv, dim, seed=1, dtype=dtype), _randn(43, kv, dim, seed=2, dtype=dtype) * 100
    k[5] = 0.0
    k[6, 0, :32] *= 2.0 ** -20
    k[7, 1, 1] = 1000.0
    ties = torch.tensor([6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -0.75, -2.5, -5] + [0.0] * 20).repeat(dim // 32)
    k[8, 0], v[9, 1] = ties.to(dtype), (ties * 2).to(dtype)
    cache = torch.full(lba.cache_shape(pages, kv, page, dim), 0x5A, dtype=torch.uint8, device="cuda")
    before = cache.clone()
    assert lba.lba_cache_append(k, v, cache, page, table, _ints(start), cu) is cache
    keys, values = cache_values(cache.cpu(), page, dim)
    written = torch.zeros(pages, page, dtype=torch.bool)
    for name, x, held in (("k", k, keys), ("v", v, values)):
        want = nearest4(x.double().cpu().numpy())
        t = 0
        for b, n in enumerate(new):
            for i in range(n):
                pos = start[b] + i
                pg, row = int(table[b, pos // page]), pos % page
                assert np.array_equal(held[pg, :, row].numpy(), want[t]), (name, t)
                written[pg, row] = True
                t += 1
    # everything else is as it was
    was = cache_values(before.cpu(), page, dim)
    for held, old in ((keys, was[0]), (values, was[1])):
        assert torch.equal(held.transpose(1, 2)[~written], old.transpose(1, 2)[~written])
    got = lba.lba_cache_read(cache, page, table, _ints(start), cu, 43, dtype)
    for g, x in zip(got, (k, v)):
        close(g, torch.from_numpy(nearest4(x.double().cpu().numpy())).cuda(), LEAST[dtype])


def test_bytes_by_the_formula():
    dim, page = 64, 16
    codes = torch.arange(dim) * 5 % 16
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])
    x = (grid[codes] * 4).cuda()
    x[0], x[32], codes[0], codes[32] = 24.0, -24.0, 7, 15   # both groups' largest is 6 x 2^2
    cache = torch.zeros(lba.cache_shape(1, 1, page, dim), dtype=torch.uint8, device="cuda")
    lba.lba_cache_append(x.view(1, 1, dim), x.view(1, 1, dim), cache, page, _ints([[0]]), _ints([3]))
    c = cache.cpu()[0, 0]
    n = page * dim // 2
    assert c[3 * 32:4 * 32].tolist() == row_bytes(codes.tolist(), True)
    assert c[n + 3 * 32:n + 4 * 32].tolist() == row_bytes(codes.tolist(), False)
    assert c[2 * n + 6:2 * n + 8].tolist() == [129, 129] and c[2 * n + 2 * page + 6:2 * n + 2 * page + 8].tolist() == [129, 129]
    assert int((c != 0).sum()) <= 2 * 32 + 4


def test_values_that_are_not_finite_and_the_ends_of_the_range():
    dim, page = 32, 16
    x = torch.zeros(6, 1, dim, device="cuda")
    x[0, 0, 3], x[1, 0, 4], x[2, 0, 5] = math.inf, math.nan, -math.inf
    x[3] = 3.0e38
    x[4, 0, :4] = torch.tensor([2.0 ** -127, 2.0 ** -126, 2.0 ** -149, -(2.0 ** -125)])
    x[5, 0, 0] = -0.0
    cache = torch.zeros(lba.cache_shape(1, 1, page, dim), dtype=torch.uint8, device="cuda")
    lba.lba_cache_append(x, x, cache, page, _ints([[0]]), _ints([0]), _ints([0, 6]))
    k, v = lba.lba_cache_read(cache, page, _ints([[0]]), _ints([0]), _ints([0, 6]), 6, torch.float32)
    want = torch.from_numpy(nearest4(x.double().cpu().numpy())).cuda()
    close(k, want, 0.0)
    close(v, want, 0.0)
    assert torch.isnan(k[:3]).all() and torch.isfinite(k[3:]).all()


def test_tokens_without_a_place():
    """pages outside the cache, positions outside the table, rows outside the sequences: not stored, read as 0, the rest as ever"""
    page, dim, kv = 16, 32, 1
    table = _ints([[0, 7, -1], [1, 2, 3]])
    cache = torch.full(lba.cache_shape(4, kv, page, dim), 0x11, dtype=torch.uint8, device="cuda")
    before = cache.clone()
    k = _randn(70, kv, dim, seed=3)
    start, cu = _ints([10, -3]), _ints([2, 32, 64])   # sequence 0: positions 10..39; sequence 1: -3..28
    lba.lba_cache_append(k, k, cache, page, table, start, cu)
    assert torch.equal(cache[3], before[3])
    got, _ = lba.lba_cache_read(cache, page, table, start, cu, 70, torch.float32, out=(torch.full((70, kv, dim), 9.0, device="cuda"), torch.empty(70, kv, dim, device="cuda")))
    want = torch.from_numpy(nearest4(k.double().cpu().numpy())).cuda()
    want[:2], want[64:] = 9.0, 9.0          # no sequence
    want[2 + 6:32] = 0.0                    # page 7 and page -1
    want[32:35] = 0.0                       # positions below 0
    close(got, want, 0.0)
    far = lba.lba_cache_read(cache, page, table, _ints([47, 100]), _ints([0, 3, 4]), 4, torch.float32)[0]
    assert (far == 0).all()


def _reference(q, cache, page, table, lengths, scale, dtype):
    """(out, bound): keys and values are exact; a query is held to 2^-12 of its largest value's size below 2^-14 of it; weights are rounded to
    binary16 (2^-11 with their factor), scores summed in 32 bits as in helpers.block_ref.attention"""
    B, H, D = q.shape
    keys, values = (t.cuda() for t in cache_values(cache.cpu(), page, D))
    out, bound = torch.zeros(B, H, D, dtype=torch.float64, device="cuda"), torch.zeros(B, H, D, dtype=torch.float64, device="cuda")
    for b in range(B):
        n = min(max(int(lengths[b]), 0), table.shape[1] * page)
        pos = torch.arange(n, device="cuda")
        pg = table[b, pos // page].long()
        ok = (pg >= 0) & (pg < cache.shape[0])
        pos, pg = pos[ok], pg[ok]
        if pos.numel() == 0:
            continue
        K, V = keys[pg, :, pos % page], values[pg, :, pos % page]
        for h in range(H):
            g = h // (H // cache.shape[1])
            x = q[b, h].double()
            s = K[:, g] @ x * scale
            off = ((D + 16) * 2.0 ** -23 * (K[:, g].abs() @ x.abs()) + 2.0 ** -24 * x.abs().max() * K[:, g].abs().sum(1)).max() * scale + 2.0 ** -20
            p = torch.softmax(s, 0)
            out[b, h] = p @ V[:, g]
            bound[b, h] = HALF[dtype] * out[b, h].abs() + (2.0 ** -11 + 2 * off + (n + 64) * 2.0 ** -23) * (p @ V[:, g].abs()) + LEAST[dtype] + 2.0 ** -37 * V[:, g].abs().max() * n
    return out, bound


def _filled(lengths, kv, dim, page, width=None, seed=0, scale_v=1.0):
    table, pages = _table(lengths, page, width, seed=seed)
    cache = torch.full(lba.cache_shape(pages, kv, page, dim), 0xFF, dtype=torch.uint8, device="cuda")   # what is never written is no number
    T = sum(lengths)
    cu = _ints(np.cumsum([0] + list(lengths)).tolist())
    k, v = _randn(T, kv, dim, seed=seed + 1), _randn(T, kv, dim, seed=seed + 2) * scale_v
    lba.lba_cache_append(k, v, cache, page, table, _ints([0] * len(lengths)), cu)
    return cache, table


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [32, 64, 96, 128])
@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 2), (8, 1), (9, 1), (32, 2), (40, 2)])
def test_attention_of_single_tokens(heads, kv, dim, dtype):
    lengths = [1, 15, 16, 17, 200, 0, 333]
    cache, table = _filled(lengths, kv, dim, 32)
    q = _randn(len(lengths), heads, dim, seed=5, dtype=dtype)
    got = lba.lba_cache_attention(q, cache, 32, table, _ints(lengths))
    close(got, *_reference(q, cache, 32, table, lengths, dim ** -0.5, dtype))
    assert (got[5] == 0).all()


@pytest.mark.parametrize("page", [16, 48, 64, 256, 1024])
@pytest.mark.parametrize("length", [1, 127, 128, 129, 1000, 2049, 9000])
def test_lengths_and_pages(length, page):
    """chunks of 128 tokens and more, the last one cut anywhere"""
    cache, table = _filled([length, 5], 2, 64, page)
    q = _randn(2, 6, 64, seed=5)
    got = lba.lba_cache_attention(q, cache, page, table, _ints([length, 5]), scale=0.3)
    close(got, *_reference(q, cache, page, table, [length, 5], 0.3, torch.bfloat16))


def test_wide_table_negative_lengths_and_bad_pages():
    cache, table = _filled([100, 300, 64], 1, 64, 16, width=500)
    q = _randn(3, 4, 64, seed=5)
    table[1, 3], table[1, 7], table[2, 0] = -1, 1 << 30, cache.shape[0]
    for lengths in ([100, 300, 64], [-5, 290, 16], [1, 100000, 5]):
        got = lba.lba_cache_attention(q, cache, 16, table, _ints(lengths))
        close(got, *_reference(q, cache, 16, table, lengths, 0.125, torch.bfloat16))


def test_groups_of_very_different_sizes():
    """values of a group 2^-15 and more below the largest that a warp has met may be dropped: 2^-14 of the largest value's size"""
    lengths = [400]
    table, pages = _table(lengths, 16)
    cache = torch.zeros(lba.cache_shape(pages, 1, 16, 64), dtype=torch.uint8, device="cuda")
    k, v = _randn(400, 1, 64, seed=1, dtype=torch.float32), _randn(400, 1, 64, seed=2, dtype=torch.float32)
    v *= torch.exp2(torch.randint(-12, 13, (400, 1, 1), generator=torch.Generator("cuda").manual_seed(4), device="cuda").float())
    lba.lba_cache_append(k, v, cache, 16, table, _ints([0]), _ints([0, 400]))
    q = _randn(1, 8, 64, seed=5, dtype=torch.float16)
    want, bound = _reference(q, cache, 16, table, lengths, 0.125, torch.float16)
    p_max = 1.0
    close(lba.lba_cache_attention(q, cache, 16, table, _ints(lengths)), want, bound + 2.0 ** -14 * 6 * 2.0 ** -15 * v.abs().max() * p_max * 400)


def test_sharp_and_flat_weights_and_query_sizes():
    cache, table = _filled([700], 1, 128, 64)
    for size in (2.0 ** -20, 1.0, 30.0, 2.0 ** 20):
        q = _randn(1, 8, 128, seed=6) * size
        for scale in (1e-3 / size, 0.3 / size):
            close(lba.lba_cache_attention(q, cache, 64, table, _ints([700]), scale=scale), *_reference(q, cache, 64, table, [700], scale, torch.bfloat16))


def test_a_group_that_is_not_a_number():
    cache, table = _filled([50, 50], 2, 64, 16)
    bad = _randn(1, 2, 64, seed=8)
    bad[0, 0, 40] = math.inf
    q = _randn(2, 4, 64, seed=9)
    clean = lba.lba_cache_attention(q, cache, 16, table, _ints([50, 50]))
    ok = _randn(1, 2, 64, seed=8)
    lba.lba_cache_append(torch.cat([ok, ok]), torch.cat([bad, ok]), cache, 16, table, _ints([20, 20]))
    out = lba.lba_cache_attention(q, cache, 16, table, _ints([50, 50]))
    assert torch.isnan(out[0, :2, 32:]).all() and torch.isfinite(out[0, :2, :32]).all() and torch.isfinite(out[0, 2:]).all() and torch.isfinite(out[1]).all()
    short = lba.lba_cache_attention(q, cache, 16, table, _ints([20, 50]))   # the token lies behind the length
    assert torch.isfinite(short).all() and torch.isfinite(clean).all()


def test_codes_and_strides():
    cache, table = _filled([77, 9], 2, 64, 16)
    x = _randn(2, 8, 64, seed=4)
    q = x[:, 2:6]
    want, bound = _reference(q, cache, 16, table, [77, 9], 0.125, torch.bfloat16)
    close(lba.lba_cache_attention(q, cache, 16, table, _ints([77, 9])), want, bound)
    s = torch.tensor([1.0 / 448], device="cuda")
    codes = lba.lba_cache_attention(q, cache, 16, table, _ints([77, 9]), out_dtype=torch.uint8, out_scale=s, prod_fmt=LbaFormat(7, 4, 0, 0, 1))
    z = want / s.double()
    close(codes.view(torch.float8_e4m3fn), z.clamp(-448, 448), (2.0 ** -4 * z.abs()).clamp_min(2.0 ** -10) * 1.001 + bound / s.double())


def test_streams_graphs_and_growing_lengths():
    cache, table = _filled([300, 40], 2, 64, 16)
    q, lengths = _randn(2, 4, 64, seed=4), _ints([290, 40])
    want = lba.lba_cache_attention(q, cache, 16, table, lengths)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = lba.lba_cache_attention(q, cache, 16, table, lengths, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    k = _randn(2, 2, 64, seed=11)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lba.lba_cache_append(k, k, cache, 16, table, lengths)
        got = lba.lba_cache_attention(q, cache, 16, table, lengths + 1)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        close(got, *_reference(q, cache, 16, table, (lengths + 1).tolist(), 0.125, torch.bfloat16))
        lengths += 1
        lengths.clamp_(max=299)
        lengths[1] = min(int(lengths[1]), 47)
