"""Cache attention over values of very different sizes: each counts with its own weight, whatever else the cache holds."""
import math

import numpy as np
import pytest
import torch

from helpers.block_ref import close
from helpers.cache_ref import attention
from paper_2401_14110_b200 import binding as lba

pytestmark = pytest.mark.gpu
PAGE = 16


def _randn(*shape, seed=0, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(dtype)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _cache(ks, vs):
    """a cache that holds these sequences' keys and values [tokens][heads][dim], and its table"""
    lengths = [k.shape[0] for k in ks]
    width = max(-(-n // PAGE) for n in lengths)
    kv, dim = ks[0].shape[1:]
    table = _ints(np.arange(width * len(ks)).reshape(len(ks), width)[:, ::-1].tolist())
    cache = torch.zeros(lba.cache_shape(width * len(ks), kv, PAGE, dim), dtype=torch.uint8, device="cuda")
    lba.lba_cache_append(torch.cat(ks), torch.cat(vs), cache, PAGE, table, _ints([0] * len(ks)), _ints(np.cumsum([0] + lengths).tolist()))
    return cache, table, lengths


def _check(q, ks, vs, scale=1.0):
    cache, table, lengths = _cache(ks, vs)
    got = lba.lba_cache_attention(q, cache, PAGE, table, _ints(lengths), scale=scale)
    close(got, *attention(q, cache, PAGE, table, lengths, scale))
    return got


def _first_value(heads, dim, dtype=torch.bfloat16):
    """queries whose scores are the keys' first values"""
    q = torch.zeros(1, heads, dim, dtype=dtype, device="cuda")
    q[..., 0] = 1.0
    return q


@pytest.mark.parametrize("dim", [32, 64, 96, 128])
@pytest.mark.parametrize("heads", [1, 8, 16])
@pytest.mark.parametrize("first,second,tokens", [(0, 1, 2), (1, 0, 2), (3, 21, 40), (21, 3, 40), (5, 3000, 3100), (3000, 5, 3100), (70, 75, 128)])
def test_a_large_value_without_weight_leaves_small_ones(first, second, tokens, heads, dim):
    """token `first` has all the weight and values of 1, token `second` 2^-184 of it and values of 2^20: in one step, in one warp's steps, in different warps"""
    k, v = torch.zeros(tokens, 1, dim, device="cuda"), _randn(tokens, 1, dim, seed=3)
    k[:, 0, 0] = -64.0
    k[first, 0, 0], v[first] = 0.0, 1.0
    k[second, 0, 0], v[second] = -128.0, 2.0 ** 20
    got = _check(_first_value(heads, dim), [k], [v])
    assert (got == 1).all()


@pytest.mark.parametrize("size", [16, 40, 60])
@pytest.mark.parametrize("tokens", [2, 40, 1000])
def test_a_large_value_with_a_small_weight_counts(tokens, size):
    """2^-46 of the weight (e^-32) and 2^`size` times the value"""
    for first, second in ((0, tokens - 1), (tokens - 1, 0)):
        k, v = torch.zeros(tokens, 1, 64, device="cuda"), torch.zeros(tokens, 1, 64, device="cuda")
        k[:, 0, 0] = -96.0
        k[first, 0, 0], v[first] = 0.0, 1.0
        k[second, 0, 0], v[second] = -32.0, -(2.0 ** size)
        _check(_first_value(4, 64), [k], [v])


@pytest.mark.parametrize("heads,kv", [(4, 1), (16, 2), (16, 1)])
@pytest.mark.parametrize("dim", [32, 96, 128])
@pytest.mark.parametrize("spread", [8, 30])
def test_sizes_and_weights_at_random(spread, dim, heads, kv):
    """sizes of values 2^+-spread and weights of up to 2^-60, neither knowing the other; some groups are 0"""
    ks, vs = [], []
    for b, n in enumerate((7, 300, 33)):
        g = torch.Generator("cuda").manual_seed(b)
        ks.append(_randn(n, kv, dim, seed=b + 1))
        size = torch.randint(-spread, spread + 1, (n, kv, dim // 32, 1), generator=g, device="cuda").float()
        v = _randn(n, kv, dim // 32, 32, seed=b + 9) * torch.exp2(size)
        v[torch.rand(n, kv, dim // 32, 1, generator=g, device="cuda").expand_as(v) < 0.05] = 0.0
        vs.append(v.view(n, kv, dim))
    for size in (0.1, 1.0):
        _check((_randn(3, heads, dim, seed=5) * size).to(torch.bfloat16), ks, vs, scale=1.0)


@pytest.mark.parametrize("dim", [32, 64, 96, 128])
@pytest.mark.parametrize("heads", [1, 8, 16])
@pytest.mark.parametrize("size", [1.0, 2.0 ** -124])
def test_groups_of_zeros_among_others(size, heads, dim):
    """a first token of zeros, others here and there and single groups, -0 among them; beside values of any size, and of a size that has the exponent byte of zeros"""
    n = 700
    k, v = _randn(n, 1, dim, seed=1), _randn(n, 1, dim, seed=2) * size
    k[0], v[0] = 0.0, 0.0
    v[200], v[333], v[96:130], v[5::50, :, :32], v[400] = 0.0, -0.0, 0.0, 0.0, 6 * 2.0 ** -127
    _check(_randn(1, heads, dim, seed=3, dtype=torch.bfloat16), [k], [v], scale=0.5)


def test_other_requests_do_not_matter():
    """a request with large values of small weight, alone and among others that change the warps' shares"""
    n, dim = 500, 64
    k, v = _randn(n, 1, dim, seed=1), _randn(n, 1, dim, seed=2)
    k[:, 0, 0] = torch.linspace(-40, 0, n, device="cuda")
    v[::7] *= 2.0 ** 18
    v[-60:] = _randn(60, 1, dim, seed=3) * 2.0 ** -3
    q = torch.cat([_first_value(4, dim) * 2, _randn(3, 4, dim, seed=4, dtype=torch.bfloat16)])
    alone = _check(q[:1], [k], [v])
    for lengths in ([100, 100, 100], [5000, 3, 60], [1, 20000, 64]):
        ks, vs = [k] + [_randn(m, 1, dim, seed=m) for m in lengths], [v] + [_randn(m, 1, dim, seed=m + 1) for m in lengths]
        among = _check(q, ks, vs)
        assert (among[0].float() - alone[0].float()).abs().max() <= 2.0 ** -6 * alone[0].float().abs().max()


def test_a_group_that_is_no_number_among_small_and_large_ones():
    k, v = torch.zeros(20, 1, 64, device="cuda"), _randn(20, 1, 64, seed=2)
    v[3, 0, 40], v[5] = math.nan, v[5] * 2.0 ** 30
    got = _check(_first_value(4, 64), [k], [v])
    assert torch.isnan(got[..., 32:]).all() and torch.isfinite(got[..., :32]).all()


@pytest.mark.parametrize("tokens", [1, 3, 100, 5000])
@pytest.mark.parametrize("size", [2.0 ** 127, 2.0 ** 100, 2.0 ** -120])
def test_values_at_the_ends_of_the_range(size, tokens):
    """an output lies between its values, however large they are"""
    k, v = _randn(tokens, 1, 64, seed=1), (_randn(tokens, 1, 64, seed=2).abs() * 0.25 + 0.5).clamp_max(1.4) * size
    cache, table, lengths = _cache([k], [v])
    q = _randn(1, 4, 64, seed=3, dtype=torch.bfloat16)
    got = lba.lba_cache_attention(q, cache, PAGE, table, _ints(lengths), scale=0.5)
    want, bound = attention(q, cache, PAGE, table, lengths, 0.5)
    close(got, want, bound + 2.0 ** -140)   # (parts of what is below 2^-126 are held to 2^-149, and a sum of parts to their number of times that)


@pytest.mark.parametrize("scale", [1e-38, 1e-20, 1.0])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_a_query_of_zeros_and_a_small_scale(dtype, scale):
    """weights are all the same: the mean of the values, whatever stands behind the last token"""
    k, v = (torch.randn(21, 1, 32, generator=torch.Generator("cuda").manual_seed(s), device="cuda") for s in (1, 2))
    cache = torch.full(lba.cache_shape(2, 1, 16, 32), 0xFF, dtype=torch.uint8, device="cuda")
    table = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda")
    ends = torch.tensor([0, 21], dtype=torch.int32, device="cuda")
    lba.lba_cache_append(k, v, cache, 16, table, ends[:1], ends)
    q = torch.zeros(1, 2, 32, dtype=dtype, device="cuda")
    q[0, 1, 5] = 2.0 ** -24
    got = lba.lba_cache_attention(q, cache, 16, table, ends[1:], scale=scale)
    close(got, *attention(q, cache, 16, table, [21], scale))
