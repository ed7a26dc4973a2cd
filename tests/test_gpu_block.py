"""A transformer block's calls in a row, as they are used: a prompt in two parts, tokens one by one behind it, and a training step."""
import math

import numpy as np
import pytest
import torch

from helpers.block_ref import attention, cache_values, close
from paper_2401_14110_b200 import ORDER_CHUNKED as CHK
from paper_2401_14110_b200 import binding as lba
from paper_2401_14110_b200 import code_domain_formats

pytestmark = pytest.mark.gpu
PROD, ACC = code_domain_formats(7, 4)
H, G, D, PAGE = 4, 2, 64, 16
WIDTH = H * D


def _randn(*shape, seed=0, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(dtype)


def _codes(x):
    x = x.float()
    s = (x.abs().amax() / 448).reshape(1)
    return (x / s).to(torch.float8_e4m3fn).view(torch.uint8), s


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Block:
    def __init__(self):
        self.w_qkv, self.s_qkv = _codes(_randn((H + 2 * G) * D, WIDTH, seed=1) * WIDTH ** -0.5)
        self.w_out, self.s_out = _codes(_randn(WIDTH, WIDTH, seed=2) * WIDTH ** -0.5)
        self.freqs = lba.rotary_frequencies(D)
        self.scale = torch.tensor([2.0 / 448], device="cuda")

    def qkv(self, x, positions):
        a, s = _codes(x)
        p = lba.lba_linear(a, self.w_qkv, s, self.s_qkv, None, PROD, ACC, CHK, 16, out_dtype=torch.bfloat16).view(-1, H + 2 * G, D)
        lba.lba_rotary(p[:, :H], p[:, H:H + G], positions, self.freqs, out=(p[:, :H], p[:, H:H + G]))
        return p[:, :H], p[:, H:H + G], p[:, H + G:]

    def out(self, codes, residual):
        return lba.lba_linear(codes.view(-1, WIDTH), self.w_out, self.scale, self.s_out, None, PROD, ACC, CHK, 16, residual=residual, out_dtype=torch.bfloat16)


def test_prompts_in_parts_and_new_tokens_behind_them():
    block, lengths = Block(), [37, 90]
    blocks = 8
    table = _ints([[3 * i + b for i in range(blocks)] for b in range(2)])
    cache = torch.zeros(lba.cache_shape(3 * blocks, G, PAGE, D), dtype=torch.uint8, device="cuda")
    seen = _ints([0, 0])
    for part in ([20, 64], [17, 26]):   # the second part attends to the first through the cache
        cu = _ints([0, part[0], sum(part)])
        x = _randn(sum(part), WIDTH, seed=sum(part), dtype=torch.bfloat16)
        pos = torch.cat([torch.arange(n, device="cuda") + s for n, s in zip(part, seen)])
        q, k, v = block.qkv(x, pos)
        lba.lba_cache_append(k, v, cache, PAGE, table, seen, cu)
        after = seen + _ints(part)
        cu_k = _ints([0, int(after[0]), int(after.sum())])
        ks, vs = lba.lba_cache_read(cache, PAGE, table, _ints([0, 0]), cu_k, int(after.sum()), torch.bfloat16)
        codes = lba.lba_attention(q, ks, vs, cu, cu_k, out_dtype=torch.uint8, out_scale=block.scale, prod_fmt=PROD)
        want = attention(q, ks, vs, cu, cu_k, True, D ** -0.5)
        z = want["out"] / block.scale.double()
        close(codes.view(torch.float8_e4m3fn), z.clamp(-448, 448), (2.0 ** -4 * z.abs()).clamp_min(2.0 ** -10) * 1.001 + want["out_bound"] / block.scale.double() * 1.1)
        y = block.out(codes, x)
        assert y.shape == x.shape and torch.isfinite(y.float()).all()
        seen = after
    assert seen.tolist() == lengths
    # one token each, twice, in one captured graph: lengths and positions are read on the GPU
    x = _randn(2, WIDTH, seed=50, dtype=torch.bfloat16)
    p = torch.empty(2, H + 2 * G, D, dtype=torch.bfloat16, device="cuda")
    a, s = _codes(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.copy_(lba.lba_linear(a, block.w_qkv, s, block.s_qkv, None, PROD, ACC, CHK, 16, out_dtype=torch.bfloat16).view(2, H + 2 * G, D))
        lba.lba_rotary(p[:, :H], p[:, H:H + G], seen, block.freqs, out=(p[:, :H], p[:, H:H + G]))
        lba.lba_cache_append(p[:, H:H + G], p[:, H + G:], cache, PAGE, table, seen)
        seen += 1
        o = lba.lba_cache_attention(p[:, :H], cache, PAGE, table, seen)
    for step in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert seen.tolist() == [n + step + 1 for n in lengths]
        keys, values = cache_values(cache.cpu(), PAGE, D)
        for b in range(2):
            n = int(seen[b])
            at = torch.arange(n)
            pages = table[b].cpu()[at // PAGE].long()
            K, V = (t[pages, :, at % PAGE].cuda() for t in (keys, values))
            for h in range(H):
                w = torch.softmax(K[:, h // 2] @ p[b, h].double() * D ** -0.5, 0)
                want = w @ V[:, h // 2]
                # weights of 11 bits, results of 8
                close(o[b, h], want, 2.0 ** -8 * want.abs() + 2.0 ** -10 * (w @ V[:, h // 2].abs()) + 1e-9)


def test_gradients_through_a_block():
    """linear layers, rotary positions and attention, forward and backward through their own calls, against 64-bit autograd of the same values (the
    estimator passes the quantisers' gradients): every stored tensor is bfloat16, 2^-8 of each value, and four of them follow one another"""
    T = 150
    w, b = _randn((H + 2 * G) * D, WIDTH, seed=3) * WIDTH ** -0.5, None
    wc, ws = _codes(w)
    xc, xs = _codes(_randn(T, WIDTH, seed=4))
    pos, freqs = torch.arange(T, device="cuda"), lba.rotary_frequencies(D)
    p, pre = lba.lba_linear(xc, wc, xs, ws, b, PROD, ACC, CHK, 16, out_dtype=torch.bfloat16, preact=torch.bfloat16)
    p = p.view(T, H + 2 * G, D)
    q, k = lba.lba_rotary(p[:, :H], p[:, H:H + G], pos, freqs)
    out, lse = lba.lba_attention(q, k, p[:, H + G:], lse=True)
    g = _randn(T, H, D, seed=5, dtype=torch.bfloat16)
    gq, gk, gv = lba.lba_attention_backward(g, q, k, p[:, H + G:], out, lse)
    gq, gk = lba.lba_rotary(gq, gk, pos, freqs, inverse=True)
    gp = torch.cat([gq, gk, gv], dim=1).view(T, -1)
    gx, gw, _ = lba.lba_linear_backward(gp, xc, wc, xs, ws, PROD, needs=(True, True, False))

    x64 = (xc.view(torch.float8_e4m3fn).double() * xs.double()).requires_grad_()
    w64 = (wc.view(torch.float8_e4m3fn).double() * ws.double()).requires_grad_()
    y = x64 @ w64.T
    y = y + (p.view(T, -1).double() - y).detach()   # the accumulator's and the storage's roundings pass the gradient
    y = y.view(T, H + 2 * G, D)
    a = pos.double()[:, None, None] * freqs
    turn = lambda t: torch.cat([t[..., :32] * a.cos() - t[..., 32:] * a.sin(), t[..., :32] * a.sin() + t[..., 32:] * a.cos()], -1)  # noqa: E731
    s = torch.einsum("ihd,jhd->hij", turn(y[:, :H]), turn(y[:, H:H + G]).repeat_interleave(H // G, 1)) / 8
    s = s.masked_fill(torch.ones(T, T, dtype=torch.bool, device="cuda").triu(1), -math.inf)
    o = torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), y[:, H + G:].repeat_interleave(H // G, 1))
    (o * g.double()).sum().backward()
    # q and k are rounded once more (2^-8 of scores of size 1 to 3), the gradients of q, k, v, of their turn and of the layer each once:
    # relative to a gradient's size, six roundings of 2^-8 / sqrt(3) at random and the scores' 2 x 2^-8
    for got, want in ((gx, x64.grad), (gw, w64.grad)):
        assert (got.double() - want).norm() <= 6 * 2.0 ** -8 * want.norm()


def test_calls_need_the_current_device_and_leave_no_state():
    x = _randn(5, 2, 64, dtype=torch.bfloat16)
    first = lba.lba_attention(x, x, x)
    ws = torch.empty(lba.attention_backward_workspace_bytes(x, x, x), dtype=torch.uint8, device="cuda").fill_(0xFF)
    out, lse = lba.lba_attention(x, x, x, lse=True)
    a = lba.lba_attention_backward(x, x, x, x, out, lse, workspace=ws)
    b = lba.lba_attention_backward(x, x, x, x, out, lse)
    assert all(torch.equal(s, t) for s, t in zip(a, b)) and torch.equal(first, out)
    cache, table, n = torch.zeros(lba.cache_shape(2, 2, 16, 64), dtype=torch.uint8, device="cuda"), _ints([[0], [1]]), _ints([4, 9])
    lba.lba_cache_append(x[:2], x[:2], cache, 16, table, n - 1)
    ws = torch.empty(lba.cache_attention_workspace_bytes(cache, 16, table, 4), dtype=torch.uint8, device="cuda").fill_(0xFF)
    q = _randn(2, 4, 64, dtype=torch.float16)
    assert torch.equal(lba.lba_cache_attention(q, cache, 16, table, n, workspace=ws), lba.lba_cache_attention(q, cache, 16, table, n))
    with pytest.raises(lba.LbaError) as e:
        lba.lba_cache_attention(q, cache, 16, table, n, workspace=ws[:-1])
    assert e.value.status == -7
    with pytest.raises(lba.LbaError) as e:
        lba.lba_attention(x, x, x, scale=0.0)
    assert e.value.status == -9


def test_native_calls_are_regular_and_agree_with_ctypes(monkeypatch):
    lba.load_library()
    if lba._native is None:
        pytest.skip("the native module was not built")
    T = 40
    p = _randn(T, H + 2 * G, D, dtype=torch.bfloat16)
    q, k, v, pos, freqs, cu = p[:, :H], p[:, H:H + G], p[:, H + G:], torch.arange(T, device="cuda"), lba.rotary_frequencies(D), _ints([0, 13, T])
    cache, table = torch.zeros(lba.cache_shape(8, G, PAGE, D), dtype=torch.uint8, device="cuda"), _ints([[0, 1], [2, 3]])
    s = torch.tensor([0.01], device="cuda")

    def all_calls():
        r = list(lba.lba_rotary(q, k, pos, freqs)) + list(lba.lba_attention(q, k, v, cu, cu, lse=True))
        r.append(lba.lba_attention(q, k, v, cu, cu, out_dtype=torch.uint8, out_scale=s, prod_fmt=PROD))
        r += lba.lba_attention_backward(r[2], q, k, v, r[2], r[3], cu, cu)
        r.append(lba.lba_cache_append(k, v, cache, PAGE, table, _ints([0, 0]), cu).clone())
        r += lba.lba_cache_read(cache, PAGE, table, _ints([0, 0]), cu, T, torch.float16)
        r.append(lba.lba_cache_attention(q[:2], cache, PAGE, table, _ints([13, 27])))
        return r
    made = []

    class Watch:
        def __getattr__(self, name):
            f = getattr(native, name)

            def call(*a):
                r = f(*a)
                made.append((name, r is not None))
                return r
            return call
    native = lba._native
    monkeypatch.setattr(lba, "_native", Watch())
    a = all_calls()
    assert made and all(regular for _, regular in made) and {n for n, _ in made} == {"rotary", "attention", "attention_backward", "cache_append", "cache_read", "cache_attention"}
    monkeypatch.setattr(lba, "_native", None)
    for x, y in zip(a, all_calls()):
        assert torch.equal(x, y)


def test_calls_on_three_streams_at_once():
    """blocks of one and of two tiles, a backward pass and a cache's reader meet on the same SMs; every result is what the call alone gives"""
    g = torch.Generator("cuda").manual_seed(5)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    cu = torch.arange(0, 25 * 100, 100, dtype=torch.int32, device="cuda")
    q, k, v = randn(2400, 8, 64), randn(2400, 4, 64), randn(2400, 4, 64)
    long_q, long_k, long_v, grad = randn(3000, 4, 128), randn(3000, 2, 128), randn(3000, 2, 128), randn(3000, 4, 128)
    out, lse = lba.lba_attention(long_q, long_k, long_v, lse=True)
    cache = torch.zeros(lba.cache_shape(40, 2, 64, 128), dtype=torch.uint8, device="cuda")
    table = torch.randperm(40, generator=g, device="cuda").to(torch.int32).view(2, 20)
    ends = torch.tensor([0, 1270, 1300], dtype=torch.int32, device="cuda")
    lba.lba_cache_append(long_k[:1300], long_v[:1300], cache, 64, table, torch.zeros(2, dtype=torch.int32, device="cuda"), ends)
    calls = [lambda s: (lba.lba_attention(q, k, v, cu, cu, stream=s),),
             lambda s: (lba.lba_attention(long_q, long_k, long_v, stream=s),),
             lambda s: lba.lba_attention_backward(grad, long_q, long_k, long_v, out, lse, stream=s),
             lambda s: (lba.lba_cache_attention(long_q[:2], cache, 64, table, torch.tensor([1270, 30], dtype=torch.int32, device="cuda"), stream=s),)]
    want = [call(torch.cuda.current_stream()) for call in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for i in range(24):
        with torch.cuda.stream(streams[i % 3]):
            got.append((i % 4, calls[i % 4](streams[i % 3])))
    torch.cuda.synchronize()
    for which, result in got:
        assert all(torch.equal(a, b) for a, b in zip(result, want[which]))
