"""Plain 64-bit forms of rotary positions, attention and the 4-bit cache, with bounds of what 32-bit sums and operands of 16 bits may be off by."""
import math

import numpy as np
import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # half a step of a rounding, relative
LEAST = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}   # half the smallest subnormal number


def rotary(x, positions, freqs, interleaved, inverse, scale):
    """(result, bound): the bound counts the rounding to x's type, and 8 steps of 2^-24 for cosine, sine, two products and their sum"""
    n = freqs.numel()
    a = positions.double()[:, None, None] * freqs.double()
    a = -a if inverse else a
    c, s, v = torch.cos(a) * scale, torch.sin(a) * scale, x.double()
    out, mag = v.clone(), torch.zeros_like(v)
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    p, q = v[..., first], v[..., second]
    out[..., first], out[..., second] = p * c - q * s, p * s + q * c
    mag[..., first] = mag[..., second] = (p.abs() + q.abs()) * abs(scale)
    return out, HALF[x.dtype] * out.abs() + 8 * 2.0 ** -24 * mag + LEAST[x.dtype]


def spans(cu, rows):
    if cu is None:
        return [(0, rows)]
    ends = [min(max(int(v), 0), rows) for v in cu]
    return [(a, max(b, a)) for a, b in zip(ends, ends[1:])]


def attention(q, k, v, cu_q, cu_k, causal, scale, grad=None, out16=None):
    """Everything of one call in 64 bits, sequence by sequence: dict of out, lse, and with `grad` grad_q, grad_k, grad_v, each with its bound
    (name + "_bound").  Rows of no sequence: NaN in out and lse, 0 in gradients.

    h: half a step of the inputs' type, by which weights, ds and results are rounded.  Scores: D products summed in 32 bits, by instructions that
    cut (2^-23 each), so off by e = (D + 16) 2^-23 sum |q k| scale; the exponential and its argument another 2^-20.  Weights are then off by
    2 e + 2^-20 of themselves (numerator and sum), sums over N keys by N 2^-23 of their terms' magnitudes."""
    Tq, H, D = q.shape
    Tk, G, _ = k.shape
    h, dev = HALF[q.dtype], q.device
    Q, K, V = q.double(), k.double(), v.double()
    res = {"out": torch.full((Tq, H, D), math.nan, dtype=torch.float64, device=dev), "lse": torch.full((H, Tq), math.nan, dtype=torch.float64, device=dev)}
    res["out_bound"], res["lse_bound"] = torch.zeros_like(res["out"]), torch.zeros_like(res["lse"])
    if grad is not None:
        for n, t in (("grad_q", Q), ("grad_k", K), ("grad_v", V)):
            res[n], res[n + "_bound"] = torch.zeros_like(t), torch.zeros_like(t)
    for (a, b), (c, d) in zip(spans(cu_q, Tq), spans(cu_k, Tk)):
        nq, nk = b - a, d - c
        seen = torch.ones(nq, nk, dtype=torch.bool, device=dev)
        if causal:
            seen = torch.arange(nk, device=dev)[None] - torch.arange(nq, device=dev)[:, None] <= nk - nq
        for i in range(H):
            g = i // (H // G)
            zero = torch.zeros(nq, nk, dtype=torch.float64, device=dev)
            s = torch.where(seen, Q[a:b, i] @ K[c:d, g].T * scale, -math.inf)
            mag = torch.where(seen, Q[a:b, i].abs() @ K[c:d, g].abs().T * scale, zero)
            any_key = seen.any(1)
            top = torch.where(any_key, s.amax(1) if nk else 0.0, 0.0)[:, None]
            e = torch.where(seen, torch.exp(s - top), zero)
            total = e.sum(1, keepdim=True)
            p = torch.where(any_key[:, None], e / total.clamp_min(1e-300), zero)
            # a masked infinity or NaN does not count
            hidden = ~seen
            vv = V[c:d, g]
            finite = torch.isfinite(vv)
            if not finite.all():
                o = torch.stack([torch.where(seen[r][:, None], p[r][:, None] * vv, torch.zeros_like(vv)).sum(0) for r in range(nq)]) if nq else Q[a:b, i]
            else:
                o = p @ vv
            res["out"][a:b, i] = o
            res["lse"][i, a:b] = torch.where(any_key, (top + torch.log(total))[:, 0], -math.inf)
            off = (D + 16) * 2.0 ** -23 * (mag.amax(1) if nk else torch.zeros(nq, device=dev).double()) + 2.0 ** -20   # of a row's scores
            rel = (2 * off)[:, None]
            res["out_bound"][a:b, i] = h * o.abs() + (h + rel + (nk + 64) * 2.0 ** -23) * (p @ vv.abs()) + LEAST[q.dtype]
            res["lse_bound"][i, a:b] = off + nk * 2.0 ** -24 + 2.0 ** -22 * torch.nan_to_num(res["lse"][i, a:b], neginf=0.0).abs()
            if grad is None:
                continue
            dO = grad[a:b, i].double()
            rel = rel + res["lse_bound"][i, a:b][:, None] + 2.0 ** -20
            dp, amp = dO @ vv.T, dO.abs() @ vv.abs().T
            delta = (dO * o).sum(1, keepdim=True)
            # delta comes from the rounded output, all sums of D terms in 32 bits
            err = (D + 16) * 2.0 ** -23 * (amp + (dO.abs() * o.abs()).sum(1, keepdim=True)) + (h * dO.abs() * o.abs()).sum(1, keepdim=True) * 1.01
            err = err + (dO.abs() * res["out_bound"][a:b, i]).sum(1, keepdim=True) * (1 if out16 is not None else 0)
            ds = torch.where(seen, p * (dp - delta) * scale, zero)
            # (binary32 exponentials, and products of them, below 2^-126 are 0: a weight of 2^-126 and its ds are lost whole)
            ds_err = torch.where(seen, p * scale * (err + (h + rel) * (dp - delta).abs()) + 2.0 ** -126 * scale * (1 + (dp - delta).abs()), zero)
            p_err = p * (h + rel) + torch.where(seen, 2.0 ** -33 if q.dtype == torch.float16 else 2.0 ** -126, zero)   # (binary16: held times 2^8)
            n = (nq * (H // G) + nk + 64) * 2.0 ** -23
            for name, rows, x, xe, y in (("grad_q", (slice(a, b), i), ds, ds_err, K[c:d, g]), ("grad_k", (slice(c, d), g), ds.T, ds_err.T, Q[a:b, i]),
                                         ("grad_v", (slice(c, d), g), p.T, p_err.T, dO)):
                res[name][rows] += x @ y
                res[name + "_bound"][rows] += (xe + n * x.abs()) @ y.abs()
    if grad is not None:
        for n in ("grad_q", "grad_k", "grad_v"):
            res[n + "_bound"] += h * res[n].abs() + LEAST[q.dtype]
    return res


def close(got, want, bound):
    """infinities equal, NaN beside NaN, everything else within its bound"""
    got, want = got.double(), want.double()
    odd = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), "NaN in other places"
    assert torch.equal(torch.nan_to_num(got[odd], nan=0.0, posinf=1.0, neginf=-1.0), torch.nan_to_num(want[odd], nan=0.0, posinf=1.0, neginf=-1.0))
    err = (got - want).abs()[~odd]
    over = err - (bound + torch.zeros_like(want))[~odd]
    if over.numel():
        assert over.max() <= 0, f"off by {err[over.argmax()].item():.3g} where {(bound + torch.zeros_like(want))[~odd][over.argmax()].item():.3g} is allowed"


# ------------------------------------------------------------------ the cache, value by value
GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def nearest4(x):
    """float64 numpy [..., D] as the cache gives it back"""
    out = np.empty_like(x)
    for at in np.ndindex(*x.shape[:-1]):
        for g in range(0, x.shape[-1], 32):
            v = x[at][g:g + 32]
            if not np.isfinite(v).all():
                out[at][g:g + 32] = np.nan
                continue
            top, e = np.abs(v).max(), -126
            while 6.0 * 2.0 ** e < top and e < 125:
                e += 1
            for j, t in enumerate(np.abs(v) / 2.0 ** e):
                # ties go to the even place in the grid
                best = min(range(8), key=lambda i: (abs(t - GRID[i]), i % 2))
                out[at][g + j] = math.copysign(GRID[best], v[j]) * 2.0 ** e
    return out


def row_bytes(codes, key):
    """4-bit codes of one head's row as its bytes, by the layout's formula"""
    d = len(codes)
    out = [0] * (d // 2)
    for c in range(4 if key else 8):
        for i in range(d // 8 if key else d // 16):
            at = 32 * (i // 4) + 8 * c + 2 * (i % 4) if key else 16 * i + 2 * c
            out[c * (d // 8 if key else d // 16) + i] = int(codes[at]) | int(codes[at + 1]) << 4
    return out


def cache_values(cache, page, dim):
    """(keys, values) float64 [pages][heads][page][dim] of cache bytes (CPU), by the layout's formula"""
    run = cache.shape[2]
    assert run == page * (dim + dim // 16)
    n = page * dim // 2
    parts = cache[..., :n], cache[..., n:2 * n], cache[..., 2 * n:2 * n + page * dim // 32], cache[..., 2 * n + page * dim // 32:]
    res = []
    for codes, exps, key in ((parts[0], parts[2], True), (parts[1], parts[3], False)):
        rows = codes.reshape(*cache.shape[:2], page, dim // 2)
        exps = exps.reshape(*cache.shape[:2], page, dim // 32).to(torch.float64)
        place = torch.empty(dim, dtype=torch.long)
        for c in range(4 if key else 8):
            for i in range(dim // 8 if key else dim // 16):
                at = 32 * (i // 4) + 8 * c + 2 * (i % 4) if key else 16 * i + 2 * c
                place[at] = 2 * (c * (dim // 8 if key else dim // 16) + i)
                place[at + 1] = place[at] + 1
        nibbles = torch.stack([rows & 15, rows >> 4], dim=-1).flatten(-2)[..., place]
        table = torch.tensor(GRID + [-g for g in GRID], dtype=torch.float64)
        scale = torch.where(exps == 0, 0.0, torch.where(exps == 255, math.nan, torch.exp2(exps - 127)))
        res.append(table[nibbles.long()] * scale.repeat_interleave(32, dim=-1))
    return res
