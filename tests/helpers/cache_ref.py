"""Attention of single tokens over the 4-bit cache in 64 bits, with a bound in which every token's value counts with that token's weight."""
import torch

from .block_ref import HALF, LEAST, cache_values


def attention(q, cache, page, table, lengths, scale):
    """(out, bound).  Keys and values are exact, and so are scores but for binary32: D products and their sum, by instructions that cut (2^-23 each), and
    queries in binary16 beside their head's largest value.  A weight and its sum are off by that twice; the weight is then rounded to binary16 (2^-11), or
    where its product with the power of two of the value's group falls below binary16's normal numbers by 2^-25 of 2^9 of the largest weight, relative to a
    power of two 2^14 above that of the least group that is not all zeros: with codes of up to 6, where that group's largest is 3 or more, 2^-25 2^-9 2^14 6/3
    = 2^-19 of the largest weight times that largest value, or of what the token with the largest weight has, for each token."""
    B, H, D = q.shape
    keys, values = (t.cuda() for t in cache_values(cache.cpu(), page, D))
    out = torch.zeros(B, H, D, dtype=torch.float64, device="cuda")
    bound = torch.zeros_like(out)
    for b in range(B):
        n = min(max(int(lengths[b]), 0), table.shape[1] * page)
        pos = torch.arange(n, device="cuda")
        at = table[b, pos // page].long()
        there = (at >= 0) & (at < cache.shape[0])
        pos, at = pos[there], at[there]
        if pos.numel() == 0:
            continue
        K, V = keys[at, :, pos % page], values[at, :, pos % page]
        for h in range(H):
            g = h // (H // cache.shape[1])
            x = q[b, h].double()
            s = K[:, g] @ x * scale
            off = ((D + 16) * 2.0 ** -23 * (K[:, g].abs() @ x.abs()) + 2.0 ** -24 * x.abs().max() * K[:, g].abs().sum(1)).max() * scale + 2.0 ** -20
            p = torch.softmax(s, 0)
            v = V[:, g]
            largest = v.abs().view(len(pos), D // 32, 32).amax(2)
            least = torch.where(largest > 0, largest, torch.inf).amin(0).nan_to_num(posinf=0.0)
            floor = len(pos) * 2.0 ** -19 * torch.maximum(p @ largest, p.max() * least).repeat_interleave(32)
            out[b, h] = p @ v
            bound[b, h] = HALF[q.dtype] * out[b, h].abs() + (2.0 ** -11 + 2 * off + (len(pos) + 64) * 2.0 ** -23) * (p @ v.abs()) + LEAST[q.dtype] + floor
    return out, bound
