"""What a layer does with the finished contraction, in 64 bits: activations and their slopes, the dropout generator, roundings."""
import math

import numpy as np
import torch

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def philox4x32(counter, key):
    """Ten rounds of Philox4x32 (Salmon et al., SC 2011) on Python integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        x, y = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(y >> 32) ^ c[1] ^ k[0], y & 0xFFFFFFFF, (x >> 32) ^ c[3] ^ k[1], x & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def keep_mask(M, N, p, seed, offset):
    """[M][N] bool: the elements that dropout keeps"""
    out = np.zeros((M, (N + 3) // 4 * 4), dtype=bool)
    below = math.floor(p * 2.0 ** 32 + 0.5)
    u = lambda v: v & 0xFFFFFFFFFFFFFFFF  # noqa: E731
    seed, offset = u(seed), u(offset)
    for m in range(M):
        for j in range((N + 3) // 4):
            w = philox4x32((j, m, offset & 0xFFFFFFFF, offset >> 32), (seed & 0xFFFFFFFF, seed >> 32))
            out[m, 4 * j:4 * j + 4] = [v >= below for v in w]
    return torch.from_numpy(out[:, :N].copy())


def act(z, name):
    z = z.double()
    if name == "relu":
        return torch.where(z <= 0, torch.zeros_like(z), z)
    if name == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def slope(z, name):
    z = z.double()
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


# A binary32 activation is off by at most |z| 2^-21.  gelu: the approximation of P by 7.5e-8, its five-term sum and the product with the
# density (at most 0.4) by 2^-23 together, 1 - q by 2^-25: 2.2e-7 < 2^-22, times |z|; two more products, 2^-23 of at most |z|.  The
# logistic function: an exponential off by (2 + 1.2 |x|) 2^-24 relative, and the slope s (1 - s) that takes it to s has x s (1 - s) <=
# 0.23 and s (1 - s) <= 1/4: below 2^-24 + 2^-25; the sum with 1 and the reciprocal (2 units) 2^-23.4 of s: below 2^-22 of 1.
ACT_ERR = 2.0 ** -21


def half_step(dtype, v):
    """what one rounding of v to dtype may change: half a step, in the subnormal range the type's own"""
    tiny = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, "e4m3": 2.0 ** -10, "m4e3": 2.0 ** -1 + 2.0 ** -5}[dtype]
    rel = {"e4m3": 2.0 ** -4, "m4e3": 2.0 ** -5}.get(dtype) or torch.finfo(dtype).eps / 2
    return v.abs() * rel + tiny

# A binary32 slope is off by at most 2^-18: a value as above (2^-21), and z times a density or s (1 - s) times a derivative that stays
# below 6 where the other factor is not 0 to the last bit; these are off by (2 + 1.2 x 9) 2^-24 relative, and z s (1 - s) u' <= 1.2.
SLOPE_ERR = 2.0 ** -18


def piece_err(dtype):
    """What is left of dz in the bfloat16 pieces that go with a result type: one rounding to 8 bits; a cut to 8 bits (remainder below
    2^-7) and a rounding of that; two cuts and the last eight of 24 bits, exact."""
    return {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -15, torch.float32: 0.0}[dtype]
