"""Linear and gated feed-forward layers on the narrow accumulator, forward and backward, as measurable cases.

Both layers take E4M3 (or M4E3) codes and accumulate as every contraction of this library does: products through Q_prod,
running sums through Q_acc after every addition (Eq. 4 of the paper), in sequential or chunked order.

  linear    z = scale_a[m] scale_b[n] y[m][n] + bias[n],   out = residual + drop(act(z))
  gated     z = gate projection, v = up projection of the same rows,   out = act(z) v
  backward  straight-through estimator: the quantisers (Q_prod, Q_acc and the operands' own) pass the gradient, so with
            dz = act'(z) drop(g):   grad_a = dz (scale_b B),   grad_b = dz^T (scale_a A),   grad_bias = sum over rows of dz

drop() keeps an element and divides it by 1 - p where a word of the counter-based generator Philox4x32-10 (Salmon et al.,
SC 2011) is at least p 2^32: words of row m, columns 4j to 4j+3, come from the counter (j, m, offset low, offset high) and
the key (seed low, seed high).  The mask is never stored; the backward pass draws it again.

`listed()` are named representatives, `draw(rng)` gives further cases of the same ranges.  A case is a dict of plain values.
"""
import numpy as np
import torch

own = False

CHUNKED, SEQUENTIAL = 1, 0
MAX_FORWARD = 1 << 33   # emulated multiply-adds of a forward case (both projections of a gated one), at most
MAX_BACKWARD = 1 << 36  # multiply-adds of a backward case's products, at most
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _case(op, M, N, K, order="chunk", chunk=16, man=7, exp=4, rounding="floor", wa="e4m3", act="none", dropout=0.0, residual="", bias=True,
          per_channel=True, dtype="bf16", pre="", name=None):
    c = dict(op=op, M=M, N=N, K=K, order=order, chunk=chunk, man=man, exp=exp, rounding=rounding, wa=wa, act=act, dropout=dropout,
             residual=residual, bias=bias, per_channel=per_channel, dtype=dtype, pre=pre)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # output projection of one new token, added to the residual stream: weights are all there is to read
        _case("linear", 1, 4096, 4096, residual="bf16", name="linear_token"),
        # the size of a unit of work in a notebook or a test, strictly sequential accumulation: latency is all of it
        _case("linear", 64, 64, 576, order="seq", act="gelu", bias=False, per_channel=False, dtype="f32", name="linear_small_seq"),
        # both projections of a gated feed-forward layer for one new token, codes for the next layer
        _case("gated", 1, 8192, 2048, act="silu", bias=False, dtype="codes", name="gated_token"),
        # the same for sixteen sequences that decode together
        _case("gated", 16, 4096, 1024, act="silu", bias=False, dtype="bf16", name="gated_rows16"),
        # down projection while fine-tuning: bias, dropout and the residual stream in one pass, dropped elements never stored
        _case("linear", 2048, 1024, 4096, dropout=0.1, residual="bf16", name="linear_train"),
        # a prompt through a gated layer while fine-tuning: the pre-activations are kept for the backward pass
        _case("gated", 1024, 4096, 1024, act="silu", bias=False, pre="bf16", name="gated_train"),
        # sizes that no tile divides, rows that are not 16-byte aligned, the paper's own operand bytes, nearest-even
        _case("linear", 333, 777, 1203, act="gelu_tanh", wa="m4e3", rounding="rne", residual="f16", dtype="f16", pre="f32", name="linear_ragged"),
        # backward of a feed-forward layer with its activation, a training batch
        _case("linear_backward", 4096, 4096, 1024, act="gelu", pre="bf16", name="linear_backward_4096"),
        # backward through dropout, gradients in 32 bits, sizes that no tile divides
        _case("linear_backward", 1000, 777, 1203, dropout=0.1, act="relu", dtype="f32", pre="f32", name="linear_backward_ragged"),
        # few rows: the end of a sequence, one short sequence
        _case("linear_backward", 32, 512, 512, act="gelu_tanh", dtype="f16", pre="f16", name="linear_backward_rows32"),
        # backward of a gated layer, a training batch: gradients of both projections and of their shared input
        _case("gated_backward", 4096, 4096, 1024, act="silu", bias=False, pre="bf16", name="gated_backward_4096"),
        # the same on a smaller batch with biases and scales per tensor
        _case("gated_backward", 500, 1024, 768, act="gelu", per_channel=False, pre="f32", dtype="bf16", name="gated_backward_500"),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def _size(rng, lo, hi):
    v = _log_int(rng, lo, hi)
    return v if rng.random() < 0.35 else max(16, v // 16 * 16)


def draw(rng):
    op = rng.choice(["linear", "linear", "gated", "linear_backward", "gated_backward"])
    act = rng.choice(["silu", "gelu", "gelu_tanh", "relu"] if op.startswith("gated") else ["none", "none", "gelu", "gelu_tanh", "relu", "silu"])
    pre = rng.choice(["bf16", "f32", "f16"])
    wa = rng.choice(["e4m3"] * 5 + ["m4e3"])
    halves = 2 if op.startswith("gated") else 1
    if op.endswith("backward"):
        while True:
            M, N, K = _log_int(rng, 1, 8192), _size(rng, 16, 8192), _size(rng, 16, 8192)
            if 2 * halves * M * N * K <= MAX_BACKWARD:
                break
        return _case(op, M, N, K, wa=wa, act=act, dropout=rng.choice([0.0, 0.1, 0.5]) if op == "linear_backward" else 0.0, bias=rng.random() < 0.5,
                     per_channel=rng.random() < 0.6, dtype=rng.choice(["bf16", "bf16", "bf16", "f16", "f32"]), pre=pre)
    order = rng.choice(["chunk"] * 4 + ["seq"])
    man, exp, rounding = rng.choice([(7, 4, "floor")] * 4 + [(7, 4, "rne"), (10, 5, "rne"), (5, 5, "floor"), (4, 4, "floor"), (10, 6, "floor")])
    while True:
        M = rng.choice([1, 1, _log_int(rng, 1, 64), _log_int(rng, 1, 4096)])
        N, K = _size(rng, 16, 16384), _size(rng, 16, 16384 if order == "chunk" else 4096)
        if halves * M * N * K <= MAX_FORWARD:
            break
    dtype = rng.choice(["bf16", "bf16", "f16", "f32", "codes"])
    linear = op == "linear"
    return _case(op, M, N, K, order=order, chunk=rng.choice([16, 16, 16, 32]), man=man, exp=exp, rounding=rounding, wa=wa, act=act,
                 dropout=rng.choice([0.0, 0.0, 0.1]) if linear else 0.0, residual=rng.choice(["", "bf16", "f32", "f16"]) if linear else "",
                 bias=rng.random() < 0.5, per_channel=rng.random() < 0.6, dtype=dtype, pre=rng.choice(["", "", pre]))


# ------------------------------------------------------------------ inputs
def _formats(case):
    """(prod_fmt, acc_fmt) as tuples (mantissa, exponent, bias, rounding, flags): the largest biases at which the largest
    product does not overflow, and half the logarithm of the chunk less for the sums (Sec. 3)."""
    m4e3 = case["wa"] == "m4e3"
    b = 2 ** case["exp"] - (16 if m4e3 else 18)
    rnd = 1 if case["rounding"] == "rne" else 0
    return (case["man"], case["exp"], b, rnd, 1 + (4 if m4e3 else 0)), (case["man"], case["exp"], b - 2, rnd, 1)


def _encode(v, wa):
    """float values -> uint8 codes, nearest, saturated"""
    if wa == "e4m3":
        return v.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
    mag = v.abs().clamp(max=248.0)
    e = torch.frexp(mag.clamp_min(1.0))[1] - 1
    idx = torch.round(torch.ldexp(mag.clamp_min(1.0), -e) * 16.0).to(torch.int32) - 16 + 16 * e   # a carry is the next binade's 0
    idx = torch.where(mag < 0.53125, 0, idx.clamp(1, 127))                                       # 1 stands for zero: nearest is 1.0625
    idx = torch.where(mag == 0.53125, 0, idx)
    return torch.where((v < 0) & (idx > 0), idx + 128, idx).to(torch.uint8)


def _decode(codes, wa, dtype):
    if wa == "e4m3":
        return codes.view(torch.float8_e4m3fn).to(dtype)
    c = torch.arange(256, device=codes.device)
    mag = torch.exp2(((c >> 4) & 7).to(dtype)) * (1 + (c & 15).to(dtype) / 16)
    table = torch.where((c & 127) == 0, 0, torch.where(c >= 128, -mag, mag)).to(dtype)
    return table[codes.to(torch.int64)]


def _quantise(t, wa, rows):
    """(codes, scale): the largest magnitude of the tensor, or of each row, becomes the largest code"""
    top = t.abs().amax(dim=1) if rows else t.abs().amax().reshape(1)
    scale = (top / (448.0 if wa == "e4m3" else 248.0)).clamp_min(1e-20)
    if wa == "m4e3":  # the flex-bias is a power of two
        scale = torch.exp2(torch.ceil(torch.log2(scale)))
    return _encode(t / (scale[:, None] if rows else scale), wa), scale.contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    M, N, K = case["M"], case["N"], case["K"]
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x = normal(M, K)
    x[:, torch.randint(0, K, (max(1, K // 100),), generator=g, device="cuda")] *= 10  # a few outlier features
    st = {"case": case, "formats": _formats(case)}
    st["a"], st["sa"] = _quantise(x, case["wa"], False)
    gated = case["op"].startswith("gated")
    for i in range(2 if gated else 1):
        st["b%d" % i], st["sb%d" % i] = _quantise(normal(N, K) * K ** -0.5, case["wa"], case["per_channel"])
        st["bias%d" % i] = normal(N) * 0.1 if case["bias"] else None
    st["rng"] = torch.randint(0, 1 << 40, (2,), generator=g, device="cuda")
    if case["op"].endswith("backward"):
        st["grad"] = (normal(M, N) * 1e-3).to(DTYPES[case["dtype"]])
        st["pre"] = normal(*([2, M, N] if gated else [M, N])).to(DTYPES[case["pre"]])
    else:
        st["residual"] = normal(M, N).to(DTYPES[case["residual"]]) if case["residual"] else None
        st["scale"] = torch.full((1,), 4.0 / 448.0, device="cuda")  # the next layer's scale, from calibration
    return st


# ------------------------------------------------------------------ plain form
def _quantiser(fmt):
    """Q of Eq. 2 in place on a 64-bit tensor: cut by the bits of the mantissa, flushed where the value itself is below 2^-b, held to R_OF"""
    man, exp, bias, rnd, _ = fmt
    cut, low, top = 52 - man, 2.0 ** -bias, 2.0 ** (2 ** exp - bias - 1) * (2 - 2.0 ** -man)

    def q(t):
        small = t.abs() < low
        u = t.view(torch.int64)
        if rnd:
            u += ((u >> cut) & 1) + ((1 << (cut - 1)) - 1)
        u &= -(1 << cut)
        return t.masked_fill_(small, 0.0).clamp_(-top, top)
    return q


def _accumulate(a, b, case, formats):
    """y[m][n] of Eq. 4 for codes a [M][K] and b [N][K]; sums are held in 64 bits, where a 24-bit sum would round before it is cut"""
    qp, qa = _quantiser(formats[0]), _quantiser(formats[1])
    K = a.shape[1]
    chunk = K if case["order"] == "seq" else min(case["chunk"], K)
    C = -(-K // chunk)
    pad = lambda t: torch.nn.functional.pad(_decode(t, case["wa"], torch.float64), (0, C * chunk - K)).reshape(-1, C, chunk)  # noqa: E731
    bv, out = pad(b).permute(2, 1, 0).contiguous(), torch.empty(a.shape[0], b.shape[0], dtype=torch.float64, device=a.device)
    rows = max(1, (1 << 27) // (C * b.shape[0]))
    for r in range(0, a.shape[0], rows):
        av = pad(a[r:r + rows])
        s = torch.zeros(av.shape[0], C, b.shape[0], dtype=torch.float64, device=a.device)
        for i in range(chunk):
            s = qa(s.add_(qp(av[:, :, i, None] * bv[i])))
        t = s[:, 0].clone()
        for j in range(1, C):
            t = qa(t.add_(s[:, j]))
        out[r:r + rows] = t
    return out.to(torch.float32)


def _project(st, i):
    z = _accumulate(st["a"], st["b%d" % i], st["case"], st["formats"]) * st["sa"] * st["sb%d" % i]
    return z if st["bias%d" % i] is None else z + st["bias%d" % i]


def _act(z, act):
    if act == "relu":
        return torch.where(z <= 0, torch.zeros_like(z), z)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh((2 / np.pi) ** 0.5 * (z + 0.044715 * z * z * z)))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * np.pi) ** -0.5
    if act == "gelu_tanh":
        c = (2 / np.pi) ** 0.5
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _kept(rng, M, N, p):
    """[M][N] truth values: what dropout keeps.  Words are held in 64-bit integers."""
    low = 0xFFFFFFFF
    key = [rng[0] & low, (rng[0] >> 32) & low]
    c = [torch.arange((N + 3) // 4, device=rng.device).expand(M, -1), torch.arange(M, device=rng.device)[:, None].expand(-1, (N + 3) // 4),
         rng[1] & low, (rng[1] >> 32) & low]
    for r in range(10):
        x, y = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((y >> 32) & low) ^ c[1] ^ key[0], y & low, ((x >> 32) & low) ^ c[3] ^ key[1], x & low]
        key = [(key[0] + 0x9E3779B9) & low, (key[1] + 0xBB67AE85) & low]
    return torch.stack([w.expand(M, (N + 3) // 4) for w in c], dim=-1).reshape(M, -1)[:, :N] >= int(p * 2.0 ** 32 + 0.5)


def _drop(st, t):
    p = st["case"]["dropout"]
    return torch.where(_kept(st["rng"], t.shape[0], t.shape[1], p), t * (1 / (1 - p)), torch.zeros_like(t)) if p else t


def _round(st, t):
    """to the output's type; codes of the operands' format, as the values they stand for (M4E3 ones in bfloat16, which holds them all)"""
    case = st["case"]
    if case["dtype"] != "codes":
        return t.to(DTYPES[case["dtype"]])
    codes = _encode(t / st["scale"], case["wa"])
    return _code_values(codes, case)


def _code_values(codes, case):
    return codes.view(torch.float8_e4m3fn) if case["wa"] == "e4m3" else _decode(codes, "m4e3", torch.bfloat16)


def _plain(st):
    case = st["case"]
    op, act = case["op"], case["act"]
    if op == "linear":
        z = _project(st, 0)
        t = _drop(st, _act(z, act))
        t = t if st["residual"] is None else t + st["residual"].to(torch.float32)
        out = {"out": _round(st, t)}
        return dict(out, pre=z.to(DTYPES[case["pre"]])) if case["pre"] else out
    if op == "gated":
        z, v = _project(st, 0), _project(st, 1)
        out = {"out": _round(st, _act(z, act) * v)}
        return dict(out, pre=torch.stack([z, v]).to(DTYPES[case["pre"]])) if case["pre"] else out
    g, pre, dt = st["grad"].to(torch.float32), st["pre"].to(torch.float32), DTYPES[case["dtype"]]
    a = _decode(st["a"], case["wa"], torch.float32) * st["sa"]
    b = [_decode(st["b%d" % i], case["wa"], torch.float32) * st["sb%d" % i].reshape(-1, 1) for i in range(2 if op == "gated_backward" else 1)]
    if op == "linear_backward":
        dz = [_drop(st, g) * _act_grad(pre, act)]
    else:
        dz = [g * pre[1] * _act_grad(pre[0], act), g * _act(pre[0], act)]
    out = {"grad_a": sum(d @ w for d, w in zip(dz, b)).to(dt)}
    for i, d in enumerate(dz):
        out["grad_b%d" % i] = (d.T @ a).to(dt)
        if case["bias"]:
            out["grad_bias%d" % i] = d.sum(dim=0)
    return out


# ------------------------------------------------------------------ the framework's calls
def _own(st):
    from paper_2401_14110_b200 import binding as lba
    case = st["case"]
    prod, acc = st["formats"]
    how = dict(order=SEQUENTIAL if case["order"] == "seq" else CHUNKED, chunk=case["chunk"], activation=case["act"])
    if case["op"] in ("linear", "gated"):
        how["out_dtype"] = torch.uint8 if case["dtype"] == "codes" else DTYPES[case["dtype"]]
        how["out_scale"] = st["scale"] if case["dtype"] == "codes" else None
        how["preact"] = DTYPES[case["pre"]] if case["pre"] else None
        if case["op"] == "linear":
            r = lba.lba_linear(st["a"], st["b0"], st["sa"], st["sb0"], st["bias0"], prod, acc, residual=st["residual"], dropout=case["dropout"],
                               rng=st["rng"] if case["dropout"] else None, **how)
        else:
            r = lba.lba_gated(st["a"], st["b0"], st["b1"], st["sa"], st["sb0"], st["sb1"], st["bias0"], st["bias1"], prod, acc, **how)
        out, pre = r if case["pre"] else (r, None)
        out = {"out": _code_values(out, case) if case["dtype"] == "codes" else out}
        return dict(out, pre=pre) if case["pre"] else out
    needs = (True, True, case["bias"])
    if case["op"] == "linear_backward":
        ga, gb, gc = lba.lba_linear_backward(st["grad"], st["a"], st["b0"], st["sa"], st["sb0"], prod, preact=st["pre"], activation=case["act"],
                                             dropout=case["dropout"], rng=st["rng"] if case["dropout"] else None, needs=needs)
        out = {"grad_a": ga, "grad_b0": gb}
        return dict(out, grad_bias0=gc) if case["bias"] else out
    ga, g0, g1, c0, c1 = lba.lba_gated_backward(st["grad"], st["a"], st["b0"], st["b1"], st["sa"], st["sb0"], st["sb1"], prod, st["pre"],
                                                activation=case["act"], needs=needs)
    if not case["bias"]:
        return {"grad_a": ga, "grad_b0": g0, "grad_b1": g1}
    return {"grad_a": ga, "grad_b0": g0, "grad_bias0": c0, "grad_b1": g1, "grad_bias1": c1}


def run(state):
    if own:
        return _own(state)
    return _plain(state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    M, N, K = case["M"], case["N"], case["K"]
    size = {"f32": 4, "bf16": 2, "f16": 2, "codes": 1, "": 0}
    halves = 2 if case["op"].startswith("gated") else 1
    read = M * K + halves * N * K + 4 * halves * ((N if case["per_channel"] else 1) + (N if case["bias"] else 0)) + 4
    if case["op"].endswith("backward"):
        moved = M * N * size[case["dtype"]] + halves * M * N * size[case["pre"]] + (M * K + halves * N * K) * size[case["dtype"]]
        return {"bytes": read + moved, "flops": 4 * halves * M * N * K}
    moved = M * N * (size[case["dtype"]] + size[case["residual"]]) + halves * M * N * size[case["pre"]]
    return {"bytes": read + moved, "flops": 2 * halves * M * N * K}


# ------------------------------------------------------------------ 64 bits, from the definition
def _q64(v, fmt):
    man, exp, bias, rnd, _ = fmt
    step = torch.ldexp(torch.ones_like(v), torch.frexp(v)[1] - 1 - man)   # of the grid of v's binade
    r = (torch.round(v / step) if rnd else torch.trunc(v / step)) * step
    top = 2.0 ** (2 ** exp - bias) - 2.0 ** (2 ** exp - bias - 1 - man)
    r = torch.where(r.abs() > top, torch.sign(r) * top, r)
    return torch.where(v.abs() >= 2.0 ** -bias, r, torch.zeros_like(v))


def _chains64(st, i):
    """Eq. 8-9 and the two hierarchies, one slice of the columns at a time; chunk by chunk along an axis in front"""
    case, (pf, af) = st["case"], st["formats"]
    a, b = _decode(st["a"], case["wa"], torch.float64), _decode(st["b%d" % i], case["wa"], torch.float64)
    M, K = a.shape
    L = case["chunk"] if case["order"] == "chunk" else K
    full = [list(range(s, min(s + L, K))) for s in range(0, K, L)]
    cols = max(1, (1 << 26) // max(1, len(full) * M))
    parts = []
    for n in range(0, b.shape[0], cols):
        w = b[n:n + cols]
        sums = torch.zeros(len(full), M, w.shape[0], dtype=torch.float64, device=a.device)
        for j in range(min(L, K)):
            k = torch.tensor([c[j] for c in full if j < len(c)], device=a.device)   # a short chunk is the last one
            p = _q64(torch.einsum("mc,nc->cmn", a[:, k], w[:, k]), pf)
            sums[:len(k)] = _q64(sums[:len(k)] + p, af)
        total = torch.zeros(M, w.shape[0], dtype=torch.float64, device=a.device)
        for c in range(len(full)):
            total = _q64(total + sums[c], af)
        parts.append(total)
    z = torch.cat(parts, dim=1) * st["sa"].double().reshape(-1, 1) * st["sb%d" % i].double().reshape(1, -1)
    return z if st["bias%d" % i] is None else z + st["bias%d" % i].double()


def _act64(z, act):
    """(value, derivative)"""
    if act == "relu":
        return z.clamp_min(0), (z > 0).double()
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * torch.sigmoid(-z)
    if act == "gelu":
        phi = torch.special.ndtr(z)
        return z * phi, phi + z * torch.exp(-z * z / 2) / np.sqrt(2 * np.pi)
    if act == "gelu_tanh":  # 1/2 (1 + tanh u) is the logistic function of 2u
        u2, du2 = np.sqrt(8 / np.pi) * (z + 0.044715 * z ** 3), np.sqrt(8 / np.pi) * (1 + 0.134145 * z ** 2)
        s = torch.sigmoid(u2)
        return z * s, s + z * s * torch.sigmoid(-u2) * du2
    return z, torch.ones_like(z)


def _factor64(st, shape):
    """what dropout multiplies by, from the generator in unsigned 32-bit words on the host"""
    p = st["case"]["dropout"]
    if not p:
        return torch.ones((), dtype=torch.float64, device="cuda")
    M, N = shape
    seed, offset = (int(v) for v in st["rng"].tolist())
    u = np.uint64
    words = np.zeros((4, M, (N + 3) // 4), dtype=np.uint32)
    words[0], words[1] = np.arange((N + 3) // 4, dtype=np.uint32)[None], np.arange(M, dtype=np.uint32)[:, None]
    words[2], words[3] = offset & 0xFFFFFFFF, offset >> 32
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        hi0 = (words[0].astype(u) * u(0xD2511F53)) >> u(32)
        hi1 = (words[2].astype(u) * u(0xCD9E8D57)) >> u(32)
        lo0, lo1 = words[0] * np.uint32(0xD2511F53), words[2] * np.uint32(0xCD9E8D57)
        words = np.stack([hi1.astype(np.uint32) ^ words[1] ^ np.uint32(k0), lo1, hi0.astype(np.uint32) ^ words[3] ^ np.uint32(k1), lo0])
        k0, k1 = (k0 + 0x9E3779B9) % 2 ** 32, (k1 + 0xBB67AE85) % 2 ** 32
    keep = np.moveaxis(words, 0, 2).reshape(M, -1)[:, :N].astype(np.float64) >= np.floor(p * 2.0 ** 32 + 0.5)
    return torch.from_numpy(keep / (1 - p)).cuda()


def _held64(st, t):
    """codes stand for what they are nearest to: the quotient itself, saturated"""
    case = st["case"]
    if case["dtype"] != "codes":
        return t
    top = 448.0 if case["wa"] == "e4m3" else 248.0
    return (t / st["scale"].double()).clamp(-top, top)


def exact(case, seed):
    st = prepare(case, seed)
    op, act = case["op"], case["act"]
    if op in ("linear", "gated"):
        z = _chains64(st, 0)
        v = _chains64(st, 1) if op == "gated" else None
        t = _act64(z, act)[0]
        if op == "linear":
            t = t * _factor64(st, t.shape)
            t = t if st["residual"] is None else t + st["residual"].double()
        else:
            t = t * v
        out = {"out": _held64(st, t)}
        return dict(out, pre=z if v is None else torch.stack([z, v])) if case["pre"] else out
    g, pre = st["grad"].double(), st["pre"].double()
    if op == "linear_backward":
        dz = [g * _factor64(st, g.shape) * _act64(pre, act)[1]]
    else:
        f, df = _act64(pre[0], act)
        dz = [g * pre[1] * df, g * f]
    x = _decode(st["a"], case["wa"], torch.float64) * st["sa"].double()
    w = [_decode(st["b%d" % i], case["wa"], torch.float64) * st["sb%d" % i].double().reshape(-1, 1) for i in range(len(dz))]
    out = {"grad_a": torch.cat(dz, dim=1) @ torch.cat(w, dim=0)}
    for i, d in enumerate(dz):
        out["grad_b%d" % i] = torch.einsum("mn,mk->nk", d, x)
        if case["bias"]:
            out["grad_bias%d" % i] = torch.einsum("mn->n", d)
    return out
