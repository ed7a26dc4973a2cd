"""What a transformer block needs between its linear layers, as measurable cases: rotary positions, attention over whole prompts with its
gradients, and a key-value cache held in 4 bits with the attention that reads it.

  rotary     pair (x, y) of a head at position p, frequency f:  (x cos pf - y sin pf, x sin pf + y cos pf); inverse: the angle's negative,
             which is also the gradient.  Angles are formed in 64 bits: at position 100000 a 32-bit one is off by 0.004
  attention  out[i] = sum_j softmax_j(scale q[i] k[j]) v[j] over the keys j of i's own sequence, with a causal mask j - i <= keys - queries;
             a row without keys gives 0.  Query head h reads key-value head h // (query heads / key-value heads)
  backward   ds = p (dp - sum p dp),  grad_q = scale ds k,  grad_k = scale ds^T q,  grad_v = p^T g, the latter two summed over a group's heads
  cache      32 neighbouring values of a head share a power of two, the smallest 2^e >= 2^-126 with max <= 6 2^e; each is then the nearest
             of 0, 1/2, 1, 3/2, 2, 3, 4, 6 times +-2^e (ties to the even code).  Pages of `page` tokens, found through a block table
  read       cached keys and values as numbers again (a chunked prompt attends to its earlier part)

A (page, head) of the cache is one run of bytes: key codes [page][D/2], value codes [page][D/2], key exponents [page][D/32], value
exponents [page][D/32] (exponent byte e + 127).  The low half of a byte is the first of two neighbouring dimensions.  A key row's byte
c (D/8) + 4 g + j holds dimensions 32 g + 8 c + 2 j, +1 (c, j < 4), a value row's byte r (D/16) + i holds 16 i + 2 r, +1 (r < 8).

`listed()` are named representatives, `draw(rng)` gives further cases of the same ranges.  A case is a dict of plain values.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
MAX_SCORES = 1 << 31      # query-key pairs over all heads of an attention case, at most (half as many without a mask)
MAX_CACHE = 1 << 21       # cached (token, head) pairs, at most


def _case(op, name=None, **kw):
    c = dict(op=op, **kw)
    return c if name is None else dict(c, name=name)


def _rotary(tokens, heads, kv, dim, rot, name=None, layout="half", inverse=False, scaling="none", far=0, dtype="bf16", fused=False):
    return _case("rotary", name, tokens=tokens, heads=heads, kv=kv, dim=dim, rot=rot, layout=layout, inverse=inverse, scaling=scaling, far=far,
                 dtype=dtype, fused=fused)


def _attention(op, lengths, heads, kv, dim, name=None, causal=True, dtype="bf16", out="same", prefix="", fused=False):
    """lengths, prefix: texts of numbers, as cases hold plain values; prefix: how many more keys than queries (negative: fewer) a sequence has"""
    return _case(op, name, lengths=lengths, heads=heads, kv=kv, dim=dim, causal=causal, dtype=dtype, out=out, prefix=prefix, fused=fused)


def _cache(op, lengths, heads, kv, dim, name=None, page=64, dtype="bf16", out="same", new=""):
    return _case(op, name, lengths=lengths, heads=heads, kv=kv, dim=dim, page=page, dtype=dtype, out=out, new=new)


def listed():
    return [
        # one new token of each of four sequences, deep in their texts: latency is all of it
        _rotary(4, 32, 8, 128, 128, far=100000, scaling="ramp", name="rotary_token"),
        # a prompt while fine-tuning, backward, queries and keys as slices of the projection's output
        _rotary(8191, 32, 8, 128, 128, inverse=True, scaling="ramp", fused=True, name="rotary_prompt"),
        # part of the head, pairs side by side, a ragged batch in binary16
        _rotary(1237, 12, 12, 96, 40, layout="interleaved", scaling="linear", far=5000, dtype="f16", name="rotary_partial"),
        # a BERT-base layer on 32 sentences of 128 tokens: 12 heads of 64, codes for the output projection
        _attention("attention", " ".join(["128"] * 32), 12, 12, 64, causal=False, out="e4m3", name="attention_sentences"),
        # packed requests of different lengths, one of them a single token, one going on behind a cached part
        _attention("attention", "1 517 64 1300 129 33 2003", 16, 4, 80, dtype="f16", prefix="0 0 448 0 0 -5 0", name="attention_packed"),
        # one long prompt, grouped heads
        _attention("attention", "8192", 32, 8, 128, fused=True, name="attention_prompt"),
        # gradients of packed sequences
        _attention("attention_backward", "700 1 999 255 93", 12, 12, 64, dtype="f16", name="attention_backward_packed"),
        # gradients of two long sequences, grouped heads
        _attention("attention_backward", "4096 4096", 16, 4, 128, name="attention_backward_prompt"),
        # one new token of one short request
        _cache("cache_attention", "777", 32, 8, 128, name="cache_token"),
        # 48 requests that decode together, every one at a length of its own
        _cache("cache_attention", " ".join(str(1 + (i * 2654435761) % 16384) for i in range(1, 49)), 32, 8, 128, name="cache_batch"),
        # the new tokens of a batch: one each, and a request that enters with its prompt's end
        _cache("cache_append", " ".join(str(64 * i + i % 7) for i in range(16)), 32, 8, 128, new=" ".join(["1"] * 15 + ["33"]), page=16,
               name="cache_new_tokens"),
        # a whole prompt into the cache and back out for its next part
        _cache("cache_append", "0 96 0", 16, 8, 128, new="8192 1000 2741", name="cache_prompt"),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def _text(values):
    return " ".join(str(v) for v in values)


def draw(rng):
    op = rng.choice(["rotary", "attention", "attention", "attention_backward", "attention_backward", "cache_attention", "cache_attention",
                     "cache_append"])
    kv = rng.choice([1, 2, 4, 8, 12])
    group = rng.choice([1, 1, 2, 3, 4, 8]) if kv <= 4 else rng.choice([1, 1, 2, 4])
    heads, dtype = kv * group, rng.choice(["bf16", "bf16", "f16"])
    if op == "rotary":
        dim = rng.choice([64, 80, 96, 128, 256])
        rot = rng.choice([dim, dim, dim // 2, 2 * rng.randint(4, dim // 2)])
        return _rotary(_log_int(rng, 1, 8192), heads, kv, dim, rot, layout=rng.choice(["half", "interleaved"]), inverse=rng.random() < 0.4,
                       scaling=rng.choice(["none", "linear", "base", "ramp"]), far=rng.choice([0, 0, 3000, 200000]),
                       dtype=rng.choice([dtype, dtype, "f32"]), fused=rng.random() < 0.5)
    if op in ("attention", "attention_backward"):
        dim = rng.choice([32, 64, 64, 80, 96, 128, 128, 8 * rng.randint(2, 16)])
        causal = rng.random() < 0.7
        while True:
            lengths = [_log_int(rng, 1, 8192) for _ in range(rng.choice([1, 1, 2, 3, 7, 20]))]
            more = [rng.choice([0, 0, 0, _log_int(rng, 1, 2048), -rng.randint(0, n)]) for n in lengths] if rng.random() < 0.3 else []
            scores = sum(n * (n + (more[i] if more else 0)) for i, n in enumerate(lengths)) * heads * (1 if causal else 2)
            if scores <= (MAX_SCORES if op == "attention" else MAX_SCORES // 4):
                break
        return _attention(op, _text(lengths), heads, kv, dim, causal=causal, dtype=dtype, prefix=_text(more), fused=rng.random() < 0.4,
                          out=rng.choice(["same", "same", "e4m3", "m4e3"]) if op == "attention" else "same")
    dim, page = rng.choice([32, 64, 96, 128, 128]), rng.choice([16, 32, 64, 64, 128])
    if op == "cache_attention":
        kv = rng.choice([1, 2, 4, 8])
        heads = kv * rng.choice([1, 2, 4, 5, 8, 12, 16])
        while True:
            lengths = [rng.choice([_log_int(rng, 1, 32768), _log_int(rng, 1, 2000)]) for _ in range(rng.choice([1, 1, 2, 5, 16, 64, 128]))]
            if sum(lengths) * kv <= MAX_CACHE:
                break
        if len(lengths) > 2 and rng.random() < 0.2:
            lengths[rng.randrange(len(lengths))] = 0    # a free place in the batch
        return _cache(op, _text(lengths), heads, kv, dim, page=page, dtype=dtype, out=rng.choice(["same", "same", "e4m3"]))
    n = rng.choice([1, 2, 5, 16, 64])
    one_each = rng.random() < 0.4
    new = [1 if one_each else _log_int(rng, 1, 8192 // n) for _ in range(n)]
    return _cache(op, _text([rng.choice([0, _log_int(rng, 1, 4000)]) for _ in range(n)]), heads, kv, dim, page=page, dtype=dtype, new=_text(new))


def _numbers(text):
    return [int(w) for w in text.split()]


def _key_lengths(case):
    more = _numbers(case["prefix"])
    return [n + (more[i] if more else 0) for i, n in enumerate(_numbers(case["lengths"]))]


def _sums(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


# ------------------------------------------------------------------ inputs
def _frequencies(case):
    """64-bit frequencies of a head's pairs, and the factor of the rotated values"""
    n, kind = case["rot"] // 2, case["scaling"]
    base = 10000.0 * (8.0 ** (case["rot"] / (case["rot"] - 2)) if kind == "base" and n > 1 else 1.0)
    f = base ** (-torch.arange(n, dtype=torch.float64) / n)
    if kind == "linear":
        f = f / 4.0
    if kind == "ramp":  # slow pairs are stretched eightfold, fast ones kept, those between blended by their turns within 8192 tokens
        keep = ((8192 * f / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
        f = keep * f + (1 - keep) * f / 8.0
    return f, (0.1 * math.log(8.0) + 1.0 if kind == "ramp" else 1.0)


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _pack_rows(codes, key):
    """4-bit codes [..., D] as cache rows [..., D/2]"""
    d = codes.shape[-1]
    pairs = codes[..., 0::2] | (codes[..., 1::2] << 4)
    if key:   # bytes (g, c, j) -> (c, g, j)
        return pairs.unflatten(-1, (d // 32, 4, 4)).transpose(-3, -2).flatten(-3)
    return pairs.unflatten(-1, (d // 16, 8)).transpose(-2, -1).flatten(-2)   # (i, r) -> (r, i)


def _unpack_rows(rows, key):
    d = rows.shape[-1] * 2
    if key:
        pairs = rows.unflatten(-1, (4, d // 32, 4)).transpose(-3, -2).flatten(-3)
    else:
        pairs = rows.unflatten(-1, (8, d // 16)).transpose(-2, -1).flatten(-2)
    return torch.stack([pairs & 15, pairs >> 4], dim=-1).flatten(-2)


def _encode4(x):
    """(codes, exponent bytes) of float32 values [..., D]; scaling by a power of two is exact"""
    m, e = torch.frexp(x.unflatten(-1, (-1, 32)).abs().amax(-1))        # max = m 2^e, 1/2 <= m < 1: 6 2^(e-3) is 3/4 2^e
    e = torch.where(m > 0.75, e - 2, e - 3).clamp_min(-126)
    e = torch.where(m == 0, -126, e)
    s = torch.ldexp(x.unflatten(-1, (-1, 32)), -e[..., None])
    mag = s.abs()
    code = torch.zeros_like(mag, dtype=torch.uint8)
    for i, (border, up) in enumerate([(0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)]):
        code += ((mag >= border) if up else (mag > border)).to(torch.uint8)
    return (code | ((s < 0).to(torch.uint8) << 3)).flatten(-2), (e + 127).to(torch.uint8)


def _decode4(codes, exponents, dtype):
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=dtype, device=codes.device)
    v = torch.where(codes >= 8, -table[(codes & 7).long()], table[(codes & 7).long()])
    return (v.unflatten(-1, (-1, 32)) * torch.exp2(exponents.to(dtype) - 127)[..., None]).flatten(-2)


def _planes(cache, page, dim):
    """views of the four planes of a cache [pages][heads][bytes], rows last but one"""
    sizes = [page * dim // 2] * 2 + [page * dim // 32] * 2
    return [p.unflatten(-1, (page, -1)) for p in cache.split(sizes, dim=-1)]


def _prepare_cache(case, g, lengths, room):
    """cache, block table; `lengths` tokens are there, `room` fit"""
    page, dim, kv = case["page"], case["dim"], case["kv"]
    blocks = [-(-n // page) for n in room]
    width, pages = max(blocks + [1]), sum(blocks) + 3
    table = torch.full((len(room), width), -1, dtype=torch.int32, device="cuda")
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    at = 0
    for b, n in enumerate(blocks):
        table[b, :n] = order[at:at + n]
        at += n
    cache = torch.zeros(pages, kv, page * (dim + dim // 16), dtype=torch.uint8, device="cuda")
    spread = 1 + 3 * (torch.rand(kv, 1, dim, generator=g, device="cuda") < 0.03)   # keys have a few wide channels
    for p in range(0, pages, 512):
        part = _planes(cache[p:p + 512], page, dim)
        for i in range(2):
            x = _normal(g, part[i].shape[0], kv, page, dim)
            codes, exps = _encode4(x * spread if i == 0 else x)
            part[i].copy_(_pack_rows(codes, i == 0))
            part[2 + i].copy_(exps)
    return cache, table


def _cuda_ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = {"case": case}
    dtype = DTYPES[case["dtype"]]
    heads, kv, dim = case["heads"], case["kv"], case["dim"]

    def qkv(tq, tk):
        if case.get("fused") and tq == tk:   # slices of one projection's output
            x = _normal(g, tq, heads + 2 * kv, dim).to(dtype)
            return x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:]
        return [_normal(g, t, h, dim).to(dtype) for t, h in ((tq, heads), (tk, kv), (tk, kv))]

    if case["op"] == "rotary":
        st["q"], st["k"], _ = qkv(case["tokens"], case["tokens"])
        first = torch.randint(0, case["far"] + 1, (case["tokens"],), generator=g, device="cuda") if case["tokens"] < 64 else case["far"]
        st["positions"] = (torch.arange(case["tokens"], device="cuda") + first).to(torch.int32)
        f, st["scale"] = _frequencies(case)
        st["freqs"] = f.cuda()
    elif case["op"].startswith("attention"):
        lq, lk = _numbers(case["lengths"]), _key_lengths(case)
        st["cu_q"], st["cu_k"] = _cuda_ints(_sums(lq)), _cuda_ints(_sums(lk))
        st["q"], st["k"], st["v"] = qkv(sum(lq), sum(lk))
        if case["op"] == "attention":
            st["out_scale"] = torch.full((1,), (1.0 if case["causal"] else 0.5) / (448.0 if case["out"] == "e4m3" else 248.0), device="cuda")
        else:   # what the forward pass kept, and a gradient (scaled with the loss in binary16)
            st["grad"] = (_normal(g, sum(lq), heads, dim) * (1e-3 if case["dtype"] == "bf16" else 1.0)).to(dtype)
            out, st["lse"] = _attend(st, torch.float32)
            st["out"] = out.to(dtype)
    else:
        lengths = _numbers(case["lengths"])
        st["lengths"] = _cuda_ints(lengths)
        if case["op"] == "cache_attention":
            st["cache"], st["table"] = _prepare_cache(case, g, lengths, lengths)
            st["q"] = _normal(g, len(lengths), heads, dim).to(dtype)
            st["out_scale"] = torch.full((1,), 1.0 / 448.0, device="cuda")
        else:
            new = _numbers(case["new"])
            st["cache"], st["table"] = _prepare_cache(case, g, lengths, [a + b for a, b in zip(lengths, new)])
            st["cu"], st["tokens"] = _cuda_ints(_sums(new)), sum(new)
            wide = 1 + 3 * (torch.rand(kv, dim, generator=g, device="cuda") < 0.03)
            st["k"], st["v"] = (_normal(g, sum(new), kv, dim) * wide).to(dtype), _normal(g, sum(new), kv, dim).to(dtype)
    return st


# ------------------------------------------------------------------ plain form
def _rotate(st, x):
    case, n = st["case"], st["case"]["rot"] // 2
    angle = (st["positions"].to(torch.float64)[:, None] * st["freqs"]) * (-1.0 if case["inverse"] else 1.0)
    cos, sin = ((t(angle) * st["scale"]).to(torch.float32)[:, None] for t in (torch.cos, torch.sin))
    v = x.to(torch.float32)
    out = v.clone()
    if case["layout"] == "half":
        a, b = v[..., :n], v[..., n:2 * n]
        out[..., :n], out[..., n:2 * n] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = v[..., 0:2 * n:2], v[..., 1:2 * n:2]
        out[..., 0:2 * n:2], out[..., 1:2 * n:2] = a * cos - b * sin, a * sin + b * cos
    return out.to(x.dtype)


def _pieces(case):
    """(sequence's query rows, its key rows, offset of the causal mask), sequence after sequence"""
    lq, lk = _numbers(case["lengths"]), _key_lengths(case)
    cq, ck = _sums(lq), _sums(lk)
    return [(slice(cq[i], cq[i + 1]), slice(ck[i], ck[i + 1]), lk[i] - lq[i]) for i in range(len(lq))]


def _scores(case, q, k, off, dtype):
    """scores of some heads' rows [heads][queries][keys], -inf where the mask holds"""
    s = (q.to(dtype).transpose(0, 1) @ k.to(dtype).permute(1, 2, 0)) * case["dim"] ** -0.5
    if case["causal"]:
        i, j = torch.arange(s.shape[1], device=s.device), torch.arange(s.shape[2], device=s.device)
        s = s.masked_fill(j > i[:, None] + off, float("-inf"))
    return s


def _attend(st, dtype):
    """(out, log of the sums [heads][queries]) in 32 or 64 bits"""
    case, q, k, v = st["case"], st["q"], st["k"], st["v"]
    group = case["heads"] // case["kv"]
    out = torch.zeros(q.shape, dtype=dtype, device=q.device)
    lse = torch.full((case["heads"], q.shape[0]), float("-inf"), dtype=dtype, device=q.device)
    for rows, keys, off in _pieces(case):
        if rows.stop == rows.start or keys.stop == keys.start:
            continue
        for h in range(case["kv"]):
            hs = slice(h * group, (h + 1) * group)
            s = _scores(case, q[rows, hs], k[keys, h:h + 1], off, dtype)
            m = s.amax(-1, keepdim=True).clamp_min(-1e30)
            p = torch.exp(s - m)
            total = p.sum(-1, keepdim=True)
            lse[hs, rows] = (m + torch.log(total))[..., 0]
            out[rows, hs] = torch.where(total > 0, (p @ v[keys, h].to(dtype)) / total, torch.zeros((), dtype=dtype, device=q.device)).transpose(0, 1)
    return out, lse


def _attention_gradients(st, dtype):
    case, q, k, v, g = st["case"], st["q"], st["k"], st["v"], st["grad"]
    group, scale = case["heads"] // case["kv"], case["dim"] ** -0.5
    dq, dk, dv = (torch.zeros(t.shape, dtype=dtype, device=t.device) for t in (q, k, v))
    for rows, keys, off in _pieces(case):
        if rows.stop == rows.start or keys.stop == keys.start:
            continue
        for h in range(case["heads"]):
            hk = h // group
            s = _scores(case, q[rows, h:h + 1], k[keys, hk:hk + 1], off, dtype)[0]
            m = s.amax(-1, keepdim=True).clamp_min(-1e30)
            p = torch.exp(s - m)
            total = p.sum(-1, keepdim=True)
            p = torch.where(total > 0, p / total, torch.zeros((), dtype=dtype, device=q.device))
            gh = g[rows, h].to(dtype)
            dv[keys, hk] += p.T @ gh
            dp = gh @ v[keys, hk].to(dtype).T
            ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * scale
            dq[rows, h] = ds @ k[keys, hk].to(dtype)
            dk[keys, hk] += ds.T @ q[rows, h].to(dtype)
    return dq, dk, dv


def _codes(t, scale, kind):
    """nearest codes of t / scale, as the values that they stand for"""
    x = t / scale
    if kind == "e4m3":
        return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    mag = x.abs().clamp(max=248.0)
    e = torch.frexp(mag.clamp_min(1.0))[1] - 1
    r = torch.ldexp(torch.round(torch.ldexp(mag.clamp_min(1.0), 4 - e)), e - 4)      # 1 stands for zero: the smallest is 1.0625
    r = torch.where(mag <= 0.53125, torch.zeros_like(r), r.clamp(1.0625, 248.0))
    return torch.where(x < 0, -r, r).to(torch.bfloat16)


def _rounded(st, t):
    case = st["case"]
    return t.to(DTYPES[case["dtype"]]) if case["out"] == "same" else _codes(t, st["out_scale"], case["out"])


def _cached(st, b, first, count, dtype):
    """keys and values [count][kv][dim] of sequence b from position `first` on"""
    case = st["case"]
    page, dim = case["page"], case["dim"]
    pos = torch.arange(first, first + count, device="cuda")
    pages, rows = st["table"][b, pos // page].long(), pos % page
    kc, vc, ke, ve = _planes(st["cache"], page, dim)
    out = []
    for codes, exps, key in ((kc, ke, True), (vc, ve, False)):
        out.append(_decode4(_unpack_rows(codes[pages, :, rows], key), exps[pages, :, rows], dtype))
    return out


def _cache_attend(st, dtype):
    case, q = st["case"], st["q"]
    out = torch.zeros(q.shape, dtype=dtype, device=q.device)
    group = case["heads"] // case["kv"]
    for b, n in enumerate(_numbers(case["lengths"])):
        if n:
            k, v = _cached(st, b, 0, n, dtype)
            s = (q[b].to(dtype).unflatten(0, (case["kv"], group)) @ k.permute(1, 2, 0)) * case["dim"] ** -0.5
            p = torch.exp(s - s.amax(-1, keepdim=True))
            out[b] = ((p @ v.transpose(0, 1)) / p.sum(-1, keepdim=True)).flatten(0, 1)
    return out


def _append(st):
    case = st["case"]
    page, starts, new = case["page"], _numbers(case["lengths"]), _numbers(case["new"])
    at = torch.cat([torch.arange(s, s + n, device="cuda") for s, n in zip(starts, new)])
    seq = torch.repeat_interleave(torch.arange(len(new), device="cuda"), torch.tensor(new, device="cuda"))
    pages, rows = st["table"][seq, at // page].long(), at % page
    kc, vc, ke, ve = _planes(st["cache"], page, case["dim"])
    for x, codes, exps, key in ((st["k"], kc, ke, True), (st["v"], vc, ve, False)):
        c, e = _encode4(x.to(torch.float32))
        codes[pages, :, rows] = _pack_rows(c, key)
        exps[pages, :, rows] = e


def _plain(st):
    case = st["case"]
    if case["op"] == "rotary":
        return {"q": _rotate(st, st["q"]), "k": _rotate(st, st["k"])}
    if case["op"] == "attention":
        out, lse = _attend(st, torch.float32)
        return {"out": _rounded(st, out), "lse": lse}
    if case["op"] == "attention_backward":
        return dict(zip(("grad_q", "grad_k", "grad_v"), (t.to(DTYPES[case["dtype"]]) for t in _attention_gradients(st, torch.float32))))
    if case["op"] == "cache_attention":
        return {"out": _rounded(st, _cache_attend(st, torch.float32))}
    _append(st)
    parts = [_cached(st, b, s, n, torch.float32) for b, (s, n) in enumerate(zip(_numbers(case["lengths"]), _numbers(case["new"])))]
    return {"k": torch.cat([p[0] for p in parts]).to(DTYPES[case["dtype"]]), "v": torch.cat([p[1] for p in parts]).to(DTYPES[case["dtype"]])}


# ------------------------------------------------------------------ the framework's calls
def _own(st):
    from paper_2401_14110_b200 import FLAG_INPUT_M4E3, LbaFormat
    from paper_2401_14110_b200 import binding as lba
    case = st["case"]
    if case["op"] == "rotary":
        q, k = lba.lba_rotary(st["q"], st["k"], st["positions"], st["freqs"], interleaved=case["layout"] == "interleaved", inverse=case["inverse"],
                              scale=st["scale"])
        return {"q": q, "k": k}
    how = {}
    if case["out"] != "same":
        how = dict(out_dtype=torch.uint8, out_scale=st["out_scale"], prod_fmt=LbaFormat(7, 4, 0, 0, 1 + (FLAG_INPUT_M4E3 if case["out"] == "m4e3" else 0)))

    def values(out):
        if case["out"] == "same":
            return out
        if case["out"] == "e4m3":
            return out.view(torch.float8_e4m3fn)
        c = torch.arange(256, device="cuda")
        mag = torch.exp2(((c >> 4) & 7).float()) * (1 + (c & 15).float() / 16)
        return torch.where((c & 127) == 0, 0, torch.where(c >= 128, -mag, mag)).to(torch.bfloat16)[out.long()]

    if case["op"] == "attention":
        out, lse = lba.lba_attention(st["q"], st["k"], st["v"], st["cu_q"], st["cu_k"], causal=case["causal"], lse=True, **how)
        return {"out": values(out), "lse": lse}
    if case["op"] == "attention_backward":
        return dict(zip(("grad_q", "grad_k", "grad_v"), lba.lba_attention_backward(st["grad"], st["q"], st["k"], st["v"], st["out"], st["lse"],
                                                                                   st["cu_q"], st["cu_k"], causal=case["causal"])))
    if case["op"] == "cache_attention":
        return {"out": values(lba.lba_cache_attention(st["q"], st["cache"], case["page"], st["table"], st["lengths"], **how))}
    lba.lba_cache_append(st["k"], st["v"], st["cache"], case["page"], st["table"], st["lengths"], st["cu"])
    k, v = lba.lba_cache_read(st["cache"], case["page"], st["table"], st["lengths"], st["cu"], st["tokens"], DTYPES[case["dtype"]])
    return {"k": k, "v": v}


def run(state):
    if own:
        return _own(state)
    return _plain(state)


# ------------------------------------------------------------------ what a pass cannot do without
def _pairs(case):
    """query-key pairs of a head that the mask leaves"""
    total = 0
    for nq, nk in zip(_numbers(case["lengths"]), _key_lengths(case)):
        if case["causal"]:
            first = nk - nq + 1                     # keys of row 0; row i has i more
            rows = max(0, nq - max(0, 1 - first))   # rows that have any
            total += rows * (max(first, 1) + nk) // 2
        else:
            total += nq * nk
    return total


def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2}[case["dtype"]]
    heads, kv, dim = case["heads"], case["kv"], case["dim"]
    if case["op"] == "rotary":
        n = case["tokens"] * (heads + kv)
        return {"bytes": 2 * n * dim * size + 4 * case["tokens"] + 4 * case["rot"], "flops": 3 * n * case["rot"]}
    if case["op"].startswith("attention"):
        tq, tk = sum(_numbers(case["lengths"])), sum(_key_lengths(case))
        q, k = tq * heads * dim, tk * kv * dim
        if case["op"] == "attention":
            return {"bytes": q * size + 2 * k * size + q * (size if case["out"] == "same" else 1) + 4 * tq * heads, "flops": 4 * _pairs(case) * heads * dim}
        return {"bytes": (4 * q + 4 * k) * size + 4 * tq * heads, "flops": 10 * _pairs(case) * heads * dim}
    row = dim + dim // 16                           # bytes of a cached token's head, key and value
    if case["op"] == "cache_attention":
        lengths = _numbers(case["lengths"])
        q = len(lengths) * heads * dim
        return {"bytes": sum(lengths) * kv * row + q * (size + (size if case["out"] == "same" else 1)), "flops": 4 * sum(lengths) * heads * dim}
    n = sum(_numbers(case["new"])) * kv
    return {"bytes": 2 * n * row + 4 * n * dim * size, "flops": 8 * n * dim}


# ------------------------------------------------------------------ 64 bits, from the definition
def _rotate64(st, x):
    """the pairs as complex numbers times e^(i p f)"""
    case, n = st["case"], st["case"]["rot"] // 2
    turn = torch.remainder(st["positions"].double()[:, None] * st["freqs"], 2 * math.pi)
    w = torch.polar(torch.full_like(turn, st["scale"]), -turn if case["inverse"] else turn)[:, None]
    v = x.double()
    head, tail = v[..., :2 * n], v[..., 2 * n:]
    z = torch.view_as_complex((head.unflatten(-1, (2, n)).transpose(-1, -2) if case["layout"] == "half" else head.unflatten(-1, (n, 2))).contiguous())
    r = torch.view_as_real(z * w)
    return torch.cat([(r.transpose(-1, -2) if case["layout"] == "half" else r).flatten(-2), tail], dim=-1)


def _softmax64(case, q, k, nq, nk):
    """(weights, log of the sums) of one head's rows"""
    s = torch.einsum("id,jd->ij", q, k) / math.sqrt(case["dim"])
    seen = torch.ones(nq, nk, dtype=torch.bool, device=s.device)
    if case["causal"]:
        seen = torch.tril(seen, diagonal=nk - nq)
    s = torch.where(seen, s, torch.full_like(s, -math.inf))
    lse = torch.logsumexp(s, dim=1)
    return torch.where(seen, torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[:, None]), torch.zeros_like(s)), lse


def _attention64(st, backward):
    case, group = st["case"], st["case"]["heads"] // st["case"]["kv"]
    q, k, v = (st[n].double() for n in "qkv")
    out, lse = torch.zeros_like(q), torch.full((case["heads"], q.shape[0]), -math.inf, dtype=torch.float64, device=q.device)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    cq, ck = _sums(_numbers(case["lengths"])), _sums(_key_lengths(case))
    for b in range(len(cq) - 1):
        i, j = slice(cq[b], cq[b + 1]), slice(ck[b], ck[b + 1])
        nq, nk = cq[b + 1] - cq[b], ck[b + 1] - ck[b]
        if nq == 0 or nk == 0:
            continue
        for h in range(case["heads"]):
            p, lse[h, i] = _softmax64(case, q[i, h], k[j, h // group], nq, nk)
            out[i, h] = torch.einsum("ij,jd->id", p, v[j, h // group])
            if backward:
                g = st["grad"][i, h].double()
                dv[j, h // group] += torch.einsum("ij,id->jd", p, g)
                dp = torch.einsum("id,jd->ij", g, v[j, h // group])
                ds = p * (dp - torch.einsum("id,id->i", g, out[i, h])[:, None]) / math.sqrt(case["dim"])
                dq[i, h] = torch.einsum("ij,jd->id", ds, k[j, h // group])
                dk[j, h // group] += torch.einsum("ij,id->jd", ds, q[i, h])
    return (dq, dk, dv) if backward else (out, lse)


def _held64(st, t):
    """codes stand for what they are nearest to: the quotient itself, saturated"""
    case = st["case"]
    if case["out"] == "same":
        return t
    top = 448.0 if case["out"] == "e4m3" else 248.0
    return (t / st["out_scale"].double()).clamp(-top, top)


def _nearest64(x):
    """values [..., D] as the cache holds them, group by group, by their distance from every representable one"""
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=x.device)
    t = x.double().unflatten(-1, (-1, 32))
    top = t.abs().amax(-1, keepdim=True)
    unit = torch.exp2(torch.ceil(torch.log2(top.clamp_min(1e-300) / 6.0)).clamp_min(-126))
    unit = torch.where(6.0 * unit < top, unit * 2, torch.where((3.0 * unit >= top) & (unit > 2.0 ** -126), unit / 2, unit))   # (a logarithm may be off by a bit)
    a = t.abs() / unit
    best, far = torch.zeros_like(a), torch.full_like(a, math.inf)
    for i in (1, 3, 5, 7, 0, 2, 4, 6):   # of two equally near ones the even code comes later
        d = (a - grid[i]).abs()
        best, far = torch.where(d <= far, grid[i], best), torch.minimum(d, far)
    return (torch.sign(t) * best * unit).flatten(-2)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rotary":
        return {"q": _rotate64(st, st["q"]), "k": _rotate64(st, st["k"])}
    if case["op"] == "attention":
        out, lse = _attention64(st, False)
        return {"out": _held64(st, out), "lse": lse}
    if case["op"] == "attention_backward":
        return dict(zip(("grad_q", "grad_k", "grad_v"), _attention64(st, True)))
    if case["op"] == "cache_append":
        return {"k": _nearest64(st["k"]), "v": _nearest64(st["v"])}
    q, out = st["q"].double(), torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_numbers(case["lengths"])):
        for h in range(case["heads"] if n else 0):
            if h % (case["heads"] // case["kv"]) == 0:
                k, v = (t[:, h // (case["heads"] // case["kv"])] for t in _cached(st, b, 0, n, torch.float64))
            p = torch.softmax(torch.einsum("jd,d->j", k, q[b, h]) / math.sqrt(case["dim"]), dim=0)
            out[b, h] = torch.einsum("j,jd->d", p, v)
    return {"out": _held64(st, out)}
