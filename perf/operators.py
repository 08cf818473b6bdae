"""The operators of a served model's 4-bit variant, as they are measured.

The options that the scheduler chooses from are variants (16-bit or 4-bit) and
runtime parameters (concurrency, batch) of the models that share the GPU.  One
step of such a 4-bit variant is made of three operators: products with 4-bit
weights, the append of new keys and values to a paged 4-bit cache with the
position rotation on the way, and attention over that cache.

A case is a dict of plain values:

  op      "w4" (the product), "append" (new rows into the cache, rotated, and
          read back), "attn" (attention over a filled cache)
  dtype   "bf16" or "f16": activations, queries, keys, values and results
  w4      M rows, N outputs, K inputs, G weights a scale, bias, zeros (own zero
          points or 8), pad (elements between the rows of x beyond K)
  cache   heads, kv_heads, D head size, G values a scale, page tokens a page
  batch   seqs sequences of kv_lo..kv_hi cached tokens (the new ones included),
          new_lo..new_hi of them new; mix numbers the lengths drawn in between
  append  rot rotated dims of D, inter: pairs (0,1), (2,3).. instead of halves
  attn    window (0: all earlier tokens), lse: the log of the softmax sum too

Lengths are a function of the case; everything else is drawn from the seed.
"""
import math
import random

import torch

own = False

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
F16_MAX = 65504.0


def _w4(**kw):
    return dict(dict(op="w4", dtype="bf16", M=1, N=4096, K=4096, G=128, bias=False, zeros=True, pad=0), **kw)


def _kv(op, **kw):
    c = dict(op=op, dtype="bf16", heads=32, kv_heads=8, D=128, G=64, page=16, seqs=1, kv_lo=1000, kv_hi=1000,
             new_lo=1, new_hi=1, mix=0)
    c.update(dict(rot=kw.get("D", 128), inter=False) if op == "append" else dict(window=0, lse=False))
    return dict(c, **kw)


def listed():
    return [
        # one request alone: a square projection of one token's activations
        _w4(name="w4_one_token"),
        # concurrency 4 (the options' largest), binary16, small groups, sizes that fill no tile
        _w4(name="w4_ragged", dtype="f16", M=4, N=5003, K=4128, G=32, bias=True, pad=24),
        # the options' largest batch, 2^5 rows, over a wide layer
        _w4(name="w4_batch32", M=32, N=8192, K=8192, G=64),
        # the output layer over a vocabulary, with several requests' draft tokens
        _w4(name="w4_vocabulary", dtype="f16", M=64, N=32768, K=8192, zeros=False),
        # one decode step of eight requests: one new token each
        _kv("append", name="append_step", seqs=8, kv_lo=200, kv_hi=2000),
        # a ragged mixed batch: some requests bring nothing, some a prompt; part of each head rotated, in pairs
        _kv("append", name="append_ragged", dtype="f16", heads=20, kv_heads=4, D=64, G=32, page=48, seqs=13, kv_lo=300,
            kv_hi=1500, new_lo=0, new_hi=300, rot=32, inter=True),
        # four whole prompts at once
        _kv("append", name="append_prompts", page=64, seqs=4, kv_lo=8192, kv_hi=8192, new_lo=8192, new_hi=8192),
        # the smallest call: one request's token over a short context
        _kv("attn", name="attn_one_request"),
        # 32 requests of all lengths decode together
        _kv("attn", name="attn_batch32", page=64, seqs=32, kv_lo=100, kv_hi=16384),
        # no shared heads, small heads and groups, short and empty requests, binary16
        _kv("attn", name="attn_own_heads", dtype="f16", heads=16, kv_heads=16, D=64, G=32, seqs=16, kv_lo=0, kv_hi=4000,
            lse=True),
        # two requests over very long contexts
        _kv("attn", name="attn_long", dtype="f16", G=128, page=128, seqs=2, kv_lo=120001, kv_hi=131072),
        # a piece of a prompt over what is cached of it: a thousand query tokens a request
        _kv("attn", name="attn_chunk", page=32, seqs=2, kv_lo=9000, kv_hi=12345, new_lo=1000, new_hi=1024),
    ]


def _log(rng, lo, hi):
    """A whole number, spread evenly over the logarithm of lo..hi."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    dtype = rng.choice(["bf16", "f16"])
    op = rng.choice(["w4", "append", "attn"])
    while True:
        if op == "w4":
            g = rng.choice([32, 64, 128])
            c = _w4(dtype=dtype, M=_log(rng, 1, 64), N=_log(rng, 500, 32768), K=g * _log(rng, max(1, 512 // g), 8192 // g), G=g,
                    bias=rng.random() < 0.4, zeros=rng.random() < 0.7, pad=rng.choice([0, 0, 8, 3]))
            if 3072 in (c["N"], c["K"]):
                continue
            return c
        kv = rng.choice([1, 2, 4, 8, 16])
        d = rng.choice([64, 128, 128, 256])
        c = dict(dtype=dtype, heads=kv * rng.choice([1, 3, 4, 5, 8] if kv < 16 else [1, 2]), kv_heads=kv, D=d,
                 G=rng.choice([g for g in (32, 64, 128) if g <= d]), page=16 * rng.choice([1, 1, 2, 3, 4, 8]),
                 mix=rng.randrange(1000))
        if op == "append":
            new = _log(rng, 1, 4096)
            c.update(new_lo=rng.choice([0, new]), new_hi=new, rot=rng.choice([d, d, d // 2]), inter=rng.random() < 0.3,
                     seqs=_log(rng, 1, max(1, min(64, 32768 // new))))
            c.update(kv_lo=new, kv_hi=new + _log(rng, 1, 4000))
            if c["seqs"] * new * (c["heads"] + 2 * kv) * d > 4 * 8192 * 48 * 128:
                continue
        else:
            new = 1 if rng.random() < 0.6 else _log(rng, 2, 1024)
            c.update(new_lo=new, new_hi=new, kv_hi=new + _log(rng, 1, 60000), seqs=_log(rng, 1, 64),
                     window=0 if rng.random() < 0.7 else _log(rng, 16, 4096), lse=rng.random() < 0.3)
            c["kv_lo"] = rng.choice([c["kv_hi"], c["kv_hi"] // 3 + 1, 0])
            # what the plain form holds of the cache and of the scores
            if c["seqs"] * c["kv_hi"] * max(2 * kv * d, c["heads"] * new) > 2 * 12345 * 32 * 1024:
                continue
        if 3072 in (c["kv_hi"], c.get("new_hi"), c["kv_lo"], c.get("window")):
            continue
        return _kv(op, **c)


def _lengths(c):
    """Per sequence: cached tokens, and how many of them are new."""
    r = random.Random("%d %d %d" % (c["mix"], c["seqs"], c["kv_hi"]))
    n = c["seqs"]
    kv = [r.randint(c["kv_lo"], c["kv_hi"]) for _ in range(n)]
    if n > 3:
        kv[r.randrange(n)] = c["kv_lo"]
    longest = r.randrange(n)
    kv[longest] = c["kv_hi"]
    new = [r.randint(c["new_lo"], c["new_hi"]) for _ in range(n)]
    new[longest] = c["new_hi"]
    return kv, [min(i, k) for i, k in zip(new, kv)] if c["op"] == "append" else new


def work(c):
    if c["op"] == "w4":
        m, n, k, g = c["M"], c["N"], c["K"], c["G"]
        return {"bytes": n * k / 2 + n * (k // g) * (3 if c["zeros"] else 2) + 2 * m * (k + n) + 2 * n * c["bias"],
                "flops": 2 * m * n * k}
    kv, new = _lengths(c)
    hq, hk, d, rows = c["heads"], c["kv_heads"], c["D"], sum(new)
    row = hk * (d + 8 * (d // c["G"]))  # a cached token, keys and values
    if c["op"] == "append":
        # rows of q, k, v in, q and the cached rows out, the cached rows in again and their values out
        return {"bytes": rows * (4 * hq * d + 8 * hk * d + 2 * row) + max(kv) * 4 * c["rot"], "flops": rows * (hq + 2 * hk) * d * 6}
    seen = sum(min(k, c["window"] + n - 1) if c["window"] else k for k, n in zip(kv, new))
    pairs = 0
    for k, n in zip(kv, new):
        for i in range(n):
            t = max(0, k - n + i + 1)
            pairs += min(t, c["window"]) if c["window"] else t
    return {"bytes": seen * row + rows * hq * (4 * d + 4 * c["lse"]), "flops": 4 * pairs * hq * d}


# ------------------------------------------------------------------ inputs

def _normal(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _w4_inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, m, n, k = DT[c["dtype"]], c["M"], c["N"], c["K"]
    x = torch.zeros(m, k + c["pad"], device="cuda", dtype=dt)[:, :k]
    # activations after a norm: most channels near 1, a few far larger
    x.copy_(_normal(g, m, k) * (1 + 8 * (torch.rand(k, device="cuda", generator=g) > 0.995)))
    codes = torch.randint(0, 256, (n, k // 2), device="cuda", generator=g, dtype=torch.uint8)
    scales = ((0.5 + torch.rand(n, k // c["G"], device="cuda", generator=g)) * (0.2 / math.sqrt(k))).to(dt)
    zeros = torch.randint(4, 12, scales.shape, device="cuda", generator=g, dtype=torch.uint8) if c["zeros"] else None
    bias = _normal(g, n).to(dt) if c["bias"] else None
    return x, codes, scales, zeros, bias


def _pages(c):
    return -(-c["kv_hi"] // c["page"])


def _cache_inputs(c, seed):
    """Lengths, page table, rotation, and the rows that the calls take."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, hk, d = DT[c["dtype"]], c["kv_heads"], c["D"]
    kv, new = _lengths(c)
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    s = dict(kv=kv, new=new, rows=start[-1])
    s["q_start"] = torch.tensor(start, dtype=torch.int32, device="cuda")
    s["kv_len"] = torch.tensor(kv, dtype=torch.int32, device="cuda")
    # pages in no order, as a server that has run for a while hands them out
    mp = _pages(c)
    s["n_pages"] = c["seqs"] * mp
    s["table"] = torch.randperm(s["n_pages"], device="cuda", generator=g).to(torch.int32).view(c["seqs"], mp)
    # keys have channels that are larger throughout
    s["wide"] = 1 + 3 * (torch.rand(hk, d, device="cuda", generator=g) > 0.95)
    s["q"] = _normal(g, s["rows"], c["heads"], d).to(dt)
    s["g"] = g
    return s


def _angles(c, n):
    half = c["rot"] // 2
    a = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    return a.cos().float(), a.sin().float()


def _fill(c, s, put):
    """All of the cache's tokens by put(q_start, kv_len, k, v), some positions of every sequence at a time."""
    hk, d, dt = c["kv_heads"], c["D"], DT[c["dtype"]]
    step = max(1, (1 << 28) // (c["seqs"] * hk * d))
    kv = s["kv_len"].long()
    for lo in range(0, max(s["kv"]), step):
        n = (kv - lo).clamp(0, step)
        rows = sum(min(max(k - lo, 0), step) for k in s["kv"])
        start = torch.zeros(c["seqs"] + 1, device="cuda", dtype=torch.int32)
        start[1:] = n.cumsum(0)
        k = (_normal(s["g"], rows, hk, d) * s["wide"]).to(dt)
        v = _normal(s["g"], rows, hk, d).to(dt)
        put(start, (kv.clamp(max=lo) + n).to(torch.int32), k, v, rows, min(step, max(s["kv"]) - lo))


def prepare(c, seed):
    if c["op"] == "w4":
        x, codes, scales, zeros, bias = _w4_inputs(c, seed)
        s = dict(c=c, x=x, bias=bias)
        if own:
            # weights are laid out once, when they are loaded
            from paper_2609_02109_amd import serve
            s["w"] = serve.W4Weight(codes, scales, zeros)
        else:
            s.update(codes=codes, scales=scales, zeros=zeros)
        return s
    s = dict(_cache_inputs(c, seed), c=c)
    if c["op"] == "append":
        s["cos"], s["sin"] = _angles(c, _pages(c) * c["page"])
        s["k"] = (_normal(s["g"], s["rows"], c["kv_heads"], c["D"]) * s["wide"]).to(DT[c["dtype"]])
        s["v"] = _normal(s["g"], s["rows"], c["kv_heads"], c["D"]).to(DT[c["dtype"]])
    # the cache as earlier calls left it
    if own:
        from paper_2609_02109_amd import serve
        cache = s["cache"] = serve.KV4Cache(s["n_pages"], c["page"], c["kv_heads"], c["D"], group=c["G"])
        s["batch"] = cache.batch(s["q_start"], s["kv_len"], s["table"], rows=s["rows"], max_new=max(s["new"]), max_kv=c["kv_hi"])
        if c["op"] == "attn":
            _fill(c, s, lambda start, kv, k, v, rows, most: cache.append(
                cache.batch(start, kv, s["table"], rows=rows, max_new=most, max_kv=c["kv_hi"]), k, v))
    else:
        _plain_cache(c, s)
        if c["op"] == "attn":
            _fill(c, s, lambda start, kv, k, v, rows, most: _plain_write(
                c, s, k.float(), v.float(), *_plain_slots(c, s, start, kv, rows)[:2]))
    del s["g"]
    return s


# -------------------------------------------------------------- plain forms

def _quantise(x, group):
    """Codes 0..15, scales and offsets of 32-bit (or 64-bit) rows, by groups of the last axis."""
    x = x.clamp(-F16_MAX, F16_MAX).unflatten(-1, (-1, group))
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    scale = ((hi - lo) * torch.tensor(1.0 / 15.0, dtype=x.dtype, device=x.device)).half()
    off = lo.half()
    wide = scale.to(x.dtype)
    inv = torch.where(wide > 0, wide.reciprocal(), torch.zeros_like(wide))
    codes = ((x - off.to(x.dtype)) * inv).round().clamp(0, 15)
    return codes.flatten(-2), scale.squeeze(-1), off.squeeze(-1)


def _values(codes, scale, off, group):
    return (codes.unflatten(-1, (-1, group)) * scale.to(codes.dtype)[..., None] + off.to(codes.dtype)[..., None]).flatten(-2)


def _rotate(x, cos, sin, inter):
    """The first 2 * cos.shape[-1] dims of x rotated: pairs of halves, or neighbours."""
    rot = 2 * cos.shape[-1]
    r, rest = x[..., :rot], x[..., rot:]
    a, b = (r[..., 0::2], r[..., 1::2]) if inter else (r[..., : rot // 2], r[..., rot // 2:])
    y, z = a * cos - b * sin, b * cos + a * sin
    r = torch.stack((y, z), -1).flatten(-2) if inter else torch.cat((y, z), -1)
    return torch.cat((r, rest), -1)


def _plain_cache(c, s):
    """Codes two a byte, scales and offsets: [page, token, keys and values, head, ..]."""
    shape = (s["n_pages"], c["page"], 2, c["kv_heads"])
    s["codes"] = torch.zeros(*shape, c["D"] // 2, dtype=torch.uint8, device="cuda")
    s["meta"] = torch.zeros(*shape, c["D"] // c["G"], 2, dtype=torch.float16, device="cuda")


def _plain_slots(c, s, start, kv, rows):
    """Page, place in it, and position of every new row."""
    seq = torch.repeat_interleave(torch.arange(c["seqs"], device="cuda"), (start[1:] - start[:-1]).long(), output_size=rows)
    pos = torch.arange(rows, device="cuda") - start[1:].long()[seq] + kv.long()[seq]
    return s["table"].long()[seq, pos // c["page"]], pos % c["page"], pos


def _plain_write(c, s, k, v, page, at):
    codes, scale, off = _quantise(torch.stack((k, v), 1), c["G"])
    codes = codes.to(torch.uint8)
    s["codes"][page, at] = codes[..., 0::2] | (codes[..., 1::2] << 4)
    s["meta"][page, at] = torch.stack((scale, off), -1)


def _plain_read(c, codes, meta):
    codes = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float()
    return _values(codes, meta[..., 0], meta[..., 1], c["G"])


def _plain_append(s):
    c, dt = s["c"], s["q"].dtype
    page, at, pos = _plain_slots(c, s, s["q_start"], s["kv_len"], s["rows"])
    cos, sin = s["cos"][pos][:, None], s["sin"][pos][:, None]
    q = _rotate(s["q"].float(), cos, sin, c["inter"])
    k = _rotate(s["k"].float(), cos, sin, c["inter"])
    _plain_write(c, s, k, s["v"].float(), page, at)
    kv = _plain_read(c, s["codes"][page, at], s["meta"][page, at]).to(dt)
    return q.to(dt), kv[:, 0].contiguous(), kv[:, 1].contiguous()


def _plain_attn(s):
    """Every sequence padded to the longest: keys and values [sequence, head, token, D], queries [sequence, head, row, D]."""
    c, q = s["c"], s["q"].float()
    n, hk, d, rep = c["seqs"], c["kv_heads"], c["D"], c["heads"] // c["kv_heads"]
    t = s["table"].long()
    kv = _plain_read(c, s["codes"][t], s["meta"][t])  # [n, pages, page, 2, head, D]
    kv = kv.flatten(1, 2).permute(2, 0, 3, 1, 4)
    most, new = max(s["new"]), (s["q_start"][1:] - s["q_start"][:-1]).long()
    i = torch.arange(most, device="cuda")
    row = (s["q_start"][:-1].long()[:, None] + i).clamp(max=max(0, s["rows"] - 1))
    qs = q[row].view(n, most, hk, rep, d).transpose(1, 2).reshape(n, hk, most * rep, d)
    sc = torch.matmul(qs, kv[0].contiguous().transpose(-1, -2)) * (1.0 / math.sqrt(d))
    last = (s["kv_len"].long()[:, None] - new[:, None] + i)[:, None, :, None]  # the newest token that row i sees
    pos = torch.arange(kv.shape[3], device="cuda")
    see = pos <= last
    if c["window"]:
        see = see & (pos > last - c["window"])
    see = see.expand(n, 1, most, pos.numel()).repeat_interleave(rep, 2)
    sc = sc.masked_fill_(~see, -math.inf)
    top = sc.amax(-1, keepdim=True).clamp(min=-3e38)
    p = sc.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, kv[1].contiguous()) / total.clamp(min=1e-38)
    lse = torch.where(total > 0, top + total.log(), torch.full_like(total, -math.inf))
    o = o.view(n, hk, most, rep, d).transpose(1, 2).reshape(n, most, c["heads"], d)
    seq = torch.repeat_interleave(torch.arange(n, device="cuda"), new, output_size=s["rows"])
    at = torch.arange(s["rows"], device="cuda") - s["q_start"].long()[seq]
    out = o[seq, at].to(s["q"].dtype)
    if not c["lse"]:
        return out
    return out, lse.view(n, hk, most, rep).transpose(1, 2).reshape(n, most, c["heads"])[seq, at]


def _plain_w4(s):
    x, codes, c = s["x"].float(), s["codes"], s["c"]
    w = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float().unflatten(-1, (-1, c["G"]))
    w = w - (s["zeros"].float()[..., None] if c["zeros"] else 8.0)
    w = (w * s["scales"].float()[..., None]).flatten(-2)
    y = x @ w.T
    if c["bias"]:
        y = y + s["bias"].float()
    return y.to(s["x"].dtype)


def run(s):
    c = s["c"]
    if not own:
        return {"w4": _plain_w4, "append": _plain_append, "attn": _plain_attn}[c["op"]](s)
    if c["op"] == "w4":
        return s["w"].matmul(s["x"], bias=s["bias"])
    cache, batch = s["cache"], s["batch"]
    if c["op"] == "append":
        q = cache.append(batch, s["k"], s["v"], cos=s["cos"], sin=s["sin"], q=s["q"], interleaved=c["inter"])
        return (q, *cache.read(batch, s["q"].dtype))
    return cache.attention(batch, s["q"], window=c["window"], lse=c["lse"])


# ------------------------------------------------------------- in 64 bits

def _exact_cache(x, group):
    """What a row of values stands for once it is cached: the definition, value by value, in 64 bits."""
    x = x.double().clamp(-F16_MAX, F16_MAX)
    y = x.reshape(*x.shape[:-1], x.shape[-1] // group, group)
    low = y.min(dim=-1, keepdim=True).values
    step = ((y.max(dim=-1, keepdim=True).values - low) / 15).to(torch.float16).double()
    low = low.to(torch.float16).double()
    code = torch.round((y - low) / torch.where(step > 0, step, torch.ones_like(step))).clamp(0, 15)
    return (low + step * code).reshape(x.shape)


def _exact_turn(x, pos, c):
    """x [rows, heads, D] turned as complex numbers by its positions' angles (the 32-bit tables that the call is given)."""
    cos, sin = _angles(c, _pages(c) * c["page"])
    turn = torch.complex(cos.double(), sin.double())[pos][:, None]
    half = c["rot"] // 2
    r = x.double()[..., : c["rot"]]
    pairs = r.reshape(*r.shape[:-1], half, 2) if c["inter"] else torch.stack((r[..., :half], r[..., half:]), -1)
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    out = x.double().clone()
    out[..., : c["rot"]] = z.reshape(r.shape) if c["inter"] else torch.cat((z[..., 0], z[..., 1]), -1)
    return out


def exact(c, seed):
    if c["op"] == "w4":
        x, codes, scales, zeros, bias = _w4_inputs(c, seed)
        n, k, g = c["N"], c["K"], c["G"]
        y = torch.empty(c["M"], n, dtype=torch.float64, device="cuda")
        for lo in range(0, n, 4096):  # some outputs at a time
            part = codes[lo:lo + 4096].to(torch.int64)
            w = torch.zeros(part.shape[0], k, dtype=torch.float64, device="cuda")
            w[:, 0::2], w[:, 1::2] = (part % 16).double(), (part // 16).double()
            at = torch.arange(k, device="cuda") // g
            w -= 8.0 if zeros is None else zeros[lo:lo + 4096].double()[:, at]
            w *= scales[lo:lo + 4096].double()[:, at]
            y[:, lo:lo + 4096] = torch.mm(x.double(), w.t())
        return y if bias is None else y + bias.double()
    s = _cache_inputs(c, seed)
    if c["op"] == "append":
        k = (_normal(s["g"], s["rows"], c["kv_heads"], c["D"]) * s["wide"]).to(DT[c["dtype"]])
        v = _normal(s["g"], s["rows"], c["kv_heads"], c["D"]).to(DT[c["dtype"]])
        pos = torch.cat([torch.arange(a - n, a) for a, n in zip(s["kv"], s["new"])]).cuda()
        return (_exact_turn(s["q"], pos, c), _exact_cache(_exact_turn(k, pos, c), c["G"]), _exact_cache(v, c["G"]))
    if sum(s["kv"]) * c["kv_heads"] * c["D"] > 1 << 29:
        return None  # too long in 64 bits
    held = [[] for _ in s["kv"]]

    def put(start, kv, k, v, rows, most):
        at = start.tolist()
        for i in range(c["seqs"]):
            held[i].append((k[at[i]:at[i + 1]], v[at[i]:at[i + 1]]))

    _fill(c, s, put)
    rep, d = c["heads"] // c["kv_heads"], c["D"]
    outs, sums, first = [], [], 0
    for i, (kv, n) in enumerate(zip(s["kv"], s["new"])):
        o = torch.zeros(n, c["heads"], d, dtype=torch.float64, device="cuda")
        ls = torch.full((n, c["heads"]), -math.inf, dtype=torch.float64, device="cuda")
        if kv:
            key = _exact_cache(torch.cat([a for a, _ in held[i]]), c["G"])
            val = _exact_cache(torch.cat([b for _, b in held[i]]), c["G"])
            where = torch.arange(kv, device="cuda")
            newest = torch.arange(kv - n, kv, device="cuda")[:, None]
            hidden = (where > newest) | ((where <= newest - c["window"]) if c["window"] else (where < 0))
            blind = hidden.all(1)
            for h in range(c["heads"]):
                w = s["q"][first:first + n, h].double() @ key[:, h // rep].t() / math.sqrt(d)
                w = w.masked_fill(hidden, -math.inf)
                ls[:, h] = torch.logsumexp(w, 1)
                o[:, h] = torch.softmax(w, 1) @ val[:, h // rep]
            o[blind] = 0.0
        outs.append(o)
        sums.append(ls)
        first += n
    out = torch.cat(outs)
    return (out, torch.cat(sums)) if c["lse"] else out
