"""The operators of a 4-bit variant's step (products with 4-bit weights, the
append to the paged 4-bit cache, attention over it) against plain
implementations in 64 bits, at the sizes, lengths, masks and layouts where they
can go wrong.

Tolerances, derived before the first run, with u the rounding unit of the
result's type (2^-8 bfloat16, 2^-11 binary16):
* products: the sums are fp32 over K terms of size up to 31 |x s|, so an
  element's error is at most u |y| (the result's rounding) plus
  64 K 2^-24 sum |x| s, and in practice far below it.
* append: codes are equal to the definition's in fp32, step for step, so the
  values read back are equal bit for bit; turned queries are two products and a
  sum in fp32, rounded once: u |y| plus 3 2^-24 (|a| + |b|).
* attention: the weights, alone and times the scales, are rounded to 16 bits
  (2^-11 of each in binary16; 2^-9, bfloat16's, against code distances of at most
  7.5 scales is asked for), so an element is within u |o| plus 2^-9 sum_t p_t 7.5
  scale_t, plus fp32 terms that 1e-4 of the largest value covers; lse: 1e-4 (fp32
  products over D <= 256).
"""
import math
import random

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


@pytest.fixture(scope="module")
def serve():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2609_02109_amd import serve as m
    return m


def _gen(seed):
    return torch.Generator().manual_seed(seed)


# --------------------------------------------------------------------- w4

def _weights(n, k, g, dt, zeros, seed):
    gen = _gen(seed)
    codes = torch.randint(0, 256, (n, k // 2), generator=gen, dtype=torch.uint8)
    scales = ((0.5 + torch.rand(n, k // g, generator=gen)) * 0.01).to(dt)
    z = torch.randint(0, 16, (n, k // g), generator=gen, dtype=torch.uint8) if zeros else None
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(1).double()
    at = torch.arange(k) // g
    w = (c - (z.double()[:, at] if zeros else 8.0)) * scales.double()[:, at]
    return codes, scales, z, w


def _check_w4(y, x, w, scales, g, bias, dt):
    want = x.double() @ w.T + (0 if bias is None else bias.double())
    at = torch.arange(w.shape[1]) // g
    mass = x.double().abs() @ scales.double().abs()[:, at].T
    tol = UNIT[dt] * want.abs() + 64 * w.shape[1] * 2.0 ** -24 * mass + 1e-7
    err = (y.cpu().double() - want).abs()
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("m,n,k,g", [
    (1, 16, 32, 32), (1, 1, 128, 128), (2, 17, 64, 64), (3, 515, 160, 32), (16, 64, 256, 64), (17, 250, 384, 128),
    (32, 1000, 1120, 32), (33, 100, 576, 64), (64, 4096, 512, 128), (65, 48, 2048, 64), (200, 33, 96, 32), (5, 31, 16384, 128),
    (16, 20000, 128, 128)])
def test_w4_product(serve, dt, m, n, k, g):
    codes, scales, z, w = _weights(n, k, g, DT[dt], (m + n) % 2 == 0, m + n + k)
    gen = _gen(1)
    x = torch.randn(m, k, generator=gen).to(DT[dt])
    bias = torch.randn(n, generator=gen).to(DT[dt]) if m % 3 else None
    W = serve.W4Weight(codes.cuda(), scales.cuda(), z if z is None else z.cuda())
    y = W.matmul(x.cuda(), bias=bias if bias is None else bias.cuda())
    assert y.dtype is DT[dt] and tuple(y.shape) == (m, n)
    _check_w4(y, x, w, scales, g, bias, dt)


@pytest.mark.parametrize("m", [1, 4, 20, 40])
def test_w4_strides_and_shapes(serve, m):
    n, k, g = 203, 416, 32
    codes, scales, z, w = _weights(n, k, g, torch.bfloat16, True, 3)
    W = serve.W4Weight(codes.cuda(), scales.cuda(), z.cuda())
    gen = _gen(2)
    # rows that are 2-byte aligned only, NaN between them; a result inside a larger one
    wide = torch.full((m, k + 7), float("nan")).to(torch.bfloat16)
    wide[:, 3:3 + k] = torch.randn(m, k, generator=gen).to(torch.bfloat16)
    big = torch.full((m, n + 5), 7.0, dtype=torch.bfloat16, device="cuda")
    out = W.matmul(wide.cuda()[:, 3:3 + k], out=big[:, 1:1 + n])
    assert out.data_ptr() == big[:, 1:].data_ptr()
    _check_w4(big[:, 1:1 + n], wide[:, 3:3 + k], w, scales, g, None, "bf16")
    assert (big[:, 0] == 7).all() and (big[:, 1 + n:] == 7).all()
    x3 = torch.randn(2, m, k, generator=gen).to(torch.bfloat16)
    y3 = W.matmul(x3.cuda())
    assert tuple(y3.shape) == (2, m, n)
    _check_w4(y3.reshape(2 * m, n), x3.reshape(2 * m, k), w, scales, g, None, "bf16")
    xt = torch.randn(k, m, generator=gen).to(torch.bfloat16)
    _check_w4(W.matmul(xt.cuda().T), xt.T, w, scales, g, None, "bf16")
    assert tuple(W.matmul(torch.empty(0, k, dtype=torch.bfloat16, device="cuda")).shape) == (0, n)
    assert tuple(W.matmul(x3[0, 0].cuda()).shape) == (n,)


def test_w4_rows_do_not_mix(serve):
    # a NaN or an infinity in one row stays in that row
    codes, scales, z, w = _weights(64, 256, 64, torch.float16, True, 4)
    W = serve.W4Weight(codes.cuda(), scales.cuda(), z.cuda())
    x = torch.randn(20, 256, generator=_gen(5)).half()
    clean = W.matmul(x.cuda())
    x[3, 17], x[18, 0] = float("nan"), float("inf")
    y = W.matmul(x.cuda())
    rest = [i for i in range(20) if i not in (3, 18)]
    assert torch.isnan(y[3]).all() and not torch.isfinite(y[18]).any()
    assert torch.equal(y[rest], clean[rest])


def test_w4_refusals(serve):
    from paper_2609_02109_amd import mf
    codes, scales, z, _ = _weights(32, 128, 32, torch.bfloat16, True, 6)
    c, s, z = codes.cuda(), scales.cuda(), z.cuda()
    W = serve.W4Weight(c, s, z)
    for bad in (lambda: serve.W4Weight(codes, scales), lambda: serve.W4Weight(c, s.float()), lambda: serve.W4Weight(c, s[:16]),
                lambda: serve.W4Weight(c, s, z[:, :2]), lambda: serve.W4Weight(c.int(), s), lambda: W.matmul(torch.empty(1, 64, dtype=torch.bfloat16, device="cuda")),
                lambda: W.matmul(torch.empty(1, 128, dtype=torch.float16, device="cuda")), lambda: W.matmul(torch.empty(1, 128, dtype=torch.bfloat16)),
                lambda: W.matmul(torch.empty(1, 128, dtype=torch.bfloat16, device="cuda"), bias=torch.empty(31, dtype=torch.bfloat16, device="cuda")),
                lambda: W.matmul(torch.empty(1, 128, dtype=torch.bfloat16, device="cuda"), out=torch.empty(1, 31, dtype=torch.bfloat16, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(mf.MfError) as e:
        serve.W4Weight(c, s[:, :1].contiguous().repeat(1, 8))   # groups of 16
    assert e.value.status == mf.MF_EUNSUPPORTED


# ------------------------------------------------------------------ cache

class Case:
    """A cache, a batch and their plain copies: every sequence's held values
    [kv, heads, D] in 64 bits, from quantising in fp32 step by step."""

    def __init__(self, serve, kv, new, heads=2, D=64, G=32, page=16, dt="bf16", seed=0, spare=3):
        self.serve, self.kv, self.new, self.heads, self.D, self.G, self.page, self.dt = serve, kv, new, heads, D, G, page, dt
        gen = _gen(seed)
        n = len(kv)
        cols = max(1, -(-max(kv + [1]) // page))
        self.n_pages = n * cols + spare
        perm = torch.randperm(self.n_pages, generator=gen).to(torch.int32)
        self.table = perm[: n * cols].view(n, cols)
        self.cache = serve.KV4Cache(self.n_pages, page, heads, D, group=G)
        self.cache.pages.fill_(255)   # what is not written: NaN scales everywhere
        self.k = [torch.randn(a, heads, D, generator=gen).to(DT[dt]) for a in kv]
        self.v = [torch.randn(a, heads, D, generator=gen).to(DT[dt]) for a in kv]
        self.gen = gen

    def batch(self, new=None, kv=None, max_kv=None, table=None):
        new, kv = self.new if new is None else new, self.kv if kv is None else kv
        start = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
        return self.cache.batch(torch.from_numpy(start).cuda(), torch.tensor(kv, dtype=torch.int32).cuda(),
                                (self.table if table is None else table).cuda(), rows=int(start[-1]), max_new=max(new),
                                max_kv=max(kv) if max_kv is None else max_kv)

    def rows(self, per_seq, new, kv):
        """The newest `new` of the first `kv` tokens of every sequence, as a step's row tensor."""
        return torch.cat([t[max(0, b - a):b] if b >= a else torch.cat((t.new_zeros(a - b, *t.shape[1:]), t[:b]))
                          for t, a, b in zip(per_seq, new, kv)])

    def fill(self, steps=1, **rot):
        """Every token, in `steps` calls of ragged sizes."""
        done = [0] * len(self.kv)
        for i in range(steps):
            upto = [a * (i + 1) // steps for a in self.kv]
            new = [b - a for a, b in zip(done, upto)]
            if sum(new):
                self.cache.append(self.batch(new, upto, max_kv=max(self.kv)), self.rows(self.k, new, upto).cuda(),
                                  self.rows(self.v, new, upto).cuda(), **rot)
            done = upto

    def held(self, x):
        return held(x.float(), self.G)


def held(x, G):
    """What a row stands for in the cache, in fp32 step by step."""
    y = x.clamp(-65504, 65504).unflatten(-1, (-1, G))
    lo, hi = y.amin(-1, keepdim=True), y.amax(-1, keepdim=True)
    s = ((hi - lo) * torch.tensor(np.float32(1 / 15.0))).half().float()
    o = lo.half().float()
    inv = torch.where(s > 0, 1.0 / s, torch.zeros_like(s))
    c = ((y - o) * inv).round().clamp(0, 15)
    return (o + s * c).flatten(-2)


def turned(x, cos, sin, inter):
    """fp32 rows [.., heads, D] turned; cos, sin [.., rot / 2]."""
    cos, sin = cos[:, None], sin[:, None]
    rot = 2 * cos.shape[-1]
    r = x[..., :rot]
    a, b = (r[..., 0::2], r[..., 1::2]) if inter else (r[..., : rot // 2], r[..., rot // 2:])
    y, z = a * cos - b * sin, b * cos + a * sin
    r = torch.stack((y, z), -1).flatten(-2) if inter else torch.cat((y, z), -1)
    return torch.cat((r, x[..., rot:]), -1)


SHAPES = [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128), (256, 32), (256, 64), (256, 128)]


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("D,G", SHAPES)
def test_append_and_read(serve, D, G, dt):
    # pages of one block and of three, several calls that end inside blocks; every token reads back as the definition's
    for page, steps, seed in ((16, 1, 1), (48, 5, 2), (16, 13, 3)):
        c = Case(serve, [1, 77, 16, 33, 130], None, heads=3, D=D, G=G, page=page, dt=dt, seed=seed)
        c.fill(steps)
        b = c.batch(new=c.kv)
        for ty in (torch.float32, DT[dt]):
            k, v = c.cache.read(b, ty)
            assert torch.equal(k.cpu(), held(torch.cat(c.k).float(), G).to(ty))
            assert torch.equal(v.cpu(), held(torch.cat(c.v).float(), G).to(ty))


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D,rot", [(64, 64), (64, 16), (128, 128), (128, 48), (256, 256), (256, 64)])
def test_append_turns_keys_and_queries(serve, D, rot, inter):
    dt = "bf16" if rot % 32 else "f16"
    c = Case(serve, [5, 70, 21], [5, 9, 1], heads=2, D=D, G=64, page=32, dt=dt, seed=rot)
    cos, sin = serve.rope_table(80, rot)
    c.fill(3, cos=cos, sin=sin, interleaved=inter)
    b = c.batch()
    q = torch.randn(15, 6, D, generator=c.gen).to(DT[dt])
    qd = q.cuda()
    qr = c.cache.append(b, c.rows(c.k, c.new, c.kv).cuda(), c.rows(c.v, c.new, c.kv).cuda(), cos=cos, sin=sin, q=qd, interleaved=inter)
    pos = torch.cat([torch.arange(a) for a in c.kv])
    k, _ = c.cache.read(c.batch(new=c.kv))
    assert torch.equal(k.cpu(), held(turned(torch.cat(c.k).float(), cos.cpu()[pos], sin.cpu()[pos], inter), 64))
    new = torch.cat([torch.arange(a - n, a) for a, n in zip(c.kv, c.new)])
    want = turned(q.double(), cos.cpu().double()[new], sin.cpu().double()[new], inter)
    partner = turned(q.double().abs(), torch.ones(15, rot // 2), -torch.ones(15, rot // 2), inter).abs() + q.double().abs()
    assert ((qr.cpu().double() - want).abs() <= UNIT[dt] * want.abs() + 3 * 2.0 ** -24 * partner + 2.0 ** -24).all()
    # over its source
    c.cache.append(b, c.rows(c.k, c.new, c.kv).cuda(), c.rows(c.v, c.new, c.kv).cuda(), cos=cos, sin=sin, q=qd, q_out=qd, interleaved=inter)
    assert torch.equal(qd, qr)


def test_append_strides(serve):
    # k and v as slices of one projection with an odd row length, heads in another order
    c = Case(serve, [40, 19], [40, 19], heads=2, D=64, G=32, dt="f16", seed=9)
    rows = 59
    wide = torch.full((rows, 2 * 2 * 64 + 5), float("nan"), dtype=torch.float16)
    wide[:, 3:131] = torch.cat(c.k).flatten(1)
    wide[:, 131:259] = torch.cat(c.v).flatten(1)
    w = wide.cuda()
    k = w.as_strided((rows, 2, 64), (261, 64, 1), 3)
    v = w.as_strided((rows, 2, 64), (261, 64, 1), 131)
    c.cache.append(c.batch(), k, v)
    a, b = c.cache.read(c.batch())
    assert torch.equal(a.cpu(), held(torch.cat(c.k).float(), 32)) and torch.equal(b.cpu(), held(torch.cat(c.v).float(), 32))
    # [heads, rows, D]
    kt = torch.cat(c.k).transpose(0, 1).contiguous().cuda().transpose(0, 1)
    vt = torch.cat(c.v).transpose(0, 1).contiguous().cuda().transpose(0, 1)
    c.cache.pages.fill_(255)
    c.cache.append(c.batch(), kt, vt)
    a, b = c.cache.read(c.batch())
    assert torch.equal(a.cpu(), held(torch.cat(c.k).float(), 32)) and torch.equal(b.cpu(), held(torch.cat(c.v).float(), 32))


def test_append_of_odd_values(serve):
    # constant groups, subnormal spreads, the largest values, infinities, NaN
    c = Case(serve, [8], [8], heads=1, D=64, G=32, dt="bf16", seed=10)
    x = c.k[0].float()
    x[0] = 1.5
    x[1] = 0.0
    x[2] = 1e-9 * torch.arange(64)
    x[3, 0, 5] = 3e38
    x[4, 0, 40] = float("-inf")
    x[5, 0, 0], x[5, 0, 1] = float("inf"), float("-inf")
    x[6, 0, 33] = float("nan")
    x = x.to(torch.bfloat16)
    c.cache.append(c.batch(), x.cuda(), x.flip(0).cuda())
    k, v = c.cache.read(c.batch())
    want = held(x.float(), 32)
    for got, w in ((k.cpu(), want), (v.cpu(), want.flip(0))):
        nan = torch.isnan(w)
        assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], w[~nan])
    assert torch.isnan(k[6, 0, 32:]).all() and torch.isfinite(k[6, 0, :32]).all() and torch.isfinite(k[[0, 1, 2, 3, 4, 5, 7]]).all()


def test_append_leaves_the_rest_alone(serve):
    # other pages, other tokens of the same block, and what lies outside of the cache's positions or pages
    c = Case(serve, [30, 45], [3, 5], heads=2, D=128, G=64, page=16, dt="bf16", seed=11, spare=5)
    c.fill(2)
    before = c.cache.read(c.batch(new=c.kv))
    b = c.batch()
    k, v = torch.randn(8, 2, 128).bfloat16().cuda(), torch.randn(8, 2, 128).bfloat16().cuda()
    c.cache.append(b, k, v)
    after = c.cache.read(c.batch(new=c.kv))
    new = torch.zeros(75, dtype=torch.bool)
    new[27:30] = new[70:75] = True
    for x, y, z in zip(before, after, (k, v)):
        assert torch.equal(x.cpu()[~new], y.cpu()[~new]) and torch.equal(y.cpu()[new], held(z.cpu().float(), 64))
    raw = c.cache.pages.clone()
    # more new tokens than tokens: those at negative positions are left out
    c.cache.append(c.batch(new=[3, 5], kv=[2, 0], max_kv=45), k, v)
    two = c.cache.read(c.batch(new=[2, 0], kv=[2, 0], max_kv=45))
    assert torch.equal(two[0].cpu(), held(k.cpu().float()[1:3], 64))
    # a page number that is none, and a max_kv below the tokens: nothing is written, zeros are read
    c.cache.pages.copy_(raw)
    bad = c.table.clone()
    bad[0, 1], bad[1, 2] = c.n_pages, -1
    c.cache.append(c.batch(table=bad), k, v)
    c.cache.append(c.batch(max_kv=20), k, v)
    torch.cuda.synchronize()
    assert torch.equal(c.cache.pages, raw)
    assert all((t == 0).all() for t in c.cache.read(c.batch(table=bad)))
    # nothing new at all
    c.cache.append(c.batch(new=[0, 0]), k[:0], v[:0])
    assert torch.equal(c.cache.pages, raw)


# -------------------------------------------------------------- attention

def plain_attention(q, k, v, heads_per, new, window, scale):
    """One sequence in 64 bits: (out, lse, sum of p * 7.5 steps) of its `new` rows over k, v [kv, kv heads, D]."""
    kv, D = k.shape[0], q.shape[-1]
    out = torch.zeros(q.shape, dtype=torch.float64)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64)
    probs = torch.zeros(q.shape[0], q.shape[1], kv, dtype=torch.float64)
    j = torch.arange(kv)
    for i in range(new):
        p = kv - new + i
        see = (j <= p) & ((j > p - window) if window else (j >= 0))
        if not see.any():
            continue
        for h in range(q.shape[1]):
            s = (k[see, h // heads_per].double() @ q[i, h].double()) * scale
            lse[i, h] = torch.logsumexp(s, 0)
            w = torch.softmax(s, 0)
            out[i, h] = w @ v[see, h // heads_per].double()
            probs[i, h, see] = w
    return out, lse, probs


def _steps(v, G):
    """Every value's step in the cache [.., D]."""
    y = v.float().unflatten(-1, (-1, G))
    s = ((y.amax(-1, keepdim=True) - y.amin(-1, keepdim=True)) / 15).half().double()
    return s.expand(*y.shape).flatten(-2)


def check_attention(c, per, window=0, scale=None, lse=True, out=None, q=None, batch=None, new=None, kv=None, stream=None):
    new, kv = c.new if new is None else new, c.kv if kv is None else kv
    heads = per * c.heads
    if q is None:
        q = (1.5 * torch.randn(sum(new), heads, c.D, generator=c.gen)).to(DT[c.dt])
    b = c.batch(new=new, kv=kv) if batch is None else batch
    got, ls = c.cache.attention(b, q.cuda(), scale=scale, window=window, lse=True, out=out, stream=stream)
    torch.cuda.synchronize()
    got, ls = got.cpu().double(), ls.cpu().double()
    at = 0
    for i, n in enumerate(new):
        hk, hv = c.held(c.k[i][: kv[i]]), c.held(c.v[i][: kv[i]])
        o, l, p = plain_attention(q[at:at + n], hk, hv, per, n, window, 1 / math.sqrt(c.D) if scale is None else scale)
        if kv[i]:
            st = _steps(c.v[i][: kv[i]], c.G)
            room = torch.stack([p[:, h] @ (7.5 * st[:, h // per]) for h in range(heads)], 1)
            top = float(hv.abs().max())
        else:
            room, top = torch.zeros_like(o), 0.0
        tol = UNIT[c.dt] * o.abs() + 2.0 ** -9 * room + 1e-4 * top
        err = (got[at:at + n] - o).abs()
        assert (err <= tol).all(), (i, n, float((err / tol.clamp(min=1e-30)).max()))
        seen = torch.isfinite(l)
        assert torch.equal(torch.isfinite(ls[at:at + n]), seen)
        assert (got[at:at + n][~seen] == 0).all() and (ls[at:at + n][~seen] == -math.inf).all()
        assert ((ls[at:at + n] - l)[seen].abs() <= 1e-4).all()
        at += n
    return got


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("D,G", SHAPES)
def test_attention_one_token(serve, D, G, dt):
    c = Case(serve, [1, 15, 16, 17, 0, 31, 33, 129, 500], [1] * 9, heads=2, D=D, G=G, page=16, dt=dt, seed=D + G)
    c.fill(2)
    for per in (1, 4, 16):
        check_attention(c, per)


@pytest.mark.parametrize("per,new", [(1, 2), (1, 17), (3, 5), (5, 7), (8, 33), (4, 70), (32, 1), (24, 2), (2, 130)])
def test_attention_several_tokens(serve, per, new):
    D, G = ((64, 32), (128, 64), (256, 128))[new % 3]
    c = Case(serve, [new, new + 40, 200, max(0, new - 3)], [new, new, new, new], heads=2, D=D, G=G, page=32, dt="bf16", seed=per * new)
    c.fill(1)
    check_attention(c, per)


def test_attention_ragged_new(serve):
    # some sequences bring nothing, one token, a prompt
    c = Case(serve, [60, 5, 90, 33, 64], [0, 1, 40, 33, 3], heads=2, D=128, G=32, page=16, dt="f16", seed=5)
    c.fill(2)
    check_attention(c, 2)


@pytest.mark.parametrize("window", [1, 15, 16, 33, 100, 5000])
def test_attention_window(serve, window):
    c = Case(serve, [300, 20, 131], [1, 1, 1], heads=1, D=64, G=64, page=48, dt="bf16", seed=window)
    c.fill(1)
    check_attention(c, 3, window=window)
    c2 = Case(serve, [300, 41, 130], [64, 41, 50], heads=1, D=64, G=32, page=16, dt="bf16", seed=window + 1)
    c2.fill(1)
    check_attention(c2, 3, window=window)


def test_attention_split_over_tokens(serve):
    # contexts long enough to be taken apart, of very different lengths, and the join of parts that hold nothing
    c = Case(serve, [9000, 3, 4097, 0], [1, 1, 1, 1], heads=1, D=128, G=64, page=64, dt="bf16", seed=6)
    c.fill(1)
    b = c.batch()
    check_attention(c, 4, batch=b)
    # sharp softmax: the largest product far into one part
    c.k[0][7777] = (c.k[0][7777].float() * 6).to(torch.bfloat16)
    c.fill(1)
    q = torch.randn(4, 4, 128, generator=c.gen)
    q[0] = c.k[0][7777, 0].float() / 6
    check_attention(c, 4, q=q.to(torch.bfloat16))
    # the same call again gives the same bits
    qd = q.to(torch.bfloat16).cuda()
    assert torch.equal(c.cache.attention(b, qd), c.cache.attention(b, qd))
    c2 = Case(serve, [5000], [100], heads=1, D=64, G=32, page=16, dt="f16", seed=7)
    c2.fill(1)
    check_attention(c2, 2)
    check_attention(c2, 2, window=700)


def test_attention_of_what_lies_beyond(serve):
    # tokens that a row must not see hold NaN: later tokens, a window's earlier ones, the rest of the last page, missing pages
    for window in (0, 24):
        c = Case(serve, [90], [20], heads=1, D=64, G=32, page=16, dt="bf16", seed=8)
        c.fill(1)
        clean = c.cache.attention(c.batch(new=[20], kv=[60]), torch.ones(20, 2, 64).bfloat16().cuda(), window=window)
        nan = torch.full((1, 1, 64), float("nan")).bfloat16().cuda()
        for pos in list(range(60, 90)) + (list(range(0, 17)) if window else []):
            c.cache.append(c.batch(new=[1], kv=[pos + 1], max_kv=90), nan, nan)
        got = c.cache.attention(c.batch(new=[20], kv=[60]), torch.ones(20, 2, 64).bfloat16().cuda(), window=window)
        assert torch.equal(got, clean)
        # a NaN that is seen shows, in the rows that see it only
        c.cache.append(c.batch(new=[1], kv=[51], max_kv=90), nan, nan)
        got = c.cache.attention(c.batch(new=[20], kv=[60]), torch.ones(20, 2, 64).bfloat16().cuda(), window=window)
        assert torch.equal(got[:10], clean[:10]) and torch.isnan(got[10:]).all()
    # a page that is none of the cache's is not seen: as without its tokens
    c = Case(serve, [64], [1], heads=1, D=64, G=32, page=16, dt="bf16", seed=9)
    c.fill(1)
    bad = c.table.clone()
    bad[0, 1] = -7
    q = torch.randn(1, 2, 64).bfloat16()
    got = c.cache.attention(c.batch(table=bad), q.cuda()).cpu().double()
    keep = torch.cat((torch.arange(16), torch.arange(32, 64)))
    o, _, _ = plain_attention(q, c.held(c.k[0])[keep], c.held(c.v[0])[keep], 2, 1, 0, 1 / 8)
    assert (got - o).abs().max() < 2e-2
    # all pages missing: an empty row
    out, ls = c.cache.attention(c.batch(table=torch.full_like(bad, 10 ** 6)), q.cuda(), lse=True)
    assert (out == 0).all() and (ls == -math.inf).all()


def test_attention_strides_scale_and_streams(serve):
    c = Case(serve, [50, 70], [3, 2], heads=2, D=64, G=32, page=16, dt="f16", seed=12)
    c.fill(1)
    q = torch.randn(5, 6, 64, generator=c.gen).half()
    base = check_attention(c, 3, q=q, scale=0.3)
    # queries as a 2-byte aligned slice, results into a slice
    wide = torch.full((5, 6 * 64 + 3), float("nan"), dtype=torch.float16, device="cuda")
    qs = wide.as_strided((5, 6, 64), (387, 64, 1), 1)
    qs.copy_(q)
    big = torch.full((5, 6, 67), 9.0, dtype=torch.float16, device="cuda")
    out = c.cache.attention(c.batch(), qs, scale=0.3, out=big[:, :, 1:65])
    assert torch.equal(out.cpu().double(), base) and (big[:, :, 0] == 9).all() and (big[:, :, 65:] == 9).all()
    # another stream than the tensors' own
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b, qd = c.batch(), q.cuda()
    torch.cuda.synchronize()
    got = c.cache.attention(b, qd, scale=0.3, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got.cpu().double(), base)


def test_attention_over_a_cache_past_32_bits(serve):
    # pages beyond 4 GiB: 60,000 of 73,728 bytes; a few sequences in the last ones
    c = Case(serve, [40, 100], [1, 2], heads=8, D=128, G=64, page=64, dt="bf16", seed=13)
    big = serve.KV4Cache(60_000, 64, 8, 128, group=64)
    assert big.pages.numel() > 2 ** 32
    c.cache, c.n_pages = big, 60_000
    c.table = (59_999 - c.table).to(torch.int32)
    c.fill(2)
    k, v = c.cache.read(c.batch(new=c.kv))
    assert torch.equal(k.cpu(), held(torch.cat(c.k).float(), 64)) and torch.equal(v.cpu(), held(torch.cat(c.v).float(), 64))
    check_attention(c, 2)


def test_a_step_in_a_graph(serve):
    """Product, append and attention captured once and replayed with the lengths moved on in place."""
    c = Case(serve, [20, 37], [1, 1], heads=2, D=64, G=32, page=16, dt="bf16", seed=14)
    c.fill(1)
    codes, scales, z, w = _weights(256, 256, 64, torch.bfloat16, True, 15)
    W = serve.W4Weight(codes.cuda(), scales.cuda(), z.cuda())
    cos, sin = serve.rope_table(64, 64)
    x = torch.randn(2, 256, generator=c.gen).bfloat16().cuda()
    b = c.batch(kv=[20, 37], max_kv=40)

    def step():
        q = W.matmul(x).view(2, 4, 64)
        qr = c.cache.append(b, q[:, :2], q[:, 2:], cos=cos, sin=sin, q=q)
        return c.cache.attention(b, qr)

    want = []
    lens = [torch.tensor([20 + i, 37 + i], dtype=torch.int32).cuda() for i in range(3)]
    for i in range(3):
        b.tensors[1].copy_(lens[i])
        want.append(step().clone())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for i in range(3):
        b.tensors[1].copy_(lens[i])
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i])
        (x * 2).sum().item()


def test_refusals(serve):
    from paper_2609_02109_amd import mf
    for bad, status in ((dict(page_size=24), mf.MF_EUNSUPPORTED), (dict(page_size=2048), mf.MF_EUNSUPPORTED), (dict(head_dim=96), mf.MF_EUNSUPPORTED),
                        (dict(group=16), mf.MF_EUNSUPPORTED), (dict(group=128, head_dim=64), mf.MF_EUNSUPPORTED), (dict(n_pages=0), mf.MF_EINVAL),
                        (dict(n_kv_heads=0), mf.MF_EINVAL)):
        with pytest.raises(mf.MfError) as e:
            serve.KV4Cache(**{**dict(n_pages=4, page_size=16, n_kv_heads=2, head_dim=64, group=32), **bad})
        assert e.value.status == status
    c = Case(serve, [20], [2], heads=2, D=64, G=32, dt="bf16", seed=16)
    b = c.batch()
    k = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    cos, sin = serve.rope_table(64, 64)
    for bad in (lambda: c.cache.append(b, k.float(), k.float()), lambda: c.cache.append(b, k, k[:1]), lambda: c.cache.append(b, k, k.half()),
                lambda: c.cache.append(b, k, k, cos=cos), lambda: c.cache.append(b, k, k, q=k), lambda: c.cache.append(b, k, k, cos=cos.cpu(), sin=sin.cpu()),
                lambda: c.cache.attention(b, k[:1]), lambda: c.cache.attention(b, k.float()), lambda: c.cache.attention(b, k, out=k[:1]),
                lambda: c.cache.batch(torch.zeros(2, dtype=torch.int64, device="cuda"), b.tensors[1], b.tensors[2], 2, 2, 20),
                lambda: c.cache.read(b, torch.int32)):
        with pytest.raises(ValueError):
            bad()
    short = serve.rope_table(19, 64)
    odd = serve.rope_table(64, 24)
    for bad, status in ((lambda: c.cache.append(b, k, k, cos=short[0], sin=short[1]), mf.MF_EINVAL),
                        (lambda: c.cache.append(b, k, k, cos=odd[0], sin=odd[1]), mf.MF_EUNSUPPORTED),
                        (lambda: c.cache.attention(c.batch(max_kv=33), k), mf.MF_EINVAL),
                        (lambda: c.cache.attention(b, k, scale=0.0), mf.MF_EINVAL), (lambda: c.cache.attention(b, k, scale=float("nan")), mf.MF_EINVAL),
                        (lambda: c.cache.attention(b, k, window=-1), mf.MF_EINVAL),
                        (lambda: c.cache.attention(b, torch.zeros(2, 3, 64, dtype=torch.bfloat16, device="cuda")), mf.MF_EINVAL),
                        (lambda: c.cache.append(b, k, k, cos=cos, sin=sin, q=k, q_out=k[:1].expand(2, 2, 64)), mf.MF_EINVAL)):
        with pytest.raises(mf.MfError) as e:
            bad()
        assert e.value.status == status


def test_random_steps(serve):
    rng = random.Random(2)
    for i in range(12):
        D, G = rng.choice(SHAPES)
        n, per, heads = rng.randint(1, 6), rng.choice([1, 2, 3, 5, 8]), rng.choice([1, 2, 3])
        kv = [rng.choice([0, 1, rng.randint(1, 60), rng.randint(1, 400)]) for _ in range(n)]
        new = [rng.choice([0, 1, rng.randint(0, 20)]) for _ in range(n)]
        if not sum(new):
            new[0] = 1
        c = Case(serve, kv, new, heads=heads, D=D, G=G, page=16 * rng.randint(1, 5), dt=rng.choice(["bf16", "f16"]), seed=100 + i)
        print(i, kv, new, heads, per, D, G, c.page, c.dt, flush=True)
        c.fill(rng.randint(1, 4))
        check_attention(c, per, window=rng.choice([0, 0, rng.randint(1, 80)]))


@pytest.mark.parametrize("kv", [200, 3000])
def test_attention_of_more_rows_than_the_batch_says(serve, kv):
    """A device array that gives a sequence more new tokens than max_new: its rows up to there, nothing past them."""
    c = Case(serve, [kv, 40], [3, 1], heads=1, D=64, G=32, page=16, dt="bf16", seed=17)
    c.fill(2)
    q = torch.randn(4, 1, 64, generator=c.gen).bfloat16()
    want = c.cache.attention(c.batch(), q.cuda())
    b = c.batch()
    b.raw.max_new = 1
    out = torch.full((4, 1, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    c.cache.attention(b, q.cuda(), out=out)
    assert (out[1:3] == 7).all()
    tol = 2 * UNIT["bf16"] * want.float().abs() + 2.0 ** -8 * float(want.float().abs().max())
    for i in (0, 3):   # other shares of the tokens: rounded elsewhere
        assert ((out[i].float() - want[i].float()).abs() <= tol[i]).all()


def test_a_graph_keeps_its_workspace(serve):
    """Attention in parts, captured, replayed after larger calls have taken other workspaces."""
    c = Case(serve, [3000, 2500], [1, 1], heads=2, D=64, G=32, page=16, dt="bf16", seed=18)
    c.fill(1)
    q = torch.randn(2, 4, 64, generator=c.gen).bfloat16().cuda()
    b = c.batch()
    want = c.cache.attention(b, q)
    assert max(b._ws_bytes.values()) > 0
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = c.cache.attention(b, q)
    big = Case(serve, [6000] * 6, [4] * 6, heads=4, D=128, G=64, page=16, dt="bf16", seed=19)
    big.fill(1)
    bq = torch.randn(24, 8, 128, generator=c.gen).bfloat16().cuda()
    bb = big.batch()
    for i in range(3):
        big.cache.attention(bb, bq)
        junk = torch.full((1 << 22,), float("nan"), device="cuda")   # over what was handed back
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
        del junk


@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_append_rounds_a_scale_twice(serve, dt):
    """Groups whose (hi - lo) / 15 rounded to fp32 and then to binary16 is not what one rounding gives."""
    x = 3 * torch.randn(2, 1 << 22, generator=_gen(20)).to(DT[dt]).float()
    lo, hi = torch.minimum(x[0], x[1]).numpy(), torch.maximum(x[0], x[1]).numpy()
    c = np.float32(1 / 15.0)
    twice, once = ((hi - lo) * c).astype(np.float16), ((hi - lo).astype(np.float64) * np.float64(c)).astype(np.float16)
    at = np.flatnonzero(twice != once)
    assert at.size >= 64
    lo, hi = (torch.from_numpy(v[at[:64]])[:, None, None] for v in (lo, hi))
    rows = (lo + (hi - lo) * torch.rand(64, 1, 64, generator=_gen(21))).to(DT[dt])
    rows = torch.minimum(torch.maximum(rows, lo.to(DT[dt])), hi.to(DT[dt]))
    rows[..., 0::32], rows[..., 5::32] = lo.to(DT[dt]), hi.to(DT[dt])
    c = Case(serve, [64], [64], heads=1, D=64, G=32, page=16, dt=dt, seed=22)
    c.cache.append(c.batch(), rows.cuda(), rows.flip(0).contiguous().cuda())
    k, v = c.cache.read(c.batch())
    assert torch.equal(k.cpu(), c.held(rows)) and torch.equal(v.cpu(), c.held(rows.flip(0)))


def test_one_batch_over_caches_of_two_shapes(serve):
    """Layers whose caches differ share a step's batch: each has its own workspace."""
    small = Case(serve, [3000, 2000], [1, 1], heads=1, D=64, G=64, page=16, dt="bf16", seed=23)
    large = Case(serve, [3000, 2000], [1, 1], heads=4, D=128, G=32, page=16, dt="bf16", seed=23)
    large.table = small.table
    for c in (small, large):
        c.fill(1)
    b = small.batch()
    for c in (small, large, small):
        check_attention(c, 2, batch=b)


def test_w4_rows_that_repeat(serve):
    codes, scales, z, _ = _weights(48, 128, 64, torch.float16, True, 24)
    W = serve.W4Weight(codes.cuda(), scales.cuda(), z.cuda())
    x = torch.randn(1, 128, generator=_gen(25)).half().cuda()
    assert torch.equal(W.matmul(x.expand(5, 128)), W.matmul(x.repeat(5, 1)))


@pytest.mark.parametrize("m,n,k,g", [
    (33, 300, 2688, 32), (40, 200, 2880, 64), (64, 500, 4736, 128), (24, 8200, 2944, 128), (20, 8200, 2080, 32),   # parts, rounds that end early
    (130, 5500, 1184, 32), (130, 5500, 1216, 64), (130, 5500, 1408, 128), (70, 8250, 544, 32), (70, 8250, 640, 64)])   # two tiles a wave
def test_w4_by_rows(serve, m, n, k, g):
    dt = "f16" if k % 3 else "bf16"
    codes, scales, z, w = _weights(n, k, g, DT[dt], True, m + n + k)
    x = torch.randn(m, k, generator=_gen(26)).to(DT[dt])
    W = serve.W4Weight(codes.cuda(), scales.cuda(), z.cuda())
    y = W.matmul(x.cuda())
    _check_w4(y, x, w, scales, g, None, dt)
    assert torch.equal(y, W.matmul(x.cuda()))
