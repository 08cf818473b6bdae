"""The paged 8-bit cache (append, read) and attention over it against plain
implementations, at the sizes, lengths, masks and layouts where they can go wrong.

Tolerances, derived before the first run, with u the rounding unit of the result's
type (2^-8 bfloat16, 2^-11 binary16):
* append and read: the definition in fp32, step for step, so values are equal bit
  for bit; a value that was held while its block's scale grew is within one step of itself.
* attention: the weights times the values' scales are rounded to binary16, 2^-11 of
  each; the logarithm of a scale and the exponent (both fp32, of numbers below 128) take 2^-16 of
  a weight.  A score is a sum of D products of up to 255 |q| scales, begun at
  128 sum q, rounded at most D / 8 times on the way: off by
      d = D / 8 * 2^-24 * 255 * scale * (largest key scale) * sum |q|,
  which moves a weight and the sum of weights by d each.  So a result is within
      u |o| + (2^-11 + 2^-16 + 2 d) sum p |v|
  of 64 bits', and 2^-24 of the largest value for fp32's sums; lse within d + 2^-16 + 2^-20 |lse|.
"""
import math
import random

import numpy as np
import pytest
import torch

from test_gpu_serve import plain_attention, turned

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}
LEAST, MOST = 2.0 ** -40, 2.0 ** 10
CAP = torch.tensor(65504.0) * torch.tensor(np.float32(1 / 127.0))


@pytest.fixture(scope="module")
def serve():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2609_02109_amd import serve as m
    return m


def _gen(seed):
    return torch.Generator().manual_seed(seed)


class Held:
    """What a sequence's keys or values are held as: the definition, call by call, in fp32."""

    def __init__(self, heads, D):
        self.codes, self.scales = torch.zeros(0, heads, D), torch.zeros(0, heads)

    def append(self, lo, x):
        """Tokens lo .. of x [tokens, heads, D]."""
        x, n = x.float(), x.shape[0]
        if n == 0:
            return
        hi = lo + n
        more = -(-hi // 16) * 16 - self.codes.shape[0]
        if more > 0:
            self.codes = torch.cat((self.codes, torch.zeros(more, *x.shape[1:])))
            self.scales = torch.cat((self.scales, torch.zeros(more // 16, x.shape[1])))
        for b in range(lo // 16, (hi - 1) // 16 + 1):
            t0, t1 = max(lo, 16 * b), min(hi, 16 * b + 16)
            new = x[t0 - lo:t1 - lo]
            nan = torch.isnan(new).any(-1).any(0)
            y = new.clamp(-65504, 65504)
            need = (y.abs().nan_to_num(0).amax((0, 2)) * torch.tensor(np.float32(1 / 127.0))).clamp(min=LEAST)
            old = self.scales[b]
            held = (torch.isnan(old) | ((old >= LEAST) & (old < MOST))) if t0 > 16 * b else torch.zeros_like(old, dtype=torch.bool)
            grown = old.clone()
            for _ in range(60):
                grown = torch.where(grown < need, (grown * 2).clamp(max=CAP), grown)
            scale = torch.where(held & (old != LEAST), grown, need)
            scale = torch.where(nan | (held & torch.isnan(old)), torch.full_like(scale, math.nan), scale)
            keep = torch.where(held & ~torch.isnan(scale), old / scale, torch.ones_like(scale))   # other codes are 0 here
            block = self.codes[16 * b:16 * b + 16]
            block.copy_((block * keep[:, None]).round().clamp(-127, 127))
            inv = torch.where(torch.isnan(scale), torch.zeros_like(scale), 1.0 / scale)
            self.codes[t0:t1] = (y * inv[:, None]).round().clamp(-127, 127).nan_to_num(0)
            self.scales[b] = scale

    def values(self, n):
        return (self.codes * self.scales.repeat_interleave(16, 0)[..., None])[:n]


class Case:
    """A cache, a batch and their plain copies."""

    def __init__(self, serve, kv, new, heads=2, D=64, page=16, dt="bf16", seed=0, spare=3, leave=255):
        self.serve, self.kv, self.new, self.heads, self.D, self.page, self.dt = serve, kv, new, heads, D, page, dt
        gen = self.gen = _gen(seed)
        n = len(kv)
        cols = max(1, -(-max(kv + [1]) // page))
        self.n_pages = n * cols + spare
        self.table = torch.randperm(self.n_pages, generator=gen).to(torch.int32)[: n * cols].view(n, cols)
        self.cache = serve.KV8Cache(self.n_pages, page, heads, D)
        self.cache.pages.fill_(leave)   # what is not written: NaN scales everywhere
        self.k = [torch.randn(a, heads, D, generator=gen).to(DT[dt]) for a in kv]
        self.v = [torch.randn(a, heads, D, generator=gen).to(DT[dt]) for a in kv]
        self.hk, self.hv = [Held(heads, D) for _ in kv], [Held(heads, D) for _ in kv]

    def batch(self, new=None, kv=None, max_kv=None, table=None):
        new, kv = self.new if new is None else new, self.kv if kv is None else kv
        start = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
        return self.cache.batch(torch.from_numpy(start).cuda(), torch.tensor(kv, dtype=torch.int32).cuda(),
                                (self.table if table is None else table).cuda(), rows=int(start[-1]), max_new=max(new),
                                max_kv=max(kv) if max_kv is None else max_kv)

    def rows(self, per_seq, new, kv):
        return torch.cat([t[b - a:b] for t, a, b in zip(per_seq, new, kv)])

    def put(self, new, upto, angles=None, inter=False):
        """One call: the newest `new` of the first `upto` tokens of every sequence."""
        rot = {} if angles is None else dict(cos=angles[0], sin=angles[1], interleaved=inter)
        self.cache.append(self.batch(new, upto, max_kv=max(self.kv)), self.rows(self.k, new, upto).cuda(), self.rows(self.v, new, upto).cuda(), **rot)
        for i, (n, u) in enumerate(zip(new, upto)):
            k = self.k[i][u - n:u].float()
            if angles is not None and n:
                k = turned(k, *(t.cpu()[u - n:u] for t in angles), inter)
            self.hk[i].append(u - n, k)
            self.hv[i].append(u - n, self.v[i][u - n:u])

    def fill(self, steps=1, angles=None, inter=False):
        """Every token, in `steps` calls of ragged sizes."""
        done = [0] * len(self.kv)
        for i in range(steps):
            upto = [a * (i + 1) // steps for a in self.kv]
            new = [b - a for a, b in zip(done, upto)]
            if sum(new):
                self.put(new, upto, angles, inter)
            done = upto

    def held(self):
        return (torch.cat([h.values(n) for h, n in zip(self.hk, self.kv)]), torch.cat([h.values(n) for h, n in zip(self.hv, self.kv)]))

    def check_read(self):
        b = self.batch(new=self.kv)
        for ty in (torch.float32, DT[self.dt]):
            for got, want in zip(self.cache.read(b, ty), self.held()):
                want = want.to(ty)
                nan = torch.isnan(want)
                assert torch.equal(torch.isnan(got.cpu()), nan) and torch.equal(got.cpu()[~nan], want[~nan])


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_append_and_read(serve, D, dt):
    # pages of one block and of three, calls that end inside blocks and go on in them; one token at a time
    for page, steps, seed in ((16, 1, 1), (48, 5, 2), (16, 13, 3), (32, 130, 4)):
        c = Case(serve, [1, 77, 16, 33, 130], None, heads=3, D=D, page=page, dt=dt, seed=seed)
        c.fill(steps)
        c.check_read()


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D,rot", [(64, 64), (64, 16), (128, 128), (128, 48), (256, 256), (256, 64)])
def test_append_turns_keys_and_queries(serve, D, rot, inter):
    dt = "bf16" if rot % 32 else "f16"
    c = Case(serve, [5, 70, 21], [5, 9, 1], heads=2, D=D, page=32, dt=dt, seed=rot)
    angles = serve.rope_table(80, rot)
    c.fill(3, angles, inter)
    c.check_read()
    q = torch.randn(15, 6, D, generator=c.gen).to(DT[dt])
    qd = q.cuda()
    k, v = c.rows(c.k, c.new, c.kv).cuda(), c.rows(c.v, c.new, c.kv).cuda()
    qr = c.cache.append(c.batch(), k, v, cos=angles[0], sin=angles[1], q=qd, interleaved=inter)
    for i, n in enumerate(c.new):   # the same tokens again: scales that are enough stay
        u = c.kv[i]
        c.hk[i].append(u - n, turned(c.k[i][u - n:].float(), *(t.cpu()[u - n:u] for t in angles), inter))
        c.hv[i].append(u - n, c.v[i][u - n:])
    c.check_read()
    new = torch.cat([torch.arange(a - n, a) for a, n in zip(c.kv, c.new)])
    cos, sin = (t.cpu().double()[new] for t in angles)
    want = turned(q.double(), cos, sin, inter)
    partner = turned(q.double().abs(), torch.ones(15, rot // 2), -torch.ones(15, rot // 2), inter).abs() + q.double().abs()
    assert ((qr.cpu().double() - want).abs() <= UNIT[dt] * want.abs() + 3 * 2.0 ** -24 * partner + 2.0 ** -24).all()
    c.cache.append(c.batch(), k, v, cos=angles[0], sin=angles[1], q=qd, q_out=qd, interleaved=inter)   # over its source
    assert torch.equal(qd, qr)


@pytest.mark.parametrize("per", [1, 5, 9, 20, 33])   # heads of queries to a head of keys
@pytest.mark.parametrize("new,D,rot,inter", [([2, 7, 1], 64, 64, False), ([2, 7, 0], 64, 32, True), ([3, 1, 5], 128, 96, False), ([3, 1, 5], 256, 256, True),
                                             ([8, 1, 0], 64, 64, False), ([40, 17, 3], 64, 16, True), ([40, 17, 3], 128, 128, False), ([9, 33, 16], 256, 64, False)])
def test_append_turns_any_number_of_queries(serve, new, D, rot, inter, per):
    c = Case(serve, [70, 50, 33], new, heads=1, D=D, seed=per)
    rows = sum(new)
    angles = serve.rope_table(80, rot)
    q = torch.randn(rows, per, D, generator=c.gen).bfloat16()
    k, v = c.rows(c.k, c.new, c.kv).cuda(), c.rows(c.v, c.new, c.kv).cuda()
    at = torch.cat([torch.arange(a - n, a) for a, n in zip(c.kv, c.new)])
    want = turned(q.double(), *(t.cpu().double()[at] for t in angles), inter)
    partner = turned(q.double().abs(), torch.ones(rows, rot // 2), -torch.ones(rows, rot // 2), inter).abs() + q.double().abs()
    for cache in (c.cache, serve.KV4Cache(c.n_pages, c.page, 1, D, group=64)):
        cache.pages.zero_()
        start = torch.tensor([0, *np.cumsum(new)], dtype=torch.int32).cuda()
        b = cache.batch(start, torch.tensor(c.kv, dtype=torch.int32).cuda(), c.table.cuda(), rows=rows, max_new=max(new), max_kv=70)
        # rows inside wider ones, whose other values stay as they are
        wide = torch.full((rows + 1, per * D + 8), 7.0, dtype=torch.bfloat16, device="cuda")
        to = wide[:rows, :per * D].view(rows, per, D)
        cache.append(b, k, v, cos=angles[0], sin=angles[1], q=q.cuda(), q_out=to, interleaved=inter)
        assert ((to.cpu().double() - want).abs() <= UNIT["bf16"] * want.abs() + 3 * 2.0 ** -24 * partner).all()
        assert (wide[rows] == 7).all() and (wide[:, per * D:] == 7).all()
        over = q.cuda()
        cache.append(b, k, v, cos=angles[0], sin=angles[1], q=over, q_out=over, interleaved=inter)
        assert torch.equal(over, to)


def test_append_strides(serve):
    # k and v as slices of one projection with an odd row length, then [heads, rows, D]
    for turn in (False, True):
        c = Case(serve, [40, 19], [40, 19], heads=2, D=64, dt="f16", seed=9)
        k, v = torch.cat(c.k), torch.cat(c.v)
        if turn:
            kd, vd = (t.transpose(0, 1).contiguous().cuda().transpose(0, 1) for t in (k, v))
        else:
            wide = torch.full((59, 2 * 2 * 64 + 5), float("nan"), dtype=torch.float16)
            wide[:, 3:131], wide[:, 131:259] = k.flatten(1), v.flatten(1)
            kd, vd = (wide.cuda().as_strided((59, 2, 64), (261, 64, 1), at) for at in (3, 131))
        c.cache.append(c.batch(), kd, vd)
        for i in range(2):
            c.hk[i].append(0, c.k[i])
            c.hv[i].append(0, c.v[i])
        c.check_read()


@pytest.mark.parametrize("D", [64, 128, 256])
def test_scales_that_grow(serve, D):
    # token by token, each larger than the ones before; a block of zeros first; a token far larger; ones that need no more
    c = Case(serve, [32, 32, 48, 16], None, heads=2, D=D, page=16, dt="bf16", seed=12)
    up = torch.tensor([1.17 ** (i % 16) for i in range(48)])[:, None, None]
    c.k[0], c.v[0] = (c.k[0].float() * up[:32]).bfloat16(), (c.v[0].float() * up[:32] ** 3).bfloat16()
    c.k[1][:9], c.v[1][:20] = 0, 0
    c.k[2][5] *= 5000
    c.v[2][18] = 2.0 ** -60
    c.v[2][17], c.v[2][16], c.v[2][19] = 0, 0, 1e-9
    c.k[3][15, 1, 3], c.v[3][0, 0, 0] = 3e38, -1e30
    for n in range(1, 49):
        upto = [min(n, a) for a in c.kv]
        c.put([int(n <= a) for a in c.kv], upto)
    c.check_read()
    # less than a step in all, however often a code was rounded
    x, got = torch.cat(c.k).float().clamp(-65504, 65504), c.cache.read(c.batch(new=c.kv))[0].cpu()
    step = torch.cat([h.scales.repeat_interleave(16, 0)[:n] for h, n in zip(c.hk, c.kv)])[..., None]
    assert ((got - x).abs() < step).all() and ((got - x).abs() > 0.55 * step).any()


def test_the_largest_values_stay_numbers(serve):
    # a block that is near the most a scale can be, and tokens at the type's end after it
    c = Case(serve, [16, 20], None, heads=2, D=64, page=16, dt="f16", seed=18)
    c.k[0][:3], c.v[0][:5] = 65280.0, -40000.0
    c.k[0][9], c.v[0][10, 1] = 65504.0, 65504.0
    c.k[1][16], c.v[1][17] = -65504.0, float("inf")
    c.fill(8)
    c.check_read()
    k, v = c.cache.read(c.batch(new=c.kv), torch.float16)
    assert torch.isfinite(k).all() and torch.isfinite(v).all()
    c.new = [3, 2]
    q = torch.zeros(5, 4, 64).half()
    got = check(c, 2, q=q)
    assert torch.isfinite(got[0]).all()


def test_append_of_odd_values(serve):
    # constants, subnormals, the largest values, infinities: each in a block of its own; a NaN, and tokens after it
    c = Case(serve, [16] * 6 + [40], None, heads=1, D=64, dt="bf16", seed=10)
    c.k[0][:], c.k[1][:] = 1.5, 0.0
    c.k[2] = (1e-9 * torch.arange(64)).expand(16, 1, 64).bfloat16()
    c.k[3][3, 0, 5] = 3e38
    c.k[4][4, 0, 40], c.k[4][4, 0, 41] = float("-inf"), float("inf")
    c.k[5][:] = 1e-39
    c.k[6][19, 0, 33] = float("nan")
    c.v = [t.flip(0) for t in c.k]
    c.fill(5)
    c.check_read()
    k, v = c.cache.read(c.batch(new=c.kv))
    assert torch.isfinite(k[:96]).all() and torch.isfinite(v[:96]).all()
    assert torch.isnan(k[96 + 16:96 + 32]).all() and torch.isfinite(k[96:96 + 16]).all() and torch.isfinite(k[96 + 32:]).all()
    assert torch.isnan(v[96 + 16:96 + 32]).all()
    # the block begun anew
    c.k[6][19, 0, 33], c.v[6][40 - 1 - 19, 0, 33] = 1.0, 1.0
    c.put([0] * 6 + [24], c.kv)
    c.check_read()


def test_append_leaves_the_rest_alone(serve):
    c = Case(serve, [30, 45], [3, 5], heads=2, D=128, page=16, dt="bf16", seed=11, spare=5)
    c.fill(2)
    k, v = torch.randn(8, 2, 128).bfloat16().cuda(), torch.randn(8, 2, 128).bfloat16().cuda()
    raw = c.cache.pages.clone()
    bad = c.table.clone()
    bad[0, 1], bad[1, 2] = c.n_pages, -1
    c.cache.append(c.batch(table=bad), k, v)    # page numbers that are none
    c.cache.append(c.batch(max_kv=20), k, v)    # tokens past max_kv
    c.cache.append(c.batch(new=[0, 0]), k[:0], v[:0])
    torch.cuda.synchronize()
    assert torch.equal(c.cache.pages, raw)
    assert all((t == 0).all() for t in c.cache.read(c.batch(table=bad)))
    # more new tokens than tokens: those at negative positions are left out
    c.cache.append(c.batch(new=[3, 5], kv=[2, 0], max_kv=45), k, v)
    h = Held(2, 128)
    h.append(0, k.cpu()[1:3])
    assert torch.equal(c.cache.read(c.batch(new=[2, 0], kv=[2, 0], max_kv=45))[0].cpu(), h.values(2))
    # a step writes its own blocks and nothing else
    c.cache.pages.copy_(raw)
    c.cache.append(c.batch(), k, v)
    torch.cuda.synchronize()
    n, rec = c.n_pages * 2, 32 * 128
    same = (c.cache.pages[: n * rec].view(n, rec) == raw[: n * rec].view(n, rec)).all(1).view(c.n_pages, 2).all(1).cpu()
    touched = {int(c.table[0, 1]), int(c.table[1, 2])}
    assert touched == set(torch.nonzero(~same).flatten().tolist())


@pytest.mark.parametrize("leave", [0, 0x3c, 0x7f, 0x80, 255])
def test_memory_that_was_never_written(serve, leave):
    # whatever the pages hold: blocks that are begun by their first token; zeros: by any
    c = Case(serve, [50, 35], None, heads=2, D=64, page=32, dt="f16", seed=13, leave=leave)
    c.fill(7)
    c.check_read()
    if leave == 0:
        c = Case(serve, [50, 35], None, heads=2, D=64, page=32, dt="f16", seed=14, leave=0)
        c.put([9, 2], c.kv)
        k, _ = c.cache.read(c.batch(new=[9, 2]))
        want = torch.cat((c.hk[0].values(50)[41:], c.hk[1].values(35)[33:]))
        assert torch.equal(k.cpu(), want) and (k.cpu() - c.rows(c.k, [9, 2], c.kv).float()).abs().max() < 3.5 / 127
        k, v = c.cache.read(c.batch(new=c.kv))   # what was there before are zeros
        old = torch.cat((torch.arange(41), torch.arange(50, 83)))
        assert (k[old] == 0).all() and (v[old] == 0).all()
        q = torch.randn(11, 4, 64, generator=c.gen).half()
        got = c.cache.attention(c.batch(new=[9, 2]), q.cuda(), lse=True)
        check(c, 2, q=q, new=[9, 2], got=got)


# -------------------------------------------------------------- attention

def check(c, per, q=None, window=0, scale=None, got=None, batch=None, new=None, kv=None, **kw):
    new, kv = c.new if new is None else new, c.kv if kv is None else kv
    heads = per * c.heads
    if q is None:
        q = (1.5 * torch.randn(sum(new), heads, c.D, generator=c.gen)).to(DT[c.dt])
    if got is None:
        got = c.cache.attention(c.batch(new=new, kv=kv) if batch is None else batch, q.cuda(), scale=scale, window=window, lse=True, **kw)
        torch.cuda.synchronize()
    out, ls = got[0].cpu().double(), got[1].cpu().double()
    sm = 1 / math.sqrt(c.D) if scale is None else scale
    at = 0
    for i, n in enumerate(new):
        hk, hv = c.hk[i].values(kv[i]).double(), c.hv[i].values(kv[i]).double()
        qs = q[at:at + n]
        o, l, p = plain_attention(qs, hk, hv, per, n, window, sm)
        if kv[i] and n:
            room = torch.stack([p[:, h] @ hv[:, h // per].abs() for h in range(heads)], 1)
            ks = c.hk[i].scales[: -(-kv[i] // 16)].amax(0).double().repeat_interleave(per)
            d = (c.D / 8 * 2.0 ** -24 * 255 * sm * ks * qs.double().abs().sum(-1))[..., None]
            top = float(hv.abs().max())
        else:
            room, d, top = torch.zeros_like(o), torch.zeros(n, heads, 1, dtype=torch.float64), 0.0
        tol = UNIT[c.dt] * o.abs() + (2.0 ** -11 + 2.0 ** -16 + 2 * d) * room + 2.0 ** -24 * top
        err = (out[at:at + n] - o).abs()
        assert (err <= tol).all(), (i, n, float((err / tol.clamp(min=1e-30)).max()))
        seen, mine = torch.isfinite(l), ls[at:at + n]
        assert torch.equal(torch.isfinite(mine), seen)
        assert (out[at:at + n][~seen] == 0).all() and (mine[~seen] == -math.inf).all()
        assert ((mine - l)[seen].abs() <= (d[..., 0] + 2.0 ** -16 + 2.0 ** -20 * l.abs())[seen]).all()
        at += n
    return got


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_attention_one_token(serve, D, dt):
    c = Case(serve, [1, 15, 16, 17, 0, 31, 33, 129, 500], [1] * 9, heads=2, D=D, page=16, dt=dt, seed=D)
    c.fill(2)
    for per in (1, 4, 16):
        check(c, per)


@pytest.mark.parametrize("per,new", [(1, 2), (1, 17), (3, 5), (5, 7), (8, 33), (4, 70), (32, 1), (24, 2), (2, 130)])
def test_attention_several_tokens(serve, per, new):
    D = (64, 128, 256)[new % 3]
    c = Case(serve, [new, new + 40, 200, max(0, new - 3)], [new, new, new, new], heads=2, D=D, page=32, dt="bf16", seed=per * new)
    c.fill(1)
    check(c, per)


def test_attention_ragged_new(serve):
    # some sequences bring nothing, one token, a prompt
    c = Case(serve, [60, 5, 90, 33, 64], [0, 1, 40, 33, 3], heads=2, D=128, page=16, dt="f16", seed=5)
    c.fill(2)
    check(c, 2)


@pytest.mark.parametrize("window", [1, 15, 16, 33, 100, 5000])
def test_attention_window(serve, window):
    c = Case(serve, [300, 20, 131], [1, 1, 1], heads=1, D=64, page=48, dt="bf16", seed=window)
    c.fill(1)
    check(c, 3, window=window)
    c = Case(serve, [300, 41, 130], [64, 41, 50], heads=1, D=64, page=16, dt="bf16", seed=window + 1)
    c.fill(1)
    check(c, 3, window=window)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_attention_split_over_tokens(serve, D):
    # contexts long enough to be taken apart, of very different lengths, and the join of parts that hold nothing
    c = Case(serve, [9000, 3, 4097, 0], [1, 1, 1, 1], heads=1, D=D, page=64, dt="bf16", seed=6)
    c.fill(1)
    check(c, 4)
    check(c, 20 if D < 256 else 9)
    check(c, 2, window=4500)


def test_attention_rows_split_over_tokens(serve):
    c = Case(serve, [5000, 120], [40, 40], heads=1, D=128, page=64, dt="f16", seed=7)
    c.fill(1)
    check(c, 2)


@pytest.mark.parametrize("kv,window", [([1057, 33], 0), ([1570, 1100], 0), ([3000, 40], 1100)])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_attention_rows_in_parts_of_odd_lengths(serve, D, kv, window):
    # parts of an odd number of times 32 tokens: a step of 64 goes past the end of one
    c = Case(serve, kv, [33, 21], heads=2, D=D, page=32, dt="bf16", seed=sum(kv))
    c.fill(1)
    check(c, 2, window=window)


def test_attention_many_sequences(serve):
    # more than a wave's lanes, with none and many tokens among them
    kv = [(37 * i) % 211 for i in range(150)] + [5000]
    c = Case(serve, kv, [1] * 151, heads=1, D=64, page=16, dt="f16", seed=8)
    c.fill(1)
    check(c, 2)


def test_attention_scale_and_strides(serve):
    c = Case(serve, [70, 40], [3, 3], heads=2, D=64, page=16, dt="bf16", seed=15)
    c.fill(3)
    check(c, 2, scale=0.5)
    q = torch.randn(6, 4, 64, generator=c.gen).bfloat16()
    want = check(c, 2, q=q)
    wide = torch.full((6, 4 * 64 + 3), float("nan"), dtype=torch.bfloat16, device="cuda")
    view = wide.as_strided((6, 4, 64), (259, 64, 1), 1)
    view.copy_(q)
    big = torch.full((6, 4 * 64 + 5), 7.0, dtype=torch.bfloat16, device="cuda")
    out = big.as_strided((6, 4, 64), (261, 64, 1), 3)
    assert torch.equal(c.cache.attention(c.batch(), view, out=out), want[0]) and (big[:, :3] == 7).all() and (big[:, 259:] == 7).all()
    turned_q = q.transpose(0, 1).contiguous().cuda().transpose(0, 1)
    assert torch.equal(c.cache.attention(c.batch(), turned_q), want[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = c.cache.attention(c.batch(), q.cuda(), stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want[0])


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("kv,new,per", [([90, 37, 20, 0], [1, 1, 1, 1], 4), ([90, 37, 21], [20, 7, 3], 2), ([2500, 37], [1, 1], 2), ([150], [60], 3)])
def test_attention_does_not_depend_on_leftovers(serve, dt, kv, new, per):
    """The rest of a sequence's last page, and pages that are none of the cache's: the same bits whatever the memory holds."""
    want = None
    for leave in (0, 0x3c, 0x7f, 0x80, 255):
        c = Case(serve, kv, new, heads=1, D=128, page=16 if kv[0] < 1000 else 64, dt=dt, seed=31, leave=leave)
        q = torch.randn(sum(new), per, 128, generator=c.gen).to(DT[dt])
        bad = c.table.clone()
        bad[0, 1], bad[-1, 0] = -1, c.n_pages
        c.fill(1)
        got = [*c.cache.attention(c.batch(), q.cuda(), lse=True), *c.cache.attention(c.batch(table=bad), q.cuda(), lse=True)]
        if want is None:
            want = got
            check(c, per, q=q, got=got[:2])
        assert all(torch.equal(a, b) for a, b in zip(got, want)), leave


@pytest.mark.parametrize("new,per", [(1, 4), (5, 4), (20, 4)])
def test_attention_in_a_window_over_pages_that_were_given_back(serve, new, per):
    """Blocks before every row's window need not be there: their pages may be another's by now."""
    tail = 300 - (300 - (24 + new - 1)) // 16 * 16
    want = None
    for leave in (0, 0x3c, 0x7f, 0x80, 255):
        c = Case(serve, [300], [new], heads=2, D=64, page=16, dt="bf16", seed=32, leave=leave)
        q = torch.randn(new, 2 * per, 64, generator=c.gen).bfloat16()
        c.put([tail], c.kv)
        got = c.cache.attention(c.batch(), q.cuda(), window=24, lse=True)
        if want is None:
            want = got
            check(c, per, q=q, window=24, got=got)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), leave


@pytest.mark.parametrize("big", [1e-6, 40.0, 3000.0])
def test_a_row_does_not_depend_on_later_blocks(serve, big):
    for window in (0, 30):
        c = Case(serve, [100], [40], heads=1, D=128, page=32, dt="f16", seed=33)
        q = torch.randn(40, 2, 128, generator=c.gen).half()
        c.fill(1)
        want = check(c, 2, q=q, window=window)
        for pos in (81, 85, 97):
            c.v[0][pos] = (c.v[0][pos].float() * big).half()
            c.k[0][pos] = (c.k[0][pos].float() * min(big, 40.0)).half()
        c.fill(1)
        got = check(c, 2, q=q, window=window)
        assert torch.equal(got[0][:20], want[0][:20]) and torch.equal(got[1][:20], want[1][:20]) and not torch.equal(got[0][20:], want[0][20:])


def test_a_cache_past_32_bits(serve):
    # pages beyond 4 GiB: 40,000 of 131,328 bytes; a few sequences in the last ones
    c = Case(serve, [40, 100, 2100], [1, 2, 1], heads=8, D=128, page=64, dt="bf16", seed=19)
    big = serve.KV8Cache(40_000, 64, 8, 128)
    assert big.pages.numel() > 2 ** 32
    c.cache, c.n_pages = big, 40_000
    c.table = (39_999 - c.table).to(torch.int32)
    c.fill(2)
    c.check_read()
    check(c, 2)


def test_sequences_that_share_pages(serve):
    """A prefix that two sequences have in common, in the same pages; the rest is each's own."""
    c = Case(serve, [70, 90], [1, 1], heads=2, D=128, page=32, dt="bf16", seed=20)
    c.table[1, :2] = c.table[0, :2]
    c.k[1][:64], c.v[1][:64] = c.k[0][:64], c.v[0][:64]
    c.put([64, 0], [64, 0])
    for held in (c.hk, c.hv):
        held[1].codes, held[1].scales = held[0].codes.clone(), held[0].scales.clone()
    c.put([6, 26], [70, 90])
    c.check_read()
    for per in (1, 4):
        check(c, per)
    check(c, 40, new=[1, 1])


def test_attention_with_a_nan(serve):
    # in a block that some rows see: those are NaN, and no others; a query with one or an infinity: its own rows
    c = Case(serve, [100, 64], [40, 1], heads=2, D=64, page=16, dt="bf16", seed=34)
    q = torch.randn(41, 4, 64, generator=c.gen).bfloat16()
    c.fill(1)
    want = check(c, 2, q=q)
    c.v[0][83, 0, 5] = float("nan")
    c.k[1][40, 1, 7] = float("nan")
    c.fill(1)
    out, _ = c.cache.attention(c.batch(), q.cuda(), lse=True)
    nan = torch.isnan(out).all(-1).cpu()
    some = torch.isnan(out).any(-1).cpu()
    wanted = torch.zeros(41, 4, dtype=torch.bool)
    wanted[20:40, :2] = True    # rows from position 80 on
    wanted[40, 2:] = True
    assert torch.equal(nan, wanted) and torch.equal(some, wanted) and torch.equal(out.cpu()[~wanted], want[0].cpu()[~wanted])
    c = Case(serve, [50], [3], heads=1, D=64, page=16, dt="f16", seed=35)
    c.fill(1)
    q = torch.randn(3, 2, 64, generator=c.gen).half()
    clean = c.cache.attention(c.batch(), q.cuda())
    q[1, 0, 3], q[2, 1, 0] = float("nan"), float("inf")
    got = c.cache.attention(c.batch(), q.cuda())
    assert torch.isnan(got[1, 0]).all() and not torch.isfinite(got[2, 1]).all()
    keep = [(0, 0), (0, 1), (1, 1), (2, 0)]
    assert all(torch.equal(got[i, h], clean[i, h]) for i, h in keep)


@pytest.mark.parametrize("big", [2.0 ** -30, 2.0 ** -12, 1.0, 2.0 ** 14])
@pytest.mark.parametrize("new,per", [(1, 4), (30, 3)])
def test_values_of_all_sizes(serve, big, new, per):
    """Blocks whose values are far smaller or larger than the others': each weighs by what it adds."""
    for at in (0, 5, 17):
        c = Case(serve, [400], [new], heads=1, D=128, page=64, dt="bf16", seed=36 + at)
        c.v[0][16 * at:16 * at + 16] = (c.v[0][16 * at:16 * at + 16].float() * big).bfloat16()
        c.v[0] = (c.v[0].float() * 2.0 ** -3).bfloat16()
        c.fill(1)
        check(c, per)
    # one token that weighs 2^20 times the others, with values of its block as small in proportion
    c = Case(serve, [400], [new], heads=1, D=128, page=64, dt="f16", seed=40)
    q = torch.zeros(new, per, 128)
    q[..., 0] = 1.0
    c.k[0][:, 0, 0], c.k[0][40, 0, 0] = 0.0, 12.0
    c.k[0][:, 0, 1:] = (c.k[0][:, 0, 1:].float() * 0.01).half()
    c.v[0][32:48] = (c.v[0][32:48].float() * 2.0 ** -18).half()
    c.fill(1)
    check(c, per, q=q.half(), scale=20 * math.log(2) / 12)


@pytest.mark.parametrize("size", [2.0 ** -100, 2.0 ** -20, 1.0, 2.0 ** 30, 2.0 ** 100])
def test_queries_of_all_sizes(serve, size):
    c = Case(serve, [200], [2], heads=1, D=128, page=16, dt="bf16", seed=41)
    c.fill(1)
    q = (torch.randn(2, 4, 128, generator=c.gen) * size).bfloat16()
    check(c, 4, q=q, scale=0.1 / size)
    check(c, 4, q=torch.zeros_like(q))


def test_deterministic_and_apart(serve):
    # the same bits again; two threads' worth of streams; a batch of rows past the last sequence stays as it was
    c = Case(serve, [3000, 700, 9], [1, 1, 1], heads=4, D=128, page=16, dt="bf16", seed=42)
    c.fill(1)
    q = torch.randn(3, 16, 128, generator=c.gen).bfloat16().cuda()
    want = c.cache.attention(c.batch(), q, lse=True)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = [c.cache.attention(c.batch(), q, lse=True, stream=s) for _ in range(4) for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))
    b = c.cache.batch(torch.tensor([0, 1, 2, 3], dtype=torch.int32).cuda(), torch.tensor(c.kv, dtype=torch.int32).cuda(), c.table.cuda(),
                      rows=5, max_new=1, max_kv=3000)
    out = torch.full((5, 16, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    c.cache.attention(b, torch.cat((q, q[:2])), out=out)
    assert torch.equal(out[:3], want[0]) and (out[3:] == 7).all()


def test_batch_arrays_that_lie(serve):
    # lengths, starts and page numbers that are none: nothing outside of the buffers is read or written, and other sequences are right
    c = Case(serve, [90, 50, 70], [1, 1, 1], heads=1, D=64, page=16, dt="bf16", seed=43)
    c.fill(1)
    q = torch.randn(3, 2, 64, generator=c.gen).bfloat16().cuda()
    want = c.cache.attention(c.batch(), q)
    raw = c.cache.pages.clone()
    i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()
    for start, kv in (([0, 1, 2, 3], [90, 2 ** 31 - 1, 70]), ([0, 1, 2, 3], [90, -5, 70]), ([0, 1, 2 ** 30, 3], [90, 50, 70]),
                      ([0, 1, -7, 3], [90, 50, 70])):
        b = c.cache.batch(i32(start), i32(kv), c.table.cuda(), rows=3, max_new=1, max_kv=90)
        got = c.cache.attention(b, q)
        assert torch.equal(got[0], want[0])
        c.cache.read(b)
    torch.cuda.synchronize()
    assert torch.equal(c.cache.pages, raw)


def test_refusals(serve):
    from paper_2609_02109_amd import mf
    c = Case(serve, [20], [1], heads=2, D=64, page=16, seed=44)
    b = c.batch()
    k = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    cos, sin = serve.rope_table(32, 64)
    for bad in (lambda: c.cache.append(b, k.float(), k), lambda: c.cache.append(b, k, k.half()), lambda: c.cache.append(b, k[:, :1], k),
                lambda: c.cache.append(b, k, k, cos=cos), lambda: c.cache.append(b, k, k, q=q), lambda: c.cache.append(b, k.cpu(), k),
                lambda: c.cache.append(b, k.clone().requires_grad_(), k), lambda: c.cache.attention(b, q[:, :, :32]), lambda: c.cache.attention(b, q.float()),
                lambda: c.cache.attention(b, q.clone().requires_grad_()), lambda: c.cache.attention(b, q, out=k), lambda: c.cache.read(b, torch.int8),
                lambda: serve.KV8Cache(2 ** 32 + 1, 16, 2, 64)):
        with pytest.raises(ValueError):
            bad()
    for sizes, want in (((4, 20, 2, 64), mf.MF_EUNSUPPORTED), ((4, 16, 2, 96), mf.MF_EUNSUPPORTED), ((0, 16, 2, 64), mf.MF_EINVAL)):
        with pytest.raises(mf.MfError) as e:
            serve.KV8Cache(*sizes)
        assert e.value.status == want
    with pytest.raises(mf.MfError):
        c.cache.attention(b, q[:, :3])
    with pytest.raises(mf.MfError):
        c.cache.attention(b, q, window=-1)
    with pytest.raises(mf.MfError):
        c.cache.append(b, k, k, cos=cos[:16], sin=sin[:16])
    # a batch of either cache's is of use to both
    other = serve.KV4Cache(c.n_pages, 16, 2, 64, group=32)
    other.append(b, k, k)
    assert c.cache.bytes_per_token == 2 * (2 * 64) + 1 and (c.cache.pages.numel() == c.n_pages * 2 * (32 * 64 + 8))


def test_a_step_in_a_graph(serve):
    """Append and attention captured and replayed while lengths, pages and rows change, beside the same calls by hand."""
    hq, hk, D, page, n = 8, 2, 128, 16, 3
    rng = random.Random(5)
    gen = _gen(45)
    lens = [rng.randint(1, 120) for _ in range(n)]
    one, two = (serve.KV8Cache(n * 10, page, hk, D) for _ in range(2))
    for cache in (one, two):
        cache.pages.zero_()
    table = torch.randperm(n * 10, generator=gen).to(torch.int32).view(n, 10).cuda()
    start, kv = torch.arange(n + 1, dtype=torch.int32).cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    cos, sin = serve.rope_table(160, D)
    qkv = torch.empty(n, hq + 2 * hk, D, dtype=torch.bfloat16, device="cuda")

    def step(cache):
        b = cache.batch(start, kv, table, n, 1, 160)
        q = cache.append(b, qkv[:, hq:hq + hk], qkv[:, hq + hk:], cos=cos, sin=sin, q=qkv[:, :hq])
        return q, *cache.attention(b, q, lse=True)

    qkv.copy_(torch.randn(qkv.shape, generator=gen))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    spare = serve.KV8Cache(n * 10, page, hk, D)
    with torch.cuda.stream(side):
        step(spare)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(one)
    for _ in range(25):
        qkv.copy_(torch.randn(qkv.shape, generator=gen) * rng.choice([0.3, 1, 4]))
        graph.replay()
        want = step(two)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        kv += 1
    assert torch.equal(one.pages, two.pages)
