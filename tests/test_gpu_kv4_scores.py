"""Attention over the 4-bit cache where scores are large: results are numbers, and the ones that the formula has.

What is expected, and how far off it may be: keys and queries have one dim that is not 0, so a score is one
product.  Tokens of the largest score have the same key, hence the same score bit for bit, and lead the others by
0.2 S > 2^17 (in powers of two), where every other weight is 0.  So a row's result is the mean of those tokens' values
as they are held.  A value is offset + scale code, below 4 + 8 here, whose factors are rounded to binary16 (2^-11,
alone and times the scale), and their sums are fp32:
    u |o| + 2 2^-11 12,   u the rounding unit of the result's type,
and lse = score + log(number) to 2^-20 of itself (key scale, factor, score and sum: four roundings of 2^-24) and 2^-16.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}
# new tokens, query heads to a key head, tokens: whole heads by tokens, by shares, rows, rows in parts
FORMS = [(1, 4, 200), (1, 4, 5000), (30, 3, 200), (64, 4, 3000)]


def _i32(*v):
    return torch.tensor(v, dtype=torch.int32).cuda()


class Case:
    """One sequence of kv tokens, one key head, whose keys have `keys` in dim 0."""

    def __init__(self, kv, new, D, dt, keys=None, heads=1, seed=0):
        from paper_2609_02109_amd import serve
        gen = self.gen = torch.Generator().manual_seed(seed)
        self.kv, self.new, self.dt = kv, new, dt
        cols = -(-kv // 64)
        self.cache = serve.KV4Cache(cols, 64, heads, D)
        table = torch.randperm(cols, generator=gen).to(torch.int32).view(1, cols).cuda()
        k = torch.randn(kv, heads, D, generator=gen).to(DT[dt])
        if keys is not None:
            k.zero_()
            k[:, 0, 0] = keys.to(DT[dt])
        v = torch.randn(kv, heads, D, generator=gen).clamp(-4, 4).to(DT[dt])
        whole = self.cache.batch(_i32(0, kv), _i32(kv), table, kv, kv, kv)
        self.cache.append(whole, k.cuda(), v.cuda())
        self.k, self.v = (t.cpu().double() for t in self.cache.read(whole))
        self.batch = self.cache.batch(_i32(0, new), _i32(kv), table, new, new, kv)

    def check(self, q, top, scale):
        """top [tokens]: those of the largest score."""
        out, lse = (t.cpu().double() for t in self.cache.attention(self.batch, q.cuda(), scale=scale, lse=True))
        for i in range(self.new):
            seen = top & (torch.arange(self.kv) <= self.kv - self.new + i)
            want = self.v[seen, 0].mean(0)
            assert ((out[i] - want).abs() <= UNIT[self.dt] * want.abs() + 2.0 ** -10 * 12).all(), (i, out[i, 0, :4], want[:4])
            s = scale * q[i, :, 0].double() * self.k[seen, 0, 0][0] + math.log(int(seen.sum()))
            assert ((lse[i] - s).abs() <= 2.0 ** -16 + 2.0 ** -20 * s.abs()).all(), (i, lse[i], s)


@pytest.mark.parametrize("dt,D,size", [("bf16", 64, 20), ("f16", 128, 20), ("bf16", 128, 27), ("f16", 64, 27), ("bf16", 256, 27), ("bf16", 128, 40),
                                       ("f16", 256, 40), ("bf16", 64, 103), ("bf16", 256, 103)])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("new,per,kv", FORMS)
def test_large_scores(new, per, kv, sign, dt, D, size):
    gen = torch.Generator().manual_seed(size)
    top = torch.rand(kv, generator=gen) < 0.05
    top[3] = True
    others = torch.rand(kv, generator=gen) * (1.5 if sign > 0 else 0.5)
    keys = torch.where(top, 1.0, others - 1.0) if sign > 0 else torch.where(top, 0.25, others + 0.5)
    most = 2.0 ** 15 if size > 100 else 1.0
    c = Case(kv, new, D, dt, keys * most, seed=50 + size)
    big = 2.0 ** (min(size, 88) if dt == "bf16" else 10)
    q = torch.zeros(new, per, D)
    q[..., 0] = sign * big
    c.check(q.to(DT[dt]), top, 2.0 ** size / most / big)


@pytest.mark.parametrize("size", [21, 27, 40, 80])
@pytest.mark.parametrize("new,per,kv", FORMS)
def test_large_scores_then_small_ones(new, per, kv, size):
    """The first half's scores are far below the rest's, which are 0."""
    keys = torch.zeros(kv)
    keys[:kv // 32 * 16] = 1.0
    c = Case(kv, new, 128, "bf16", keys, seed=60)
    q = torch.zeros(new, per, 128)
    q[..., 0] = -2.0 ** size
    c.check(q.bfloat16(), keys == 0, 1.0)


@pytest.mark.parametrize("size", [12, 21, 40, 85])
@pytest.mark.parametrize("new,kv", [(1, 200), (1, 5000), (30, 200), (64, 3000)])
def test_rows_with_large_scores_leave_the_others_alone(new, kv, size):
    c = Case(kv, new, 128, "bf16", heads=2, seed=70)
    q = torch.randn(new, 8, 128, generator=c.gen).bfloat16()
    want = c.cache.attention(c.batch, q.cuda(), lse=True)
    q[:, 1::4] *= 2.0 ** size
    q[new // 2:, 6] *= -2.0 ** size
    got = c.cache.attention(c.batch, q.cuda(), lse=True)
    assert all(torch.isfinite(t).all() for t in got)
    keep = torch.ones(new, 8, dtype=torch.bool)
    keep[:, 1::4] = False
    keep[new // 2:, 6] = False
    for a, b in zip(got, want):
        assert torch.equal(a[keep], b[keep])
