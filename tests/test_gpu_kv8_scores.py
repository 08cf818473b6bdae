"""Attention over the 8-bit cache where scores are large: results are numbers, and the ones that the formula has.

What is expected, and how far off it may be: keys and queries have one dim that is not 0, so a score is one
product.  Tokens of the largest score have the same key in blocks of the same scale, hence the same score bit for
bit, and lead the others by 0.25 S > 2^17 (in powers of two), where every other weight is 0.  So a row's
result is the mean of those tokens' values as they are held (blocks of values have one scale), with weights that
are rounded to binary16 once (2^-11) and their sum in fp32:
    u |o| + (2^-11 + 2^-20) mean |v|,   u the rounding unit of the result's type,
and lse = score + log(number) to 2^-20 of itself (key scale, factor, score and sum: four roundings of 2^-24) and 2^-16.
"""
import math

import pytest
import torch

from test_gpu_kv8 import DT, UNIT, Case, serve  # noqa: F401

pytestmark = pytest.mark.gpu

# new tokens, query heads to a key head, tokens: whole heads by tokens, by shares, rows, rows in parts
FORMS = [(1, 4, 200), (1, 4, 5000), (30, 3, 200), (64, 4, 3000)]


def _case(serve, new, per, kv, D, dt, keys, seed):
    """keys [tokens]: what dim 0 of every key is."""
    c = Case(serve, [kv], [new], heads=1, D=D, page=64, dt=dt, seed=seed)
    c.k[0] = torch.zeros(kv, 1, D).to(DT[dt])
    c.k[0][:, 0, 0] = keys.to(DT[dt])
    c.v[0] = c.v[0].clamp(-3.5, 3.5)
    c.v[0][:, 0, 0] = 4.0   # every block's largest
    c.fill(1)
    return c


def _check(c, q, top, scale, per):
    """top [tokens]: those of the largest score."""
    new, kv = c.new[0], c.kv[0]
    out, lse = (t.cpu().double() for t in c.cache.attention(c.batch(), q.cuda(), scale=scale, lse=True))
    key, value = c.hk[0].values(kv).double()[:, 0, 0], c.hv[0].values(kv).double()[:, 0]
    unit = UNIT[c.dt]
    for i in range(new):
        seen = top & (torch.arange(kv) <= kv - new + i)
        n = int(seen.sum())
        want, room = value[seen].mean(0), value[seen].abs().mean(0)
        assert ((out[i] - want).abs() <= unit * want.abs() + (2.0 ** -11 + 2.0 ** -20) * room).all(), (i, out[i, 0, :4], want[:4])
        s = scale * q[i, :, 0].double() * key[seen][0] + math.log(n)
        assert ((lse[i] - s).abs() <= 2.0 ** -16 + 2.0 ** -20 * s.abs()).all(), (i, lse[i], s)


def _tops(kv, gen):
    top = torch.rand(kv, generator=gen) < 0.05
    top[3] = True
    top[15::16] = top[-1] = False   # of the others there is one to a block
    return top


@pytest.mark.parametrize("dt,D,size", [("bf16", 64, 20), ("f16", 128, 20), ("bf16", 128, 27), ("f16", 64, 27), ("bf16", 256, 27), ("bf16", 128, 40),
                                       ("f16", 256, 40), ("bf16", 64, 103), ("bf16", 256, 103)])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("new,per,kv", FORMS)
def test_large_scores(serve, new, per, kv, sign, dt, D, size):
    gen = torch.Generator().manual_seed(size)
    top = _tops(kv, gen)
    others = torch.rand(kv, generator=gen) * (1.5 if sign > 0 else 0.5)
    keys = torch.where(top, 1.0, others - 1.0) if sign > 0 else torch.where(top, 0.25, others + 0.5)
    keys[15::16] = keys[-1] = -1.0 if sign > 0 else 1.0
    most = 2.0 ** 15 if size > 100 else 1.0
    c = _case(serve, new, per, kv, D, dt, keys * most, seed=50 + size)
    # scale times the query stays below 2^90
    big = 2.0 ** (min(size, 88) if dt == "bf16" else 10)
    q = torch.zeros(new, per, D)
    q[..., 0] = sign * big
    _check(c, q.to(DT[dt]), top, 2.0 ** size / most / big, per)


@pytest.mark.parametrize("size", [21, 27, 40, 80])
@pytest.mark.parametrize("new,per,kv", FORMS)
def test_large_scores_then_small_ones(serve, new, per, kv, size):
    """The first half's scores are far below the rest's, which are 0."""
    keys = torch.zeros(kv)
    keys[:kv // 32 * 16] = 1.0
    c = _case(serve, new, per, kv, 128, "bf16", keys, seed=60)
    q = torch.zeros(new, per, 128)
    q[..., 0] = -2.0 ** size
    _check(c, q.bfloat16(), keys == 0, 1.0, per)


@pytest.mark.parametrize("size", [12, 21, 40, 85])
@pytest.mark.parametrize("new,kv", [(1, 200), (1, 5000), (30, 200), (64, 3000)])
def test_rows_with_large_scores_leave_the_others_alone(serve, new, kv, size):
    c = Case(serve, [kv], [new], heads=2, D=128, page=64, dt="bf16", seed=70)
    c.fill(1)
    q = torch.randn(new, 8, 128, generator=c.gen).bfloat16()
    want = c.cache.attention(c.batch(), q.cuda(), lse=True)
    q[:, 1::4] *= 2.0 ** size
    q[new // 2:, 6] *= -2.0 ** size
    got = c.cache.attention(c.batch(), q.cuda(), lse=True)
    assert all(torch.isfinite(t).all() for t in got)
    keep = torch.ones(new, 8, dtype=torch.bool)
    keep[:, 1::4] = False
    keep[new // 2:, 6] = False
    for a, b in zip(got, want):
        assert torch.equal(a[keep], b[keep])
