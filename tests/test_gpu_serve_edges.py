"""The served steps' operators where what they hold is unusual: pages with
leftovers of other requests, values of all sizes, batches of many sequences, and
calls on other streams.

Tolerances, derived before the first run, with u the rounding unit of the result's
type (2^-8 bfloat16, 2^-11 binary16):
* attention: a softmax weight and its product with a token's scale are each rounded
  to binary16, 2^-11 of them, so an element is within
    u |o| + 2^-11 sum_t p_t (|v_t| + scale_t code_t) <= u |o| + 2^-10 sum_t p_t (|v_t| + |off_t|),
  plus 2^-13 sum_t p_t |v_t| for fp32 scores (2^-22 of products that sum to some
  hundred), and half of binary16's smallest step, 2^-25, where it is the result's type.
* products: with the codes 16 + c and the zero points 16 + z (at most 31) a group is two
  sums of at most 128 products, by matrix instructions of 32: five levels of sums and one
  onto the last, four times, and the group's own two operations, so at most 32 roundings of
  2^-24 (2^-23 where an instruction cuts off) each stand above any product:
  u |y| + 2^-18 31 sum |x| s, and 64 more of the sum so far, 2^-18 of max |sum| <= sum |x s (c - z)|.
"""
import gc
import math
import threading

import pytest
import torch

from test_gpu_serve import DT, SHAPES, UNIT, Case, _gen, _weights, plain_attention, serve  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def _parts(x, G):
    """What a row stands for in the cache and the size of its offset, [.., D] each, in fp32 step by step."""
    y = x.float().clamp(-65504, 65504).unflatten(-1, (-1, G))
    lo, hi = y.amin(-1, keepdim=True), y.amax(-1, keepdim=True)
    s = ((hi - lo) * torch.tensor(1 / 15.0, dtype=torch.float32)).half().float()
    o = lo.half().float()
    c = ((y - o) * torch.where(s > 0, 1.0 / s, torch.zeros_like(s))).round().clamp(0, 15)
    return (o + s * c).flatten(-2).double(), o.abs().expand(*y.shape).flatten(-2).double()


def check(c, per, q, got, lse=None, window=0, scale=None, kv=None, new=None):
    """got [rows, heads, D] against 64 bits, at the tolerance above."""
    kv, new = c.kv if kv is None else kv, c.new if new is None else new
    scale, at = 1 / math.sqrt(c.D) if scale is None else scale, 0
    for i, n in enumerate(new):
        if n and kv[i]:
            k, _ = _parts(c.k[i][: kv[i]], c.G)
            v, off = _parts(c.v[i][: kv[i]], c.G)
            o, l, p = plain_attention(q[at:at + n], k, v, per, n, window, scale)
            for h in range(q.shape[1]):
                mass, offs = p[:, h] @ v[:, h // per].abs(), p[:, h] @ off[:, h // per]
                tol = UNIT[c.dt] * o[:, h].abs() + 2.0 ** -10 * (mass + offs) + 2.0 ** -13 * mass + (2.0 ** -25 if c.dt == "f16" else 0) + 1e-30
                err = (got[at:at + n, h].cpu().double() - o[:, h]).abs()
                assert (err <= tol).all(), (i, h, float((err / tol).max()))
            if lse is not None:
                seen = torch.isfinite(l)
                assert torch.equal(torch.isfinite(lse[at:at + n].cpu()), seen) and ((lse[at:at + n].cpu().double() - l)[seen].abs() <= 1e-4).all()
        at += n


# ------------------------------------------------------- leftovers in the pages

# what pages hold before anything is written, as binary16: scales from the smallest to the largest, infinities, NaN
LEFTOVERS = [6e-8, 1e-3, 2.0, 100.0, 65504.0, float("inf"), float("nan")]


def _leave(cache, value):
    cache.pages.view(torch.float16).fill_(value)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("D,G", SHAPES)
@pytest.mark.parametrize("kv,new,per", [([90, 37, 20, 0], [1, 1, 1, 1], 4), ([90, 37, 21], [20, 7, 3], 2), ([2500, 37], [1, 1], 2), ([150], [60], 3)])
def test_attention_does_not_depend_on_leftovers(serve, D, G, dt, kv, new, per):
    """The rest of a sequence's last page, and pages that are none of the cache's: the same bits whatever the memory holds."""
    c = Case(serve, kv, new, heads=1, D=D, G=G, page=16 if kv[0] < 1000 else 64, dt=dt, seed=31)
    q = torch.randn(sum(new), per, D, generator=c.gen).to(DT[dt])
    bad = c.table.clone()
    bad[0, 1], bad[-1, 0] = -1, c.n_pages
    want = None
    for value in [0.0] + LEFTOVERS:
        _leave(c.cache, value)
        c.fill(1)
        got = [*c.cache.attention(c.batch(), q.cuda(), lse=True), *c.cache.attention(c.batch(table=bad), q.cuda(), lse=True)]
        if want is None:
            want = got
            check(c, per, q, *got[:2])
        assert all(torch.equal(a, b) for a, b in zip(got, want)), value


@pytest.mark.parametrize("new,per", [(1, 4), (5, 4), (20, 4)])
def test_attention_in_a_window_over_pages_that_were_given_back(serve, new, per):
    """Tokens before every row's window need not be there: their pages may be another's by now, or partly written."""
    c = Case(serve, [300], [new], heads=2, D=64, G=32, page=16, dt="bf16", seed=32)
    q = torch.randn(new, 2 * per, 64, generator=c.gen).bfloat16()
    tail = 24 + new - 1   # what the rows see
    want = None
    for value in [0.0] + LEFTOVERS:
        _leave(c.cache, value)
        c.cache.append(c.batch(new=[tail]), c.k[0][-tail:].cuda(), c.v[0][-tail:].cuda())
        got = c.cache.attention(c.batch(), q.cuda(), window=24)
        if want is None:
            want = got
            check(c, per, q, got, window=24)
        assert torch.equal(got, want), value


@pytest.mark.parametrize("big", [1e-6, 3e-3, 40.0, 3000.0])
def test_a_row_does_not_depend_on_later_tokens(serve, big):
    """Rows of a chunk before a token whose values are of another size: the same bits as without it."""
    for window in (0, 30):
        c = Case(serve, [100], [40], heads=1, D=128, G=64, page=32, dt="f16", seed=33)
        q = torch.randn(40, 2, 128, generator=c.gen).half()
        c.fill(1)
        want = c.cache.attention(c.batch(), q.cuda(), window=window)
        for pos in (71, 75, 90):
            c.v[0][pos] = (c.v[0][pos].float() * big).half()
        c.fill(1)
        got = c.cache.attention(c.batch(), q.cuda(), window=window)
        check(c, 2, q, got, window=window)
        assert torch.equal(got[:11], want[:11]) and not torch.equal(got[11:], want[11:])


# --------------------------------------------------------- values of all sizes

def _sink(c, at, powers, per):
    """Keys and queries for which token `at` weighs 2^powers times the others, which weigh about the same."""
    D = c.D
    q = torch.zeros(sum(c.new), per * c.heads, D)
    q[..., 0] = 1.0
    for k in c.k:
        k.copy_((k.float() * 0.01).to(k.dtype))
        k[:, :, 0] = 0.0
        if k.shape[0] > at:
            k[at, :, 0] = powers * math.log(2) * math.sqrt(D)
    return q.to(DT[c.dt])


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("size", [1.0, 0.05, 1e-2, 1e-3, 1e-4, 1e-5])
@pytest.mark.parametrize("kv,new,per", [([700], [1], 4), ([9000], [1], 2), ([1500], [40], 2)])
@pytest.mark.parametrize("powers", [11, 14])
def test_attention_of_small_values_beside_a_heavy_token(serve, size, dt, kv, new, per, powers):
    c = Case(serve, kv, new, heads=1, D=64, G=32, page=64, dt=dt, seed=34)
    q = _sink(c, 3, powers, per)
    for v in c.v:
        v.copy_((v.float() * size).to(v.dtype))
        v[3] = 0
    c.fill(1)
    out, lse = c.cache.attention(c.batch(), q.cuda(), lse=True)
    check(c, per, q, out, lse)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("kv,new,per", [([700], [1], 4), ([9000], [1], 2), ([1500], [40], 2)])
def test_attention_of_large_values(serve, dt, kv, new, per):
    """Values of 30 to binary16's largest, in some tokens and some groups only, the largest late; one heavy token before them."""
    for powers in (0, 10):
        c = Case(serve, kv, new, heads=1, D=128, G=32, page=64, dt=dt, seed=35)
        q = _sink(c, 3, powers, per)
        n = kv[0]
        for pos, size, dims in ((5, 30.0, slice(0, 32)), (n // 3, 700.0, slice(0, 128)), (n // 2, 9000.0, slice(64, 96)), (n - 50, 65504.0, slice(32, 64))):
            c.v[0][pos, :, dims] = ((c.v[0][pos, :, dims].float() * size).clamp(-65504, 65504)).to(DT[dt])
        c.v[0][n // 2:, :, 96:] = (c.v[0][n // 2:, :, 96:].float() * 1e-4).to(DT[dt])
        c.fill(1)
        out, lse = c.cache.attention(c.batch(), q.cuda(), lse=True)
        check(c, per, q, out, lse)


# ------------------------------------------------------------- many sequences

@pytest.mark.parametrize("n", [65, 128, 130])
def test_attention_of_many_sequences(serve, n):
    """Shares that go over more than 64 sequences, with empty ones where the lanes wrap round; heads that end inside shares."""
    gen = _gen(n)
    kv = [int(x) for x in torch.randint(1, 90, (n,), generator=gen)]
    new = [1] * n
    for i in (7, 63, 64, n - 1):
        kv[i] = 0
    if n > 65:
        kv[65] = 0
    kv[3], kv[n // 2], kv[n - 2] = 5000, 2600, 4400
    new[9] = new[62] = 0
    c = Case(serve, kv, new, heads=1, D=64, G=32, page=64, dt="bf16", seed=36)
    c.fill(1)
    q = torch.randn(sum(new), 3, 64, generator=c.gen).bfloat16()
    out, lse = c.cache.attention(c.batch(), q.cuda(), lse=True)
    check(c, 3, q, out, lse)
    empty = [sum(new[:i]) for i in range(n) if new[i] and not kv[i]]
    assert (out[empty] == 0).all() and (lse[empty] == -math.inf).all()
    out, lse = c.cache.attention(c.batch(), q.cuda(), lse=True, window=2000)
    check(c, 3, q, out, lse, window=2000)


def test_attention_of_a_chunk_beside_long_decodes(serve):
    """A batch of one prompt's chunk, single tokens over long contexts and drafts of nine."""
    c = Case(serve, [600, 9000, 5, 3333, 0, 800], [300, 1, 1, 9, 0, 1], heads=2, D=64, G=64, page=64, dt="f16", seed=37)
    c.fill(1)
    q = torch.randn(312, 4, 64, generator=c.gen).half()
    out, lse = c.cache.attention(c.batch(), q.cuda(), lse=True)
    check(c, 2, q, out, lse)


# ------------------------------------------------------------------- products

def _check_w4(y, x, w, scales, g, dt):
    """y against 64 bits, at the tolerance above; -> the same as a truth value, for a y that is off."""
    x, at = x.double(), torch.arange(w.shape[1]) // g
    want = x @ w.T
    tol = UNIT[dt] * want.abs() + 2.0 ** -18 * (31 * (x.abs() @ scales.double().abs()[:, at].T) + x.abs() @ w.abs().T)
    return bool(((y.cpu().double() - want).abs() <= tol).all())


W4_LONG = [(1, 40, 16384, 128), (16, 24, 16384, 128), (1, 33, 8224, 32), (16, 17, 10272, 32), (1, 20, 9536, 64), (16, 48, 12352, 64), (5, 31, 8704, 128),
           (3, 5003, 4128, 32), (20, 200, 8256, 64), (40, 100, 12320, 32), (64, 130, 16384, 128)]


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("m,n,k,g", W4_LONG)
def test_w4_over_many_inputs(serve, m, n, k, g, dt):
    """Every group of the inputs counts: the bound tells a product that lacks any one of them (planted in the plain form)."""
    codes, scales, z, w = _weights(n, k, g, DT[dt], True, m + n + k)
    x = torch.randn(m, k, generator=_gen(38)).to(DT[dt])
    whole = x.double() @ w.T
    for i in range(0, k, g):
        assert not _check_w4(whole - x[:, i:i + g].double() @ w[:, i:i + g].T, x, w, scales, g, dt), i
    assert _check_w4(serve.W4Weight(codes.cuda(), scales.cuda(), z.cuda()).matmul(x.cuda()), x, w, scales, g, dt)


# -------------------------------------------------------------------- streams

def _busy():
    """Some tenths of a second of work on the current stream."""
    a = torch.ones(8192, 8192, device="cuda")
    for _ in range(40):
        a = (a @ a).clamp_(0, 1)
    return a


def test_copies_run_on_the_stream_of_the_call(serve):
    """What is not contiguous is copied within a call: on its stream, not on the current one, which is busy."""
    n, k, g = 80, 256, 64
    codes, scales, z, _ = _weights(n, k, g, torch.bfloat16, True, 39)
    codes, scales, z = codes.cuda(), scales.cuda(), z.cuda()
    turned = [t.t().contiguous().t() for t in (codes, scales, z)]
    xt = torch.randn(k, 40, generator=_gen(40)).bfloat16().cuda()
    x3 = torch.randn(3, k, 5, generator=_gen(41)).bfloat16().cuda().transpose(1, 2)
    c = Case(serve, [3000, 40], [2, 1], heads=2, D=64, G=32, page=16, dt="bf16", seed=42)
    c.fill(1)
    b, cos, sin = c.batch(), *serve.rope_table(3008, 64)
    rows = [torch.randn(3, h, 64, 2, generator=c.gen).bfloat16().cuda()[..., 0] for h in (2, 2, 8)]

    def calls(stream):
        w = serve.W4Weight(*turned, stream=stream)
        y = w.matmul(xt.t(), stream=stream)
        y3 = w.matmul(x3, stream=stream)
        q = c.cache.append(b, rows[0], rows[1], cos=cos, sin=sin, q=rows[2], stream=stream)
        o, ls = c.cache.attention(b, rows[2], lse=True, stream=stream)
        return [w.packed, y, y3, q, o, ls, *c.cache.read(b, stream=stream)]

    W = serve.W4Weight(codes, scales, z)
    want = calls(None)
    assert torch.equal(want[0], W.packed) and torch.equal(want[1], W.matmul(xt.t().contiguous()))
    main, side = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(main):
        for _ in range(3):
            # what the caching allocator hands out next on `main` is still being written there
            freed = [torch.full_like(t, 3) for t in want for _ in range(2)]
            busy = _busy()
            for t in freed:
                t.fill_(7)
            del freed, t
            got = calls(side)
            side.synchronize()
            copies = [t.cpu() for t in got]   # on `main`, after what is under way there
            main.synchronize()
            assert all(torch.equal(a, b.cpu()) for a, b in zip(copies, want))
            del busy


def test_results_of_another_stream_outlive_it(serve):
    """A result is not handed out again while the caller's stream still reads it."""
    codes, scales, z, _ = _weights(4096, 256, 64, torch.bfloat16, True, 43)
    W = serve.W4Weight(codes.cuda(), scales.cuda(), z.cuda())
    x = torch.randn(64, 256, generator=_gen(44)).bfloat16().cuda()
    want, side = W.matmul(x), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        y = W.matmul(x, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        busy = _busy()
        kept = y.clone()   # after the work above
        del y
        for _ in range(4):
            W.matmul(-x, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(kept, want)
        del busy


def test_operands_that_require_a_gradient_are_refused(serve):
    codes, scales, z, _ = _weights(64, 128, 64, torch.bfloat16, True, 45)
    W = serve.W4Weight(codes.cuda(), scales.cuda(), z.cuda())
    c = Case(serve, [20], [2], heads=2, D=64, G=32, dt="bf16", seed=46)
    c.fill(1)
    b, (cos, sin) = c.batch(), serve.rope_table(32, 64)
    plain = lambda *shape: torch.randn(*shape, generator=c.gen).bfloat16().cuda()
    x, bias, k, q = plain(3, 128), plain(64), plain(2, 2, 64), plain(2, 4, 64)
    asked = lambda t: t.clone().requires_grad_()
    calls = [lambda f: W.matmul(f(x)), lambda f: W.matmul(x, bias=f(bias)), lambda f: W.matmul(f(x)[0]), lambda f: c.cache.append(b, f(k), k),
             lambda f: c.cache.append(b, k, f(k)), lambda f: c.cache.append(b, k, k, cos=cos, sin=sin, q=f(q)), lambda f: c.cache.attention(b, f(q))]
    for call in calls:
        with pytest.raises(ValueError):
            call(asked)
        want = call(lambda t: t)
        with torch.no_grad():
            got = call(asked)
        assert want is got is None or torch.equal(got, want)


def test_a_window_past_32_bits_is_refused(serve):
    c = Case(serve, [40], [1], heads=1, D=64, G=32, dt="bf16", seed=47)
    c.fill(1)
    q = torch.randn(1, 1, 64, generator=c.gen).bfloat16().cuda()
    for window in (2 ** 32, 2 ** 32 + 5, -2 ** 32 + 5, 2 ** 31):
        with pytest.raises(ValueError):
            c.cache.attention(c.batch(), q, window=window)
    assert torch.equal(c.cache.attention(c.batch(), q, window=2 ** 31 - 1), c.cache.attention(c.batch(), q))


def test_a_thread_hands_its_workspaces_back(serve):
    """Calls of threads that end leave nothing behind; the thread that goes on keeps its own."""
    c = Case(serve, [3000, 2500], [1, 1], heads=2, D=64, G=32, page=16, dt="bf16", seed=48)
    c.fill(1)
    q, b = torch.randn(2, 4, 64, generator=c.gen).bfloat16().cuda(), c.batch()
    want = c.cache.attention(b, q)
    assert max(b._ws_bytes.values()) > 0
    torch.cuda.synchronize()
    before, got = torch.cuda.memory_allocated(), []
    for _ in range(8):
        t = threading.Thread(target=lambda: got.append(torch.equal(c.cache.attention(b, q), want)))
        t.start()
        t.join()
    gc.collect()
    assert got == [True] * 8 and torch.cuda.memory_allocated() == before


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("kv,new,per", [([90, 37], [1, 1], 4), ([2500, 37], [1, 1], 2), ([150], [60], 3)])
def test_attention_of_tiny_queries_and_scales(serve, dt, kv, new, per):
    """Scores that are all nearly the same, up to queries of zero and the smallest scales: every token weighs alike."""
    c = Case(serve, kv, new, heads=1, D=64, G=32, page=16, dt=dt, seed=49)
    c.fill(1)
    q = torch.randn(sum(new), per, 64, generator=c.gen).to(DT[dt])
    for x, scale in ((q * 0, 0.125), (q * 0, 1e-12), (q * 0, 1e-38), (q, 1e-12), (q, 1e-38), (q, 1e-45), (q * 2.0 ** -12, 1e-30)):
        out, lse = c.cache.attention(c.batch(), x.cuda(), lse=True, scale=scale)
        check(c, per, x, out, lse, scale=scale)


@pytest.mark.parametrize("seed", range(12))
def test_attention_of_values_of_any_size(serve, seed):
    """Every token and group of its own size, 2^-20 to 2^15, some of zeros, under sharp and flat weights: as above, and
    half of the smallest weight that is held, 2^-35 of a row's largest."""
    gen = _gen(1000 + seed)
    pick = lambda *v: v[int(torch.randint(0, len(v), (1,), generator=gen))]
    D, G = SHAPES[seed % len(SHAPES)]
    kv, new, per = pick(([700, 33], [1, 2], 4), ([5000, 40], [1, 1], 2), ([300, 64], [40, 9], 3))
    c = Case(serve, kv, new, heads=2, D=D, G=G, page=pick(16, 64), dt=pick("bf16", "f16"), seed=50 + seed)
    for v in c.v:
        size = 2.0 ** (35 * torch.rand(*v.shape[:2], D // G, generator=gen) - 20) * (torch.rand(*v.shape[:2], D // G, generator=gen) > 0.1)
        v.copy_((v.float().clamp(-2, 2).unflatten(-1, (-1, G)) / 2 * size[..., None]).flatten(-2).to(v.dtype))
    c.fill(pick(1, 2))
    q = (pick(0.1, 1.0, 4.0) * torch.randn(sum(new), 2 * per, D, generator=gen)).to(DT[c.dt])
    window = pick(0, 0, 100)
    out = c.cache.attention(c.batch(), q.cuda(), window=window).cpu().double()
    at = 0
    for i, n in enumerate(new):
        k, _ = _parts(c.k[i], G)
        v, off = _parts(c.v[i], G)
        o, _, p = plain_attention(q[at:at + n], k, v, per, n, window, 1 / math.sqrt(D))
        for h in range(2 * per):
            mass, offs, top = p[:, h] @ v[:, h // per].abs(), p[:, h] @ off[:, h // per], p[:, h].amax(-1, keepdim=True)
            floor = 2.0 ** -35 * top * ((p[:, h] > 0).double() @ (v[:, h // per].abs() + off[:, h // per]))
            tol = UNIT[c.dt] * o[:, h].abs() + 2.0 ** -10 * (mass + offs) + 2.0 ** -13 * mass + floor + (2.0 ** -25 if c.dt == "f16" else 0) + 1e-30
            err = (out[at:at + n, h] - o[:, h]).abs()
            assert (err <= tol).all(), (i, h, float((err / tol).max()))
        at += n
