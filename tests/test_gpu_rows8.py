"""Rows in 8 bits (the norm with the residual's addition, the gate, rows as they
are) and the products of them with 8-bit weights, against plain implementations
in 64 bits.

Tolerances, derived before the first run, with u the rounding unit of the
result's type (2^-8 bfloat16, 2^-11 binary16) and e = 2^-24, fp32's:
* rows as they are: the definition's fp32 steps, so codes and scales are equal.
* norm: a thread adds up to 128 squares in a row, then ten levels of sums, so the
  sum is within 2 (128 + 10) e of itself, its root within half of that; with three
  products more, y is within 150 e < 2^-16 of itself and so is the scale.  The value
  is then within half a code and 127 * 2 * 2^-16 of one.
* gate: the exponent is rounded by |g| e, four operations more: below 2^-16 for |g| <= 200.
* products: the sum is exact; its conversion, two products and the bias's addition
  are off by at most 4 e of the larger terms, and the result is rounded once.  Half a
  step is u |y| down to the type's smallest normal number; below it steps are even,
  2^-24 in binary16, so that half of one is 2^-25 there (bfloat16's are below all of this).
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}
E = 2.0 ** -24


@pytest.fixture(scope="module")
def serve():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2609_02109_amd import serve as m
    return m


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def quantised(y):
    """The definition, in fp32 step by step: codes and scales."""
    scale = y.abs().amax(-1) * torch.tensor(1.0 / 127.0, dtype=torch.float32)
    scale = torch.where(scale < 2.0 ** -126, torch.zeros_like(scale), scale)
    inv = torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))
    return (y * inv[..., None]).round().clamp(-127, 127).to(torch.int8), scale


def _near(rows, y, off=2.0 ** -16):
    """Whether rows stand for y (64 bits), whose computation is off by `off` of itself."""
    top = y.abs().amax(-1)
    scales, codes = rows.scales.cpu().double(), rows.codes.cpu().double()
    assert ((scales - top / 127).abs() <= (off + 4 * E) * top / 127).all()
    assert ((codes * scales[..., None] - y).abs() <= (0.5 + 127 * 2 * off + 127 * 4 * E) * scales[..., None] + 1e-300).all()
    assert int(codes.abs().max()) <= 127


# one value, odd widths, the ends of every number of threads and values that a row is laid out with
WIDTHS = [1, 7, 8, 509, 512, 513, 1024, 1031, 2048, 2050, 4096, 4099, 8192, 8201, 16384, 16390, 65536, 65537, 131072]


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("n", WIDTHS)
def test_rows_as_they_are(serve, n, dt):
    x = (torch.randn(5, n, generator=_gen(n)) * 3).to(DT[dt])
    rows = serve.quantise_rows(x.cuda())
    codes, scales = quantised(x.float())
    assert torch.equal(rows.scales.cpu(), scales) and torch.equal(rows.codes.cpu(), codes)
    for ty in (torch.float32, DT[dt]):
        assert torch.equal(rows.values(ty).cpu(), (codes.float() * scales[:, None]).to(ty))


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("n", WIDTHS)
def test_norm(serve, n, dt):
    gen = _gen(n + 1)
    x, r = ((torch.randn(6, n, generator=gen) * 2).to(DT[dt]) for _ in range(2))
    w = (1 + 0.3 * torch.randn(n, generator=gen)).to(DT[dt])
    rows, h = serve.norm_rows(x.cuda(), w.cuda(), residual=r.cuda(), eps=1e-5)
    want = (x.float() + r.float()).to(DT[dt])
    assert torch.equal(h.cpu(), want)
    norm = lambda v: v.double() / torch.sqrt(v.double().square().mean(-1, keepdim=True) + 1e-5) * w.double()
    _near(rows, norm(want))
    alone, same = serve.norm_rows(x.cuda(), w.cuda(), eps=1e-5)
    _near(alone, norm(x))
    assert torch.equal(same.cpu(), x)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("n", WIDTHS)
def test_gate(serve, n, dt):
    both = torch.randn(4, 2 * n, generator=_gen(n + 2)) * 4
    both[:, 0] = 150.0
    both[:, n - 1] -= 160.0
    both = both.to(DT[dt]).cuda()
    rows = serve.gate_rows(both[:, :n], both[:, n:])
    g, u = both[:, :n].cpu().double(), both[:, n:].cpu().double()
    _near(rows, g * torch.sigmoid(g) * u)


def test_rows_of_all_kinds(serve):
    # zeros; one value; the smallest and the largest of the type; an infinity or a NaN in one place
    for dt in (torch.bfloat16, torch.float16):
        tiny, huge = torch.finfo(dt).smallest_normal, torch.finfo(dt).max
        x = torch.zeros(9, 300, dtype=dt)
        x[1, 17] = -1.0
        x[2, 5], x[2, 6] = tiny, -tiny / 2
        x[3] = huge
        x[4, 299], x[5, 0], x[6, 8] = float("inf"), float("-inf"), float("nan")
        x[7] = torch.arange(300) - 150.0
        rows = serve.quantise_rows(x.cuda())
        good = [0, 1, 2, 3, 7, 8]
        codes, scales = quantised(x[good].float())
        assert torch.equal(rows.codes[good].cpu(), codes) and torch.equal(rows.scales[good].cpu(), scales)
        assert torch.isnan(rows.scales[[4, 5, 6]]).all() and (rows.codes[[4, 5, 6]] == 0).all()
        assert torch.isnan(rows.values()[4:7]).all()
        w = torch.ones(300, dtype=dt).cuda()
        rows, _ = serve.norm_rows(x.cuda(), w)
        assert torch.isnan(rows.scales[[4, 5, 6]]).all() and (rows.codes[[4, 5, 6]] == 0).all()
        assert (rows.scales[0] == 0) and (rows.codes[0] == 0).all()
        assert torch.isnan(rows.scales[3]) if dt is torch.bfloat16 else (rows.codes[3] == 127).all()   # squares past fp32
        rows = serve.gate_rows(x.cuda(), torch.ones_like(x).cuda())
        assert torch.isnan(rows.scales[[4, 5, 6]]).all() and torch.isfinite(rows.scales[good]).all()


@pytest.mark.parametrize("n", [24, 777, 3001, 20000])
def test_rows_inside_wider_ones(serve, n):
    # rows that are 2-byte aligned only, NaN between them; leading dimensions; the sum over the residual or over x
    gen = _gen(n)
    wide = torch.full((2, 3, n + 5), float("nan"), dtype=torch.bfloat16)
    x = torch.randn(2, 3, n, generator=gen).bfloat16()
    wide[..., 3:3 + n] = x
    wide = wide.cuda()
    view = wide[..., 3:3 + n]
    codes, scales = quantised(x.float())
    rows = serve.quantise_rows(view)
    assert rows.codes.shape == x.shape and torch.equal(rows.codes.cpu(), codes) and torch.equal(rows.scales.cpu(), scales)
    assert torch.equal(serve.quantise_rows(x.cuda().transpose(0, 1)).codes.cpu(), codes.transpose(0, 1))
    r = torch.randn(6, n, generator=gen).bfloat16()
    w = torch.randn(n, generator=gen).bfloat16().cuda()
    want, h = serve.norm_rows(x.cuda().view(6, n), w, residual=r.cuda())
    for over in ("residual", "x", "neither"):
        a, b = wide.clone().view(6, n + 5), torch.full((6, n + 9), 7.0, dtype=torch.bfloat16, device="cuda")
        av, bv = a[:, 3:3 + n], b[:, 1:1 + n]
        bv.copy_(r)
        out = dict(residual=bv, x=av, neither=torch.full((6, n + 2), 5.0, dtype=torch.bfloat16, device="cuda")[:, 1:1 + n])[over]
        got, back = serve.norm_rows(av, w, residual=bv, out=out)
        assert back is out and torch.equal(out, h) and torch.equal(got.codes, want.codes) and torch.equal(got.scales, want.scales)
        assert (b[:, 0] == 7).all() and (b[:, 1 + n:] == 7).all() and torch.isnan(a[:, :3]).all() and torch.isnan(a[:, 3 + n:]).all()


def test_many_rows_and_none(serve):
    x = torch.randn(200_003, 8, generator=_gen(3)).bfloat16()
    codes, scales = quantised(x.float())
    rows = serve.quantise_rows(x.cuda())
    assert torch.equal(rows.codes.cpu(), codes) and torch.equal(rows.scales.cpu(), scales)
    assert torch.equal(rows.values().cpu(), codes.float() * scales[:, None])
    none = serve.quantise_rows(x[:0].cuda())
    assert none.codes.shape == (0, 8) and none.values().shape == (0, 8)
    one = serve.quantise_rows(x[0].cuda())
    assert torch.equal(one.codes.cpu(), codes[0]) and one.scales.shape == ()


def test_rows_refusals(serve):
    from paper_2609_02109_amd import mf
    x = torch.randn(4, 64).bfloat16().cuda()
    w, r = torch.ones(64, dtype=torch.bfloat16, device="cuda"), torch.zeros_like(x)
    for bad in (lambda: serve.quantise_rows(x.float()), lambda: serve.quantise_rows(x.cpu()), lambda: serve.quantise_rows(x[:, :0]),
                lambda: serve.quantise_rows(x.clone().requires_grad_()), lambda: serve.norm_rows(x, w[:32]), lambda: serve.norm_rows(x, w.half()),
                lambda: serve.norm_rows(x, w, residual=r[:2]), lambda: serve.norm_rows(x, w, residual=r.half()), lambda: serve.norm_rows(x, w, out=r),
                lambda: serve.norm_rows(x, w, residual=r, out=r[:2]), lambda: serve.norm_rows(x, w.clone().requires_grad_()),
                lambda: serve.gate_rows(x, x[:, :32]), lambda: serve.gate_rows(x, x.half()), lambda: serve.gate_rows(x, x.clone().requires_grad_()),
                lambda: serve.Rows8(x, w).values(), lambda: serve.quantise_rows(x).values(torch.int8),
                lambda: serve.Rows8(serve.quantise_rows(x).codes, torch.ones(3, device="cuda")).values()):
        with pytest.raises(ValueError):
            bad()
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(mf.MfError):
            serve.norm_rows(x, w, eps=eps)
    with pytest.raises(mf.MfError) as e:
        serve.quantise_rows(torch.zeros(1, 2 ** 17 + 1, dtype=torch.bfloat16, device="cuda"))
    assert e.value.status == mf.MF_EUNSUPPORTED


# --------------------------------------------------------------- products

def _weights(n, k, seed):
    gen = _gen(seed)
    codes = torch.randint(-128, 128, (n, k), generator=gen, dtype=torch.int8)
    return codes, (0.5 + torch.rand(n, generator=gen)) * 0.01


def _rows(m, k, seed):
    gen = _gen(seed)
    return torch.randint(-127, 128, (m, k), generator=gen, dtype=torch.int8), (0.5 + torch.rand(m, generator=gen)) * 0.02


def _check(y, codes, scales, wc, ws, bias, dt):
    part = (codes.double() @ wc.double().T) * scales.double()[:, None] * ws.double()
    want = part if bias is None else part + bias.double()
    tol = UNIT[dt] * want.abs() + 4 * E * (part.abs() + (0 if bias is None else bias.double().abs())) + (2.0 ** -25 if dt == "f16" else 1e-30)
    err = (y.cpu().double() - want).abs()
    assert (err <= tol).all(), float((err / tol).max())


SIZES = [(1, 16, 16), (1, 1, 64), (2, 17, 80), (3, 515, 160), (16, 64, 256), (17, 250, 400), (32, 1000, 1120), (33, 100, 576), (64, 4096, 512),
         (65, 48, 2048), (77, 333, 4112), (128, 128, 128), (129, 257, 144), (200, 33, 96), (300, 700, 1040), (5, 31, 16384), (16, 20000, 128),
         (513, 1025, 272), (4, 8, 131056),
         # the forms for many rows or outputs
         (20, 17000, 80), (4, 6000, 8192), (5, 300, 8208), (130, 5000, 400), (500, 4100, 272), (3000, 2500, 144), (4090, 4090, 208),
         (25, 5001, 272), (30, 4099, 144), (43, 6600, 368), (64, 4100, 4096), (512, 4093, 4096), (600, 5003, 272)]


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_product(serve, m, n, k, dt):
    wc, ws = _weights(n, k, m + n + k)
    xc, xs = _rows(m, k, m)
    bias = torch.randn(n, generator=_gen(1)).to(DT[dt]) if m % 3 else None
    W = serve.W8Weight(wc.cuda(), ws.cuda(), dtype=DT[dt])
    b = None if bias is None else bias.cuda()
    y = W.matmul(serve.Rows8(xc.cuda(), xs.cuda()), bias=b)
    assert y.dtype is DT[dt] and tuple(y.shape) == (m, n)
    _check(y, xc, xs, wc, ws, bias, dt)
    x = torch.randn(m, k, generator=_gen(2)).to(DT[dt])
    codes, scales = quantised(x.float())
    _check(W.matmul(x.cuda(), bias=b), codes, scales, wc, ws, bias, dt)


def test_sums_at_the_ends_of_32_bits(serve):
    k = 131056
    wc = torch.full((20, k), -128, dtype=torch.int8)
    wc[1::2] = 127
    xc = torch.full((70, k), -128, dtype=torch.int8)
    W = serve.W8Weight(wc.cuda(), torch.ones(20).cuda())
    for m in (1, 20, 70):
        _check(W.matmul(serve.Rows8(xc[:m].cuda(), torch.ones(m).cuda())), xc[:m], torch.ones(m), wc, torch.ones(20), None, "bf16")


@pytest.mark.parametrize("m", [1, 4, 20, 40, 150])
def test_product_strides_and_shapes(serve, m):
    n, k = 203, 416
    wc, ws = _weights(n, k, 3)
    W = serve.W8Weight(wc.cuda(), ws.cuda())
    xc, xs = _rows(2 * m, k, 4)
    # rows at any byte, others' codes between them; a result inside a larger one
    wide = torch.full((m, k + 7), 99, dtype=torch.int8)
    wide[:, 3:3 + k] = xc[:m]
    big = torch.full((m, n + 5), 7.0, dtype=torch.bfloat16, device="cuda")
    out = W.matmul(serve.Rows8(wide.cuda()[:, 3:3 + k], xs[:m].cuda()), out=big[:, 1:1 + n])
    assert out.data_ptr() == big[:, 1:].data_ptr()
    _check(out, xc[:m], xs[:m], wc, ws, None, "bf16")
    assert (big[:, 0] == 7).all() and (big[:, 1 + n:] == 7).all()
    y = W.matmul(serve.Rows8(xc.view(2, m, k).cuda(), xs.view(2, m).cuda()))
    assert tuple(y.shape) == (2, m, n)
    _check(y.view(2 * m, n), xc, xs, wc, ws, None, "bf16")
    assert torch.equal(W.matmul(serve.Rows8(xc.T.contiguous().cuda().T, xs.repeat(2, 1).T.cuda()[:, 0])), y.view(2 * m, n))
    x = torch.full((m, k + 3), float("nan"), dtype=torch.bfloat16)
    x[:, 1:1 + k] = torch.randn(m, k, generator=_gen(5)).bfloat16()
    codes, scales = quantised(x[:, 1:1 + k].float())
    _check(W.matmul(x.cuda()[:, 1:1 + k]), codes, scales, wc, ws, None, "bf16")
    assert tuple(W.matmul(torch.empty(0, k, dtype=torch.bfloat16, device="cuda")).shape) == (0, n)
    assert tuple(W.matmul(x[0, 1:1 + k].cuda()).shape) == (n,)
    assert torch.equal(W.matmul(serve.quantise_rows(x[0, 1:1 + k].cuda())), W.matmul(x[0, 1:1 + k].cuda()))


@pytest.mark.parametrize("m,k", [(1, 32768), (1, 32784), (2, 16384), (2, 16400), (3, 8192), (3, 8208), (3, 10912), (3, 10928), (4, 8192), (4, 8208), (4, 16), (3, 48), (2, 4112),
                                 (5, 4096), (8, 4096), (8, 4112), (7, 16), (6, 2000), (9, 4096)])
def test_rows_in_16_bits_up_to_what_a_product_takes(serve, m, k):
    wc, ws = _weights(37, k, 15)
    W = serve.W8Weight(wc.cuda(), ws.cuda())
    x = torch.randn(m, k, generator=_gen(16)).bfloat16()
    x[:, -1] = torch.arange(1, m + 1) * 20   # the largest, at the end
    codes, scales = quantised(x.float())
    _check(W.matmul(x.cuda()), codes, scales, wc, ws, None, "bf16")
    assert torch.equal(W.matmul(x.cuda()), W.matmul(serve.quantise_rows(x.cuda())))


@pytest.mark.parametrize("m", [1, 6, 40])
def test_outputs_beside_inputs_and_over_them(serve, m):
    from paper_2609_02109_amd import mf
    k = n = 160
    wc, ws = _weights(n, k, 13)
    W = serve.W8Weight(wc.cuda(), ws.cuda())
    x = torch.randn(m, k, generator=_gen(14)).bfloat16().cuda()
    w = torch.ones(k, dtype=torch.bfloat16, device="cuda")
    # inputs and outputs as the columns of one buffer
    both = torch.cat([x, torch.zeros_like(x)], 1)
    assert torch.equal(W.matmul(both[:, :k], out=both[:, k:]), W.matmul(x)) and torch.equal(both[:, :k], x)
    rows, h = serve.norm_rows(both[:, :k], w, residual=both[:, k:], out=both[:, k:])
    want = serve.norm_rows(x, w, residual=W.matmul(x))
    assert torch.equal(h, want[1]) and torch.equal(rows.codes, want[0].codes) and torch.equal(both[:, :k], x)
    # over the inputs, or a part of them
    for call in (lambda: W.matmul(both[:, :k], out=both[:, :k]), lambda: W.matmul(both[:, :k], out=both[:, 8:8 + k]),
                 lambda: serve.norm_rows(both[:, :k], w, residual=x, out=both[:, 8:8 + k])):
        with pytest.raises(mf.MfError) as e:
            call()
        assert e.value.status == mf.MF_EINVAL


@pytest.mark.parametrize("m", [5, 20, 90])
def test_rows_do_not_mix(serve, m):
    # a row with a NaN or an infinity is NaN, and the others are as without it
    wc, ws = _weights(70, 256, 6)
    W = serve.W8Weight(wc.cuda(), ws.cuda(), dtype=torch.float16)
    x = torch.randn(m, 256, generator=_gen(7)).half()
    clean = W.matmul(x.cuda())
    x[1, 17], x[m - 1, 0] = float("nan"), float("inf")
    y = W.matmul(x.cuda())
    rest = [i for i in range(m) if i not in (1, m - 1)]
    assert torch.isnan(y[[1, m - 1]]).all() and torch.equal(y[rest], clean[rest])


def test_product_refusals(serve):
    from paper_2609_02109_amd import mf
    wc, ws = (t.cuda() for t in _weights(32, 128, 8))
    W = serve.W8Weight(wc, ws)
    rows = serve.Rows8(torch.zeros(2, 128, dtype=torch.int8, device="cuda"), torch.ones(2, device="cuda"))
    x = torch.zeros(2, 128, dtype=torch.bfloat16, device="cuda")
    for bad in (lambda: serve.W8Weight(wc.cpu(), ws), lambda: serve.W8Weight(wc, ws.half()), lambda: serve.W8Weight(wc, ws[:16]),
                lambda: serve.W8Weight(wc.to(torch.uint8), ws), lambda: serve.W8Weight(wc, ws, dtype=torch.float32), lambda: W.matmul(x[:, :64]),
                lambda: W.matmul(x.half()), lambda: W.matmul(x.cpu()), lambda: W.matmul(rows.codes), lambda: W.matmul((rows.codes[:, :64], rows.scales)),
                lambda: W.matmul((rows.codes, rows.scales[:1])), lambda: W.matmul((rows.codes, rows.scales.half())),
                lambda: W.matmul(x, bias=torch.zeros(31, dtype=torch.bfloat16, device="cuda")), lambda: W.matmul(x, bias=torch.zeros(32, device="cuda")),
                lambda: W.matmul(x, out=torch.zeros(2, 31, dtype=torch.bfloat16, device="cuda")), lambda: W.matmul(x.clone().requires_grad_()),
                lambda: serve.W8Weight(wc, ws.clone().requires_grad_())):
        with pytest.raises(ValueError):
            bad()
    for k in (24, 131072):
        with pytest.raises(mf.MfError) as e:
            serve.W8Weight(torch.zeros(2, k, dtype=torch.int8, device="cuda"), torch.ones(2, device="cuda"))
        assert e.value.status == mf.MF_EUNSUPPORTED


def test_a_layer_in_a_graph(serve):
    """Norm, product, gate and product as a step runs them, on another stream, captured, and replayed beside eager calls."""
    gen = _gen(9)
    m, n, inner = 3, 512, 1040
    up, down = ((serve.W8Weight(c.cuda(), s.cuda())) for c, s in (_weights(2 * inner, n, 10), _weights(n, inner, 11)))
    w = torch.randn(n, generator=gen).bfloat16().cuda()

    def layer(x, r):
        rows, h = serve.norm_rows(x, w, residual=r)
        g = up.matmul(rows)
        return down.matmul(serve.gate_rows(g[:, :inner], g[:, inner:])), down.matmul(g[:, :inner]), h

    xs = [torch.randn(2, m, n, generator=gen).bfloat16().cuda() for _ in range(4)]
    want = [layer(*x) for x in xs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    x = xs[0].clone()
    with torch.cuda.stream(side):
        layer(*x)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = layer(*x)
    for i in (1, 2, 3, 0, 2):
        x.copy_(xs[i])
        graph.replay()
        other = layer(*xs[(i + 1) % 4])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want[i])) and all(torch.equal(a, b) for a, b in zip(other, want[(i + 1) % 4]))
    by_hand = torch.cuda.Stream()
    by_hand.wait_stream(torch.cuda.current_stream())
    rows, h = serve.norm_rows(*[xs[1][0], w], residual=xs[1][1], stream=by_hand)
    g = up.matmul(rows, stream=by_hand)
    y = down.matmul(serve.gate_rows(g[:, :inner], g[:, inner:], stream=by_hand), stream=by_hand)
    torch.cuda.current_stream().wait_stream(by_hand)
    assert torch.equal(y, want[1][0]) and torch.equal(h, want[1][2])


def test_a_norm_of_many_sizes_is_finite(serve):
    # sums stay in range up to where the type ends
    for scale in (2.0 ** -20, 1.0, 2.0 ** 12):
        x = (torch.randn(3, 1000, generator=_gen(12)) * scale).bfloat16()
        rows, _ = serve.norm_rows(x.cuda(), torch.ones(1000, dtype=torch.bfloat16, device="cuda"), eps=0.0)
        _near(rows, x.double() / x.double().square().mean(-1, keepdim=True).sqrt())
        assert math.isfinite(float(rows.scales.sum()))
