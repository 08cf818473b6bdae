"""Operands whose gradient or tangent would be lost: every operand of every operator, in both modes."""
import pytest
import torch
from torch.autograd import forward_ad

pytestmark = pytest.mark.gpu


def _calls():
    """name -> (operator, operands)."""
    from paper_2609_02109_amd import serve
    gen = torch.Generator().manual_seed(1)
    draw = lambda *s: torch.randn(*s, generator=gen).bfloat16().cuda()
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32).cuda()
    x = dict(x=draw(2, 64), y=draw(2, 64), weight=draw(64), bias=draw(32), wide=draw(2, 3, 64))
    codes, scales = torch.ones(32, 64, dtype=torch.int8, device="cuda"), torch.ones(32, device="cuda")
    codes4, scales4 = torch.zeros(32, 32, dtype=torch.uint8, device="cuda"), draw(32, 1)
    w8, w4 = serve.W8Weight(codes, scales), serve.W4Weight(codes4, scales4)
    rows = (torch.ones(2, 64, dtype=torch.int8, device="cuda"), torch.ones(2, device="cuda"))
    k, v, q = draw(2, 1, 64), draw(2, 1, 64), draw(2, 4, 64)
    cos, sin = serve.rope_table(16, 64)
    calls = {
        "quantise": (lambda x: serve.quantise_rows(x), dict(x=x["x"])),
        "quantise in three dims": (lambda x: serve.quantise_rows(x), dict(x=x["wide"])),
        "norm": (lambda x, weight: serve.norm_rows(x, weight), dict(x=x["x"], weight=x["weight"])),
        "norm with a residual": (lambda x, weight, y: serve.norm_rows(x, weight, residual=y), dict(x=x["x"], weight=x["weight"], y=x["y"])),
        "gate": (lambda x, y: serve.gate_rows(x, y), dict(x=x["x"], y=x["y"])),
        "values": (lambda scales: serve.Rows8(rows[0], scales).values(), dict(scales=rows[1])),
        "8-bit weight": (lambda scales: serve.W8Weight(codes, scales), dict(scales=scales)),
        "8-bit product": (lambda x, bias: w8.matmul(x, bias=bias), dict(x=x["x"], bias=x["bias"])),
        "8-bit product of codes": (lambda scales: w8.matmul((rows[0], scales)), dict(scales=rows[1])),
        "4-bit weight": (lambda scales: serve.W4Weight(codes4, scales), dict(scales=scales4)),
        "4-bit product": (lambda x, bias: w4.matmul(x, bias=bias), dict(x=x["x"], bias=x["bias"])),
    }
    for kind, cache in (("4-bit", serve.KV4Cache(1, 16, 1, 64)), ("8-bit", serve.KV8Cache(1, 16, 1, 64))):
        cache.pages.zero_()
        batch = cache.batch(i32(0, 2), i32(2), i32(0).view(1, 1), 2, 2, 2)
        calls[kind + " append"] = (lambda k, v, q, cos, sin, c=cache, b=batch: c.append(b, k, v, cos=cos, sin=sin, q=q), dict(k=k, v=v, q=q, cos=cos, sin=sin))
        calls[kind + " attention"] = (lambda q, c=cache, b=batch: c.attention(b, q), dict(q=q))
    return calls


NAMES = ["quantise", "quantise in three dims", "norm", "norm with a residual", "gate", "values", "8-bit weight", "8-bit product", "8-bit product of codes",
         "4-bit weight", "4-bit product", "4-bit append", "4-bit attention", "8-bit append", "8-bit attention"]


@pytest.mark.parametrize("name", NAMES)
def test_every_operand(name):
    calls = _calls()
    assert list(sorted(calls)) == sorted(NAMES)
    call, operands = calls[name]
    call(**operands)
    for which, t in operands.items():
        with pytest.raises(ValueError, match="gradient"):
            call(**{**operands, which: t.clone().requires_grad_()})
        with torch.no_grad():
            call(**{**operands, which: t.clone().requires_grad_()})
        with forward_ad.dual_level():
            dual = forward_ad.make_dual(t, torch.ones_like(t))
            for guard in (torch.enable_grad(), torch.no_grad()):
                with guard, pytest.raises(ValueError, match="tangent"):
                    call(**{**operands, which: dual})
            call(**{**operands, which: dual.detach()})
            call(**operands)   # no tangents in a level are as no level
    torch.cuda.synchronize()


def test_outputs_of_the_caller():
    from paper_2609_02109_amd import serve
    x = torch.ones(2, 64, dtype=torch.bfloat16, device="cuda")
    with forward_ad.dual_level():
        out = forward_ad.make_dual(torch.zeros_like(x), torch.ones_like(x))
        with pytest.raises(ValueError, match="tangent"):
            serve.norm_rows(x, x[0], residual=x.clone(), out=out)
