"""A 4-bit variant's decode step out of its operators (`step.Decoder`) against
the same layers in 64 bits, and captured in a graph.

Tolerance, derived before the first run: a layer rounds ten tensors to bfloat16
(2^-9 of an element each at most), so the output is within
10 2^-9 = 2^-5.7 of its norm; 2^-5 is asked for.
"""
import math

import pytest
import torch

from test_gpu_serve import held, turned

pytestmark = pytest.mark.gpu


def _wide(codes, scales, zeros):
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(1).double()
    at = torch.arange(c.shape[1], device=c.device) // (c.shape[1] // scales.shape[1])
    return ((c - zeros.double()[:, at]) * scales.double()[:, at]).cpu()


def _norm(x):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)


def _plain(model, x, kv_group):
    """One layer over whole sequences x [n, tokens, width], in 64 bits but for the cache's codes, and rounded to
    bfloat16 where the operators are up to there: a code is a step function of what it is made from."""
    w = {n: _wide(*d) for n, d in model.drawn[0].items()}
    hq, hk, d, out = model.heads, model.kv_heads, model.head_dim, []
    for s in x.double():
        t = s.shape[0]
        qkv = (_norm(s).bfloat16().double() @ w["qkv"].T).bfloat16().double().view(t, hq + 2 * hk, d)
        cos, sin = model.cos[:t].cpu(), model.sin[:t].cpu()
        q = turned(qkv[:, :hq].float(), cos, sin, False).double()
        k = held(turned(qkv[:, hq:hq + hk].float(), cos, sin, False), kv_group).double().repeat_interleave(hq // hk, 1)
        v = held(qkv[:, hq + hk:].float(), kv_group).double().repeat_interleave(hq // hk, 1)
        sc = torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(d)
        sc = sc.masked_fill(torch.triu(torch.ones(t, t, dtype=torch.bool), 1), -math.inf)
        o = torch.einsum("hij,jhd->ihd", sc.softmax(-1), v).reshape(t, hq * d)
        s = s + o @ w["out"].T
        gate, up = (_norm(s) @ w["up"].T).chunk(2, -1)
        out.append(s + (gate * torch.sigmoid(gate) * up) @ w["down"].T)
    return torch.stack(out)


def test_a_prompt_and_steps_after_it():
    from paper_2609_02109_amd import step
    model = step.Decoder(2, 60, heads=4, kv_heads=2, head_dim=64, inner=512, group=64, kv_group=32, page=16)
    x = torch.randn(2, 60, 256, generator=torch.Generator().manual_seed(1)).bfloat16()
    want = _plain(model, x, 32)
    got = torch.empty_like(x)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32).cuda()
    got[:, :50] = model(model.batch(i32(0, 50, 100), i32(50, 50), 100, 50), x[:, :50].reshape(100, 256).cuda()).view(2, 50, 256).cpu()
    for t in range(50, 60):
        got[:, t] = model(model.batch(i32(0, 1, 2), i32(t + 1, t + 1), 2, 1), x[:, t].cuda()).cpu()
    err = (got.double() - want).norm(dim=-1) / want.norm(dim=-1)
    assert float(err.max()) < 2.0 ** -5


def test_options():
    from paper_2609_02109_amd import step
    got = step.options([1, 3], 100, steps=2, heads=4, kv_heads=2, head_dim=64, inner=512, group=64, kv_group=32, page=16)
    assert [o["concurrency"] for o in got] == [1, 3] and all(o["ms_per_step"] > 0 for o in got) and got[1]["gb"] > got[0]["gb"]


def test_a_captured_step_follows_the_lengths():
    from paper_2609_02109_amd import step
    model = step.Decoder(2, 60, layers=2, heads=4, kv_heads=2, head_dim=64, inner=512, group=64, kv_group=32, page=16)
    for c in model.caches:
        c.pages.zero_()
    start, kv = torch.arange(3, dtype=torch.int32).cuda(), torch.zeros(2, dtype=torch.int32).cuda()
    x = torch.zeros(2, 256, dtype=torch.bfloat16, device="cuda")
    batch = model.batch(start, kv, 2, 1)
    xs = torch.randn(5, 2, 256, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()

    def play(once):
        got = []
        for i in range(5):
            kv.fill_(i + 1)
            x.copy_(xs[i])
            got.append(once().clone())
            torch.cuda.synchronize()
        return torch.stack(got)

    want = play(lambda: model(batch, x))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        model(batch, x)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = model(batch, x)

    def replay():
        graph.replay()
        return out

    assert torch.equal(play(replay), want)
