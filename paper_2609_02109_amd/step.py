"""The decode step of a 4-bit variant, run and timed as an option.

The scheduler's options for a language model are variants x concurrency, each
with a latency, a throughput and the memory it holds.  `Decoder` is such a
model in its 4-bit variant, out of the operators in `serve`: per layer a
product for queries, keys and values, their append to the 4-bit cache with the
position rotation, attention over the cache, and the products after it.
`options` times a step at several concurrencies and returns one line per option;

    python -m paper_2609_02109_amd.step --context 2000 --concurrency 1,2,4

prints them.  Weights are drawn at random: what a step costs does not depend on them.
"""
from __future__ import annotations

import argparse

import torch

from . import serve


def _norm(x):
    y = x.float()
    return (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)


def draw_weight(n_out, n_in, group, dtype, gen, device):
    """Codes, scales and zero points of a random 4-bit weight [n_out, n_in]; outputs are about as large as inputs."""
    codes = torch.randint(0, 256, (n_out, n_in // 2), generator=gen, device=device, dtype=torch.uint8)
    # codes less 8 have a standard deviation of about 4.6
    scales = ((0.5 + torch.rand(n_out, n_in // group, generator=gen, device=device)) * (0.2 * n_in ** -0.5)).to(dtype)
    return codes, scales, torch.full(scales.shape, 8, device=device, dtype=torch.uint8)


class Decoder:
    """layers x (attention, gated products) over a cache that holds `seqs` sequences of up to `context` tokens."""

    def __init__(self, seqs, context, layers=1, heads=32, kv_heads=8, head_dim=128, inner=8192, group=128, kv_group=64, page=64,
                 dtype=torch.bfloat16, seed=0, device="cuda"):
        self.heads, self.kv_heads, self.head_dim, self.width, self.context = heads, kv_heads, head_dim, heads * head_dim, context
        self._shapes = dict(qkv=((heads + 2 * kv_heads) * head_dim, self.width), out=(self.width, heads * head_dim),
                            up=(2 * inner, self.width), down=(self.width, inner))
        self._drawn = (layers, group, dtype, seed, device)
        gen = torch.Generator(device=device).manual_seed(seed)
        self.layers = [{n: serve.W4Weight(*draw_weight(*s, group, dtype, gen, device)) for n, s in self._shapes.items()} for _ in range(layers)]
        cols = -(-context // page)
        self.caches = [serve.KV4Cache(seqs * cols, page, kv_heads, head_dim, group=kv_group, device=device) for _ in range(layers)]
        self.table = torch.randperm(seqs * cols, generator=gen, device=device).to(torch.int32).view(seqs, cols)
        self.cos, self.sin = serve.rope_table(cols * page, head_dim, device=device)

    @property
    def drawn(self):
        """Codes, scales and zero points of every layer's weights, drawn again: they are not held beside the laid out ones."""
        layers, group, dtype, seed, device = self._drawn
        gen = torch.Generator(device=device).manual_seed(seed)
        return [{n: draw_weight(*s, group, dtype, gen, device) for n, s in self._shapes.items()} for _ in range(layers)]

    @property
    def bytes(self):
        """Device memory of the weights as they are used, and of the caches."""
        return sum(w.packed.numel() for layer in self.layers for w in layer.values()) + sum(c.pages.numel() for c in self.caches)

    def batch(self, q_start, kv_len, rows, max_new, max_kv=None):
        return self.caches[0].batch(q_start, kv_len, self.table[: kv_len.shape[0]], rows, max_new, self.context if max_kv is None else max_kv)

    def __call__(self, batch, x):
        """x [rows, width], the batch's new tokens -> [rows, width]; their keys and values go into the caches."""
        hq, hk, d = self.heads, self.kv_heads, self.head_dim
        for w, cache in zip(self.layers, self.caches):
            qkv = w["qkv"].matmul(_norm(x)).view(x.shape[0], hq + 2 * hk, d)
            q = cache.append(batch, qkv[:, hq:hq + hk], qkv[:, hq + hk:], cos=self.cos, sin=self.sin, q=qkv[:, :hq], q_out=qkv[:, :hq])
            x = x + w["out"].matmul(cache.attention(batch, q).view(x.shape[0], hq * d))
            gate, up = w["up"].matmul(_norm(x)).chunk(2, -1)
            x = x + w["down"].matmul(torch.nn.functional.silu(gate.float()).mul(up.float()).to(x.dtype))
        return x


def _option(n, context, steps, decoder):
    model = Decoder(n, context, **decoder)
    for c in model.caches:
        c.pages.zero_()
    dev = model.table.device
    batch = model.batch(torch.arange(n + 1, dtype=torch.int32, device=dev), torch.full((n,), context, dtype=torch.int32, device=dev), n, 1)
    x = torch.randn(n, model.width, device=dev).to(model.layers[0]["qkv"].dtype)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        model(batch, x)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        model(batch, x)
    for _ in range(3):
        graph.replay()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(steps):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    ms = begin.elapsed_time(end) / steps
    return dict(variant="4-bit", concurrency=n, context=context, ms_per_step=ms, tokens_per_s=1e3 * n / ms, gb=model.bytes / 1e9)


def options(concurrency, context, steps=20, **decoder):
    """One dict per concurrency: ms a step (captured in a graph, all sequences at full context; torch's elementwise
    operations between the operators are part of it), tokens/s, GB.  One model at a time is on the device."""
    return [_option(n, context, steps, decoder) for n in concurrency]


def main(argv=None):
    p = argparse.ArgumentParser(description="options of a model's 4-bit variant: ms a step, tokens/s and memory by concurrency")
    p.add_argument("--concurrency", default="1,2,4", help="sequences that decode together, comma separated")
    p.add_argument("--context", type=int, default=2000, help="cached tokens of every sequence")
    p.add_argument("--layers", type=int, default=4)
    a = p.parse_args(argv)
    for o in options([int(c) for c in a.concurrency.split(",")], a.context, layers=a.layers):
        print(f"4-bit x{o['concurrency']}: {o['ms_per_step']:.3f} ms a step, {o['tokens_per_s']:.0f} tokens/s, {o['gb']:.2f} GB", flush=True)


if __name__ == "__main__":
    main()
