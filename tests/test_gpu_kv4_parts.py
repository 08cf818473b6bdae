"""Attention over the 4-bit cache by rows whose tokens are in parts: the bits that the parts' sum had when a workgroup
added up one row, whatever form it has now.  The digests are of the results of that form, for inputs that are made of whole
numbers (no generator of random numbers is in between)."""
import hashlib

import pytest
import torch

pytestmark = pytest.mark.gpu


def _drawn(seed, *shape):
    n = 1
    for d in shape:
        n *= d
    i = torch.arange(n, dtype=torch.int64) * 2654435761 + seed * 40503
    x = ((i ^ (i >> 15)) * 2246822519) % (1 << 32)
    return (((x >> 8) % 65536).float() / 16384 - 2).view(shape).bfloat16().cuda()


def _digest(n, kv, new, heads, kv_heads, D):
    from paper_2609_02109_amd import serve
    cols = -(-kv // 32)
    cache = serve.KV4Cache(n * cols, 32, kv_heads, D)
    table = torch.arange(n * cols, dtype=torch.int32).view(cols, n).t().contiguous().cuda()
    lens = torch.full((n,), kv, dtype=torch.int32).cuda()
    starts = torch.arange(n + 1, dtype=torch.int32).cuda()
    cache.append(cache.batch(starts * kv, lens, table, n * kv, kv, kv), _drawn(1, n * kv, kv_heads, D), _drawn(2, n * kv, kv_heads, D))
    out, lse = cache.attention(cache.batch(starts * new, lens, table, n * new, new, kv), _drawn(3, n * new, heads, D), lse=True)
    h = hashlib.sha256(out.cpu().view(torch.int16).numpy().tobytes())
    h.update(lse.cpu().numpy().tobytes())
    return h.hexdigest()[:16]


# parts: three, three, five, eight, sixteen, two; three of more rows
@pytest.mark.parametrize("size,want", [
    ((2, 3000, 64, 4, 1, 128), "561b1ac800f1be19"),
    ((1, 2500, 100, 2, 2, 64), "7a1ce99f2e3ff72d"),
    ((1, 5000, 40, 4, 1, 128), "22dd77a4361326b1"),
    ((1, 8000, 33, 2, 1, 128), "5a71d8a1f15af54f"),
    ((1, 16000, 40, 1, 1, 64), "1d7b9a85f2bc191d"),
    ((1, 2000, 70, 2, 1, 256), "9a9f394134203f11"),
    ((2, 2500, 64, 16, 4, 128), "fa0ebf0bf06d0971"),
    ((3, 3000, 64, 16, 4, 64), "32631d038010c5bd"),
    ((4, 3000, 64, 8, 2, 256), "1f8c84f94b38f3e3"),
])
def test_the_bits_of_parts_added_up(size, want):
    assert _digest(*size) == want
