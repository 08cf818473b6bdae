"""The served steps' operators over batches and layers so wide that their work
does not fit one launch (2^32 threads): the results of narrower calls, bit for bit."""
import pytest
import torch

from test_gpu_serve import _gen, serve  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.as_tensor(x).to(torch.int32).cuda()


def _starts(new):
    return _i32(torch.cat((torch.zeros(1, dtype=torch.int64), torch.as_tensor(new).cumsum(0))))


def test_append_and_read_of_one_prompt_among_4096(serve):
    # 4096 sequences x 8 heads x 2049 blocks of a prompt of 32768: over 2^26 workgroups of 64
    n, long, heads = 4096, 32768, 8
    new = torch.ones(n, dtype=torch.int64)
    new[1234] = long
    rows = int(new.sum())
    table = torch.zeros(n, 32, dtype=torch.int32)
    table[:, 0] = torch.arange(n)
    table[1234, 1:] = torch.arange(n, n + 31)
    gen = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(rows, heads, 64, device="cuda", generator=gen, dtype=torch.bfloat16) for _ in range(2))
    start, kv, table = _starts(new), _i32(new), table.cuda()
    wide, narrow = (serve.KV4Cache(n + 31, 1024, heads, 64, group=64) for _ in range(2))
    wide.pages.zero_()
    narrow.pages.zero_()
    batch = wide.batch(start, kv, table, rows, long, long)
    wide.append(batch, k, v)
    # the others alone, then the prompt
    narrow.append(narrow.batch(start, torch.where(kv == 1, kv, torch.zeros_like(kv)), table, rows, 1, 1), k, v)
    narrow.append(narrow.batch(_i32([0, long]), _i32([long]), table[1234:1235], long, long, long), k[1234:1234 + long], v[1234:1234 + long])
    assert torch.equal(wide.pages, narrow.pages)
    one = narrow.read(narrow.batch(_i32([0, long]), _i32([long]), table[1234:1235], long, long, long), torch.bfloat16)
    got = wide.read(batch, torch.bfloat16)
    few = narrow.read(narrow.batch(_i32(range(101)), _i32([1] * 100), table[:100], 100, 1, 1), torch.bfloat16)
    for a, b, c in zip(got, one, few):
        assert torch.equal(a[1234:1234 + long], b) and torch.equal(a[:100], c) and a.abs().sum(-1).min() > 0


def test_append_and_read_of_a_million_sequences(serve):
    # 2^20 sequences x 128 heads: several launches; a row each of 64 of them
    n, heads = 2 ** 20, 128
    at = torch.randperm(n, generator=_gen(2))[:62].sort().values.tolist()
    at = [0] + [i for i in at if 0 < i < n - 1] + [n - 1]
    new = torch.zeros(n, dtype=torch.int64)
    new[at] = 1
    rows = len(at)
    table = torch.full((n, 1), -1, dtype=torch.int32)
    table[at, 0] = torch.arange(rows, dtype=torch.int32)
    k, v = (torch.randn(rows, heads, 64, generator=_gen(i)).half().cuda() for i in (3, 4))
    wide, narrow = (serve.KV4Cache(rows, 16, heads, 64, group=32) for _ in range(2))
    wide.pages.zero_()
    narrow.pages.zero_()
    batch = wide.batch(_starts(new), _i32(new), table.cuda(), rows, 1, 1)
    wide.append(batch, k, v)
    small = narrow.batch(_i32(range(rows + 1)), _i32([1] * rows), _i32(range(rows))[:, None], rows, 1, 1)
    narrow.append(small, k, v)
    assert torch.equal(wide.pages, narrow.pages)
    for a, b in zip(wide.read(batch), narrow.read(small)):
        assert torch.equal(a, b)


def test_attention_of_one_prompt_among_2048(serve):
    # 2048 sequences x 8 heads x 1025 tiles of a prompt of 32800 tokens of four heads: over 2^24 workgroups of 256
    n, long, heads, at = 2048, 32800, 8, 1500
    new = torch.ones(n, dtype=torch.int64)
    new[at] = long
    kv = torch.randint(1, 60, (n,), generator=_gen(5))
    kv[at] = long
    table = torch.zeros(n, 33, dtype=torch.int32)
    table[:, 0] = torch.arange(n)
    table[at, 1:] = torch.arange(n, n + 32)
    cache = serve.KV4Cache(n + 32, 1024, heads, 64, group=64)
    gen = torch.Generator(device="cuda").manual_seed(6)
    k, v = (torch.randn(int(kv.sum()), heads, 64, device="cuda", generator=gen, dtype=torch.bfloat16) for _ in range(2))
    table = table.cuda()
    cache.append(cache.batch(_starts(kv), _i32(kv), table, int(kv.sum()), long, long), k, v)
    rows = int(new.sum())
    q = torch.randn(rows, 4 * heads, 64, device="cuda", generator=gen, dtype=torch.bfloat16)
    out, lse = cache.attention(cache.batch(_starts(new), _i32(kv), table, rows, long, long), q, lse=True)
    one, ls = cache.attention(cache.batch(_i32([0, long]), _i32([long]), table[at:at + 1], long, long, long), q[at:at + long], lse=True)
    assert torch.equal(out[at:at + long], one) and torch.equal(lse[at:at + long], ls)
    # the single tokens as a batch of their own: other tiles, so roundings of the weights (2^-10 of values up to 5) and the result's
    few, ls = cache.attention(cache.batch(_i32(range(at + 1)), _i32(kv[:at]), table[:at], at, 1, 64), q[:at], lse=True)
    assert ((out[:at].float() - few.float()).abs() <= 2.0 ** -7 * few.float().abs() + 2.0 ** -9 * 5).all()
    assert ((lse[:at] - ls).abs() <= 1e-4).all()
    rest = n - at - 1
    few, ls = cache.attention(cache.batch(_i32(range(rest + 1)), _i32(kv[at + 1:]), table[at + 1:], rest, 1, 64), q[at + long:], lse=True)
    assert ((out[at + long:].float() - few.float()).abs() <= 2.0 ** -7 * few.float().abs() + 2.0 ** -9 * 5).all()
    assert ((lse[at + long:] - ls).abs() <= 1e-4).all()


def test_attention_of_a_million_sequences(serve):
    # 2^20 sequences x 16 heads, a workgroup each: two launches; eight pages that all of them share
    n, heads = 2 ** 20, 16
    gen = torch.Generator(device="cuda").manual_seed(7)
    cache = serve.KV4Cache(8, 16, heads, 64, group=32)
    k, v = (torch.randn(128, heads, 64, device="cuda", generator=gen, dtype=torch.float16) for _ in range(2))
    cache.append(cache.batch(_i32(range(0, 144, 16)), _i32([16] * 8), _i32(range(8))[:, None], 128, 16, 16), k, v)
    table = torch.randint(0, 8, (n, 1), device="cuda", generator=gen, dtype=torch.int32)
    kv = torch.randint(0, 17, (n,), device="cuda", generator=gen, dtype=torch.int32)
    q = torch.randn(n, heads, 64, device="cuda", generator=gen, dtype=torch.float16)
    start = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    out = cache.attention(cache.batch(start, kv, table, n, 1, 16), q)
    for lo in (0, n // 2 - 1000, n - 2000):
        few = cache.attention(cache.batch(start[:2001], kv[lo:lo + 2000], table[lo:lo + 2000], 2000, 1, 16), q[lo:lo + 2000])
        assert torch.equal(out[lo:lo + 2000], few) and few.abs().max() > 0


def test_w4_with_the_most_outputs(serve):
    # a workgroup for each of 2^23 - 1 tiles of outputs
    n, k = 2 ** 27 - 16, 32
    gen = torch.Generator(device="cuda").manual_seed(8)
    codes = torch.randint(0, 256, (n, k // 2), device="cuda", generator=gen, dtype=torch.uint8)
    scales = torch.rand(n, 1, device="cuda", generator=gen).bfloat16()
    x = torch.randn(2, k, device="cuda", generator=gen).bfloat16()
    y = serve.W4Weight(codes, scales).matmul(x)
    for lo in (0, n // 2, n - 4096):
        assert torch.equal(y[:, lo:lo + 4096], serve.W4Weight(codes[lo:lo + 4096], scales[lo:lo + 4096]).matmul(x))
