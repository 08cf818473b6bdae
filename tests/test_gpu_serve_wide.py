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
