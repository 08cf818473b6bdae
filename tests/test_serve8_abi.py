"""The 8-bit step's C entries on the host: sizes, and arguments that are refused
before anything is enqueued (no GPU is needed, none is touched)."""
import ctypes as C

import pytest

from paper_2609_02109_amd import mf, serve

INF, NAN = float("inf"), float("nan")


def _bytes(call, *args):
    nb = C.c_size_t(0)
    s = call(*[C.byref(a) for a in args], C.byref(nb))
    return nb.value if s == mf.MF_OK else -s


def _row(dt=mf.MF_BF16, rows=2, n=64, x=1024, xs=64, codes=2048, cs=64, scales=4096):
    return serve.Rows8Args(dt, rows, n, x, xs, codes, cs, scales)


ROWS = [(dict(dt=mf.MF_F32), mf.MF_EINVAL), (dict(dt=-1), mf.MF_EINVAL), (dict(rows=-1), mf.MF_EINVAL), (dict(n=0), mf.MF_EINVAL), (dict(n=-5), mf.MF_EINVAL),
        (dict(n=2 ** 17 + 1, xs=2 ** 18, cs=2 ** 18), mf.MF_EUNSUPPORTED), (dict(rows=2 ** 30 + 1), mf.MF_EUNSUPPORTED), (dict(x=None), mf.MF_EINVAL),
        (dict(x=1025), mf.MF_EINVAL), (dict(codes=None), mf.MF_EINVAL), (dict(scales=None), mf.MF_EINVAL), (dict(scales=4098), mf.MF_EINVAL),
        (dict(xs=63), mf.MF_EINVAL), (dict(xs=-1), mf.MF_EINVAL), (dict(cs=63), mf.MF_EINVAL), (dict(cs=2 ** 41), mf.MF_EINVAL), (dict(rows=0), mf.MF_OK),
        (dict(rows=0, x=None), mf.MF_OK)]


@pytest.mark.parametrize("kw,want", ROWS)
def test_rows_refusals(kw, want):
    r = _row(**kw)
    assert mf.lib.mf_rows8(C.byref(r), None) == want
    assert mf.lib.mf_norm8(C.byref(serve.Norm8Args(r, None, 0, None, 0, 1024, 1e-6)), None) == want
    assert mf.lib.mf_gate8(C.byref(serve.Gate8Args(r, 1024, 64)), None) == want


@pytest.mark.parametrize("res,rs,total,ss,weight,eps,want", [
    (None, 0, None, 0, None, 1e-6, mf.MF_EINVAL), (None, 0, None, 0, 3, 1e-6, mf.MF_EINVAL), (None, 0, None, 0, 2, -1.0, mf.MF_EINVAL),
    (None, 0, None, 0, 2, NAN, mf.MF_EINVAL), (None, 0, None, 0, 2, INF, mf.MF_EINVAL), (2, 64, None, 64, 2, 1e-6, mf.MF_EINVAL),
    (3, 64, 2, 64, 2, 1e-6, mf.MF_EINVAL), (2, 64, 3, 64, 2, 1e-6, mf.MF_EINVAL), (2, 63, 2, 64, 2, 1e-6, mf.MF_EINVAL),
    (2, 64, 2, 63, 2, 1e-6, mf.MF_EINVAL), (2, -1, 2, 64, 2, 1e-6, mf.MF_EINVAL), (2, 64, 2, 66, 2, 1e-6, mf.MF_EINVAL),
    (2, 64, 1024, 66, 2, 1e-6, mf.MF_EINVAL)])
def test_norm_refusals(res, rs, total, ss, weight, eps, want):
    assert mf.lib.mf_norm8(C.byref(serve.Norm8Args(_row(), res, rs, total, ss, weight, eps)), None) == want


def test_gate_and_value_refusals():
    for up, us in ((None, 64), (3, 64), (2, 63), (2, -1)):
        assert mf.lib.mf_gate8(C.byref(serve.Gate8Args(_row(), up, us)), None) == mf.MF_EINVAL
    good = dict(dt=mf.MF_F32, rows=2, n=64, codes=1, cs=64, scales=4, out=4, os=64)
    for kw, want in ((dict(dt=7), mf.MF_EINVAL), (dict(rows=-1), mf.MF_EINVAL), (dict(n=0), mf.MF_EINVAL), (dict(n=2 ** 17 + 1), mf.MF_EUNSUPPORTED),
                     (dict(codes=None), mf.MF_EINVAL), (dict(scales=2), mf.MF_EINVAL), (dict(out=2), mf.MF_EINVAL), (dict(out=None), mf.MF_EINVAL),
                     (dict(cs=63), mf.MF_EINVAL), (dict(os=63), mf.MF_EINVAL), (dict(rows=0), mf.MF_OK)):
        a = {**good, **kw}
        assert mf.lib.mf_rows8_values(a["dt"], a["rows"], a["n"], a["codes"], a["cs"], a["scales"], a["out"], a["os"], None) == want, kw
    for f in (mf.lib.mf_rows8, mf.lib.mf_norm8, mf.lib.mf_gate8):
        assert f(None, None) == mf.MF_EINVAL


# weights: records of 16 outputs and 64 inputs, an even number of them, and whole tiles of scales
@pytest.mark.parametrize("n,k,dt,want", [
    (16, 128, mf.MF_BF16, 2048 + 64), (17, 160, mf.MF_F16, 2 * 4 * 1024 + 128), (1, 16, mf.MF_BF16, 2048 + 64), (64, 256, mf.MF_F32, -mf.MF_EINVAL),
    (64, 256, 9, -mf.MF_EINVAL), (64, 24, mf.MF_BF16, -mf.MF_EUNSUPPORTED), (0, 64, mf.MF_BF16, -mf.MF_EINVAL), (64, 0, mf.MF_BF16, -mf.MF_EINVAL),
    (-1, 64, mf.MF_BF16, -mf.MF_EINVAL), (2 ** 27 - 16, 16, mf.MF_BF16, (2 ** 23 - 1) * (2048 + 64)), (2 ** 27 - 15, 16, mf.MF_BF16, -mf.MF_EUNSUPPORTED),
    (1, 131056, mf.MF_BF16, 2048 * 1024 + 64), (1, 131072, mf.MF_BF16, -mf.MF_EUNSUPPORTED), (2 ** 40, 16, mf.MF_BF16, -mf.MF_EUNSUPPORTED)])
def test_weight_sizes(n, k, dt, want):
    assert _bytes(mf.lib.mf_w8_pack_bytes, serve.W8Desc(n, k, dt)) == want


def test_pack_refusals():
    d = serve.W8Desc(16, 128, mf.MF_BF16)
    for codes, scales, packed, room, want in ((None, 4, 256, 2112, mf.MF_EINVAL), (1, None, 256, 2112, mf.MF_EINVAL), (1, 2, 256, 2112, mf.MF_EINVAL),
                                              (1, 4, None, 2112, mf.MF_EINVAL), (1, 4, 128, 2112, mf.MF_EINVAL), (1, 4, 256, 2111, mf.MF_ENOMEM)):
        assert mf.lib.mf_w8_pack(C.byref(d), codes, scales, packed, C.c_size_t(room), None) == want


def _w8(n=64, k=256, dt=mf.MF_BF16, rows=1, x=1024, scales=4096, y=8192, packed=1 << 20, bias=None, xs=None, ys=None):
    return serve.W8Args(serve.W8Desc(n, k, dt), packed, x, scales, bias, y, rows, k if xs is None else xs, n if ys is None else ys)


@pytest.mark.parametrize("kw,want", [
    (dict(dt=mf.MF_F32), mf.MF_EINVAL), (dict(rows=-1), mf.MF_EINVAL), (dict(rows=2 ** 20 + 1), mf.MF_EUNSUPPORTED), (dict(packed=None), mf.MF_EINVAL),
    (dict(packed=1025), mf.MF_EINVAL), (dict(x=None), mf.MF_EINVAL), (dict(x=1025, scales=None), mf.MF_EINVAL), (dict(scales=4098), mf.MF_EINVAL),
    (dict(y=None), mf.MF_EINVAL), (dict(y=8193), mf.MF_EINVAL), (dict(bias=3), mf.MF_EINVAL), (dict(rows=2, xs=255), mf.MF_EINVAL),
    (dict(xs=-1), mf.MF_EINVAL), (dict(rows=2, ys=63), mf.MF_EINVAL), (dict(rows=2, ys=2 ** 41), mf.MF_EINVAL), (dict(k=40), mf.MF_EUNSUPPORTED),
    (dict(rows=2 ** 20, n=2 ** 17 + 1, k=16), mf.MF_EUNSUPPORTED), (dict(rows=0), mf.MF_OK), (dict(rows=0, packed=None), mf.MF_OK)])
def test_product_refusals(kw, want):
    assert mf.lib.mf_w8_matmul(C.byref(_w8(**kw)), None, 0, None) == want


# outputs over inputs: rows of 64 values of 2 bytes at x = 1024, a step of 128 bytes (256 where wide)
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("at,want_narrow,want_wide", [
    (1024 - 128, mf.MF_EINVAL, None), (1024, mf.MF_EINVAL, mf.MF_EINVAL), (1024 + 2, mf.MF_EINVAL, mf.MF_EINVAL), (1024 + 126, mf.MF_EINVAL, mf.MF_EINVAL),
    (1024 + 130, mf.MF_EINVAL, mf.MF_EINVAL), (1024 + 254, mf.MF_EINVAL, mf.MF_EINVAL)])
def test_outputs_over_inputs_are_refused(wide, at, want_narrow, want_wide):
    step, want = (128, want_wide) if wide else (64, want_narrow)
    if want is None:
        return   # between the rows, or before them: it would run
    a = _w8(n=64, k=64, rows=4, x=1024, scales=None, xs=step, y=at, ys=step)
    assert mf.lib.mf_w8_matmul(C.byref(a), None, 0, None) == want
    if at != 1024:   # a sum may be over its row itself
        r = _row(rows=4, xs=step, codes=1 << 20)
        assert mf.lib.mf_norm8(C.byref(serve.Norm8Args(r, 1 << 16, step, at, step, 2, 1e-6)), None) == want
        r = _row(rows=4, x=1 << 16, xs=step, codes=1 << 20)
        assert mf.lib.mf_norm8(C.byref(serve.Norm8Args(r, 1024, step, at, step, 2, 1e-6)), None) == want


def test_codes_over_rows_are_refused():
    for at in (1024, 1025, 1024 + 4 * 128 - 1, 1024 - 255):
        assert mf.lib.mf_rows8(C.byref(_row(rows=4, codes=at)), None) == mf.MF_EINVAL
    # at other steps between one another
    assert mf.lib.mf_rows8(C.byref(_row(rows=4, xs=128, codes=1024 + 128, cs=64)), None) == mf.MF_EINVAL
    assert mf.lib.mf_rows8(C.byref(_row(rows=2 ** 30, xs=2 ** 40, codes=1 << 50, cs=2 ** 40)), None) == mf.MF_EINVAL


def test_product_workspace():
    size = lambda **kw: _bytes(mf.lib.mf_w8_workspace_size, _w8(**kw))
    # rows in 8 bits need none, nor do a few in 16, which the product takes as they are
    assert size(rows=5000) == 0 and size(rows=0, scales=None) == 0 and size(rows=4, scales=None) == 0 and size(rows=4, k=8192, scales=None) == 0
    assert size(rows=5, scales=None) == 5 * 256 + 5 * 4
    assert size(rows=3, k=16 * 1000, scales=None) == (3 * 16000 + 255) // 256 * 256 + 12
    assert size(rows=3, k=8192, scales=None) == 0 and size(rows=3, k=8208, scales=None) == (3 * 8208 + 255) // 256 * 256 + 12
    assert size(rows=1, k=32784, scales=None) == (32784 + 255) // 256 * 256 + 4
    a = _w8(rows=5, scales=None)
    need = _bytes(mf.lib.mf_w8_workspace_size, a)
    assert mf.lib.mf_w8_matmul(C.byref(a), 4096, need - 1, None) == mf.MF_ENOMEM
    assert mf.lib.mf_w8_matmul(C.byref(a), None, need, None) == mf.MF_ENOMEM
    assert mf.lib.mf_w8_matmul(C.byref(a), 4097, need, None) == mf.MF_EINVAL
    for f in (mf.lib.mf_w8_pack_bytes, mf.lib.mf_w8_workspace_size, mf.lib.mf_kv8_cache_bytes):
        assert f(None, None) == mf.MF_EINVAL
    assert mf.lib.mf_w8_matmul(None, None, 0, None) == mf.MF_EINVAL and mf.lib.mf_w8_workspace_size(C.byref(a), None) == mf.MF_EINVAL


def _cache(pages=4, page=16, heads=2, d=64, at=1 << 20):
    return serve.Cache8(pages, page, heads, d, at)


def _batch(n=1, new=1, kv=20, rows=1, start=1024, lens=2048, table=4096, stride=4, cols=4):
    return serve.Batch(n, new, kv, rows, start, lens, table, stride, cols)


def _attn(dt=mf.MF_BF16, heads=4, q=1024, out=2048, lse=None, s=256, h=64, os=256, oh=64, scale=0.125, window=0):
    return serve.AttnArgs(dt, heads, q, out, lse, s, h, os, oh, scale, window)


def test_cache_bytes():
    # per token and head 2 D bytes of codes, and two scales for 16 tokens
    for d in (64, 128, 256):
        assert _bytes(mf.lib.mf_kv8_cache_bytes, _cache(3, 48, 5, d)) == 3 * 3 * 5 * (32 * d + 8)
    assert _bytes(mf.lib.mf_kv8_cache_bytes, _cache(2 ** 31 - 1, 1024, 1024, 256)) == (2 ** 31 - 1) * 64 * 1024 * (32 * 256 + 8)


@pytest.mark.parametrize("cache,batch,args,want", [
    ({}, dict(n=-1), {}, mf.MF_EINVAL), ({}, dict(kv=65), {}, mf.MF_EINVAL), ({}, dict(n=2 ** 20 + 1), {}, mf.MF_EUNSUPPORTED),
    ({}, dict(start=None), {}, mf.MF_EINVAL), ({}, dict(table=None), {}, mf.MF_EINVAL), (dict(at=None), {}, {}, mf.MF_EINVAL), (dict(at=128), {}, {}, mf.MF_EINVAL),
    (dict(d=96), {}, {}, mf.MF_EUNSUPPORTED), (dict(page=20), {}, {}, mf.MF_EUNSUPPORTED), (dict(page=2048), {}, {}, mf.MF_EUNSUPPORTED),
    (dict(heads=1025), {}, {}, mf.MF_EUNSUPPORTED), (dict(pages=0), {}, {}, mf.MF_EINVAL), ({}, {}, dict(dt=mf.MF_F32), mf.MF_EINVAL),
    ({}, {}, dict(heads=3), mf.MF_EINVAL), ({}, {}, dict(heads=4098), mf.MF_EUNSUPPORTED), ({}, {}, dict(scale=0.0), mf.MF_EINVAL),
    ({}, {}, dict(scale=INF), mf.MF_EINVAL), ({}, {}, dict(window=-1), mf.MF_EINVAL), ({}, {}, dict(q=None), mf.MF_EINVAL), ({}, {}, dict(out=2049), mf.MF_EINVAL),
    ({}, {}, dict(lse=2), mf.MF_EINVAL), ({}, {}, dict(oh=63), mf.MF_EINVAL), ({}, dict(rows=2 ** 30), dict(heads=4096), mf.MF_EUNSUPPORTED),
    ({}, dict(rows=0), {}, mf.MF_OK), ({}, dict(n=0), {}, mf.MF_OK), ({}, dict(new=0), {}, mf.MF_OK)])
def test_attention_refusals(cache, batch, args, want):
    c, b, a = _cache(**cache), _batch(**batch), _attn(**args)
    assert mf.lib.mf_kv8_attention(C.byref(c), C.byref(b), C.byref(a), None, 0, None) == want


def test_attention_workspace():
    c, a = _cache(), _attn()
    assert _bytes(mf.lib.mf_kv8_workspace_size, c, _batch(), a) == 0
    b = _batch(kv=60000, cols=4000, stride=4000)
    need = _bytes(mf.lib.mf_kv8_workspace_size, c, b, a)
    assert need > 0 and _bytes(mf.lib.mf_kv8_workspace_size, c, b, _attn(window=100)) == 0
    assert mf.lib.mf_kv8_attention(C.byref(c), C.byref(b), C.byref(a), None, need, None) == mf.MF_ENOMEM
    assert mf.lib.mf_kv8_attention(C.byref(c), C.byref(b), C.byref(a), 4096, need - 1, None) == mf.MF_ENOMEM
    assert mf.lib.mf_kv8_attention(C.byref(c), C.byref(b), C.byref(a), 4097, need, None) == mf.MF_EINVAL


def _append(dt=mf.MF_BF16, k=1024, v=2048, cos=4096, sin=8192, n_pos=64, rot=64, heads=0, q=None, qo=None, k_s=128, o_h=64):
    return serve.AppendArgs(dt, k, v, k_s, 64, 128, 64, cos, sin, n_pos, rot, 0, heads, q, qo, 256, 64, 256, o_h)


@pytest.mark.parametrize("args,want", [
    (dict(dt=mf.MF_F32), mf.MF_EINVAL), (dict(cos=None), mf.MF_EINVAL), (dict(n_pos=19), mf.MF_EINVAL), (dict(rot=8), mf.MF_EINVAL),
    (dict(rot=80), mf.MF_EINVAL), (dict(rot=24), mf.MF_EUNSUPPORTED), (dict(cos=4097), mf.MF_EINVAL), (dict(k=None), mf.MF_EINVAL),
    (dict(v=2049), mf.MF_EINVAL), (dict(k_s=-1), mf.MF_EINVAL), (dict(q=1024, heads=4), mf.MF_EINVAL), (dict(q=1024, qo=2048, heads=4097), mf.MF_EUNSUPPORTED),
    (dict(q=1024, qo=2048, heads=4, cos=None, sin=None), mf.MF_EINVAL), (dict(q=1024, qo=2048, heads=4, o_h=63), mf.MF_EINVAL)])
def test_append_refusals(args, want):
    c, b, a = _cache(), _batch(), _append(**args)
    assert mf.lib.mf_kv8_append(C.byref(c), C.byref(b), C.byref(a), None) == want


def test_read_and_null_refusals():
    c, b = _cache(), _batch()
    for ty, k, v, want in ((5, 1024, 2048, mf.MF_EINVAL), (mf.MF_F32, 1026, 2048, mf.MF_EINVAL), (mf.MF_BF16, 1025, 2048, mf.MF_EINVAL),
                           (mf.MF_BF16, None, None, mf.MF_OK)):
        assert mf.lib.mf_kv8_read(C.byref(c), C.byref(b), ty, k, v, None) == want
    assert mf.lib.mf_kv8_append(None, C.byref(b), None, None) == mf.MF_EINVAL and mf.lib.mf_kv8_append(C.byref(c), None, None, None) == mf.MF_EINVAL
    assert mf.lib.mf_kv8_append(C.byref(c), C.byref(b), None, None) == mf.MF_EINVAL
    assert mf.lib.mf_kv8_attention(C.byref(c), C.byref(b), None, None, 0, None) == mf.MF_EINVAL


# ---------------------------------------------------- what Python refuses, without a GPU

@pytest.mark.parametrize("field", ["n_pages", "page_size", "n_kv_heads", "head_dim"])
@pytest.mark.parametrize("past", [2 ** 32, -2 ** 32, 2 ** 64])
def test_sizes_past_32_bits_are_refused(field, past):
    sizes = dict(n_pages=4, page_size=16, n_kv_heads=2, head_dim=64)
    with pytest.raises(ValueError):
        serve.KV8Cache(**{**sizes, field: sizes[field] + past})


def test_tensors_of_the_host_are_refused():
    import torch
    x, codes = torch.zeros(2, 64, dtype=torch.bfloat16), torch.zeros(2, 64, dtype=torch.int8)
    for bad in (lambda: serve.quantise_rows(x), lambda: serve.norm_rows(x, x[0]), lambda: serve.gate_rows(x, x), lambda: serve.quantise_rows(None),
                lambda: serve.Rows8(codes, torch.ones(2)).values(), lambda: serve.W8Weight(codes, torch.ones(2))):
        with pytest.raises(ValueError):
            bad()


def test_a_batch_of_another_device_is_refused():
    import torch
    cache, batch = object.__new__(serve.KV8Cache), object.__new__(serve.KV4Batch)
    cache.device, batch.device = torch.device("cuda", 0), torch.device("cuda", 1)
    for call in (lambda: cache.append(batch, None, None), lambda: cache.read(batch), lambda: cache.attention(batch, None)):
        with pytest.raises(ValueError):
            call()
