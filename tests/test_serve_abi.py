"""The served steps' C entries on the host: sizes, and arguments that are
refused before anything is enqueued (no GPU is needed, none is touched)."""
import ctypes as C

import pytest

from paper_2609_02109_amd import mf, serve


def _w4(n=64, k=256, g=64, dt=mf.MF_BF16, rows=1, x=1024, y=4096, packed=1 << 20, bias=None, xs=None, ys=None):
    return serve.W4Args(serve.W4Desc(n, k, g, dt), packed, x, bias, y, rows, k if xs is None else xs, n if ys is None else ys)


def _bytes(call, *args):
    nb = C.c_size_t(0)
    s = call(*[C.byref(a) for a in args], C.byref(nb))
    return nb.value if s == mf.MF_OK else -s


def _cache(pages=4, page=16, heads=2, d=64, g=32, at=1 << 20):
    return serve.Cache(pages, page, heads, d, g, at)


def _batch(n=1, new=1, kv=20, rows=1, start=1024, lens=2048, table=4096, stride=4, cols=4):
    return serve.Batch(n, new, kv, rows, start, lens, table, stride, cols)


def _attn(dt=mf.MF_BF16, heads=4, q=1024, out=2048, lse=None, s=256, h=64, os=256, oh=64, scale=0.125, window=0):
    return serve.AttnArgs(dt, heads, q, out, lse, s, h, os, oh, scale, window)


def _append(dt=mf.MF_BF16, k=1024, v=2048, cos=4096, sin=8192, n_pos=64, rot=64, heads=0, q=None, qo=None, **kw):
    st = dict(k_s=128, k_h=64, v_s=128, v_h=64, q_s=256, q_h=64, o_s=256, o_h=64, inter=0)
    st.update(kw)
    return serve.AppendArgs(dt, k, v, st["k_s"], st["k_h"], st["v_s"], st["v_h"], cos, sin, n_pos, rot, st["inter"], heads, q, qo,
                            st["q_s"], st["q_h"], st["o_s"], st["o_h"])


@pytest.mark.parametrize("n,k,g,dt,want", [
    (16, 128, 128, mf.MF_BF16, 1024 + 64), (17, 160, 32, mf.MF_F16, 4 * (1024 + 256)), (1, 32, 32, mf.MF_BF16, 1024 + 256),
    (64, 256, 64, mf.MF_F32, -mf.MF_EINVAL), (64, 256, 64, 77, -mf.MF_EINVAL), (64, 256, 64, -1, -mf.MF_EINVAL), (64, 256, 16, mf.MF_BF16, -mf.MF_EUNSUPPORTED),
    (64, 256, 0, mf.MF_BF16, -mf.MF_EUNSUPPORTED), (64, 192, 128, mf.MF_BF16, -mf.MF_EINVAL), (0, 256, 64, mf.MF_BF16, -mf.MF_EINVAL),
    (64, 0, 64, mf.MF_BF16, -mf.MF_EINVAL), (-5, 256, 64, mf.MF_BF16, -mf.MF_EINVAL), (2 ** 31 - 15, 32, 32, mf.MF_BF16, -mf.MF_EUNSUPPORTED),
    (64, 2 ** 24 + 64, 64, mf.MF_BF16, -mf.MF_EUNSUPPORTED)])
def test_w4_sizes(n, k, g, dt, want):
    assert _bytes(mf.lib.mf_w4_pack_bytes, serve.W4Desc(n, k, g, dt)) == want


@pytest.mark.parametrize("kw,want", [
    (dict(dt=mf.MF_F32), mf.MF_EINVAL), (dict(rows=-1), mf.MF_EINVAL), (dict(rows=2 ** 20 + 1), mf.MF_EUNSUPPORTED), (dict(packed=None), mf.MF_EINVAL),
    (dict(packed=1025), mf.MF_EINVAL), (dict(x=None), mf.MF_EINVAL), (dict(x=1025), mf.MF_EINVAL), (dict(y=None), mf.MF_EINVAL),
    (dict(y=4097), mf.MF_EINVAL), (dict(bias=3), mf.MF_EINVAL), (dict(rows=2, xs=255), mf.MF_EINVAL), (dict(xs=-1), mf.MF_EINVAL),
    (dict(rows=2, ys=63), mf.MF_EINVAL), (dict(rows=2, ys=2 ** 41), mf.MF_EINVAL), (dict(rows=0), mf.MF_OK)])
def test_w4_matmul_refusals(kw, want):
    assert mf.lib.mf_w4_matmul(C.byref(_w4(**kw)), None, 0, None) == want


def test_w4_workspace():
    assert _bytes(mf.lib.mf_w4_workspace_size, _w4(rows=0)) == 0 and _bytes(mf.lib.mf_w4_workspace_size, _w4(rows=1)) == 0
    a = _w4(n=4096, k=8192, rows=40)
    need = _bytes(mf.lib.mf_w4_workspace_size, a)
    assert need > 0 and need % (40 * 4096 * 4) == 0
    assert mf.lib.mf_w4_matmul(C.byref(a), 4096, need - 1, None) == mf.MF_ENOMEM
    assert mf.lib.mf_w4_matmul(C.byref(a), None, need, None) == mf.MF_ENOMEM
    assert mf.lib.mf_w4_matmul(C.byref(a), 4097, need, None) == mf.MF_EINVAL
    for f in (mf.lib.mf_w4_pack_bytes, mf.lib.mf_w4_workspace_size, mf.lib.mf_kv4_cache_bytes):
        assert f(None, None) == mf.MF_EINVAL
    assert mf.lib.mf_w4_matmul(None, None, 0, None) == mf.MF_EINVAL


def test_w4_pack_refusals():
    d = serve.W4Desc(16, 128, 128, mf.MF_BF16)
    for codes, scales, packed, room, want in ((None, 2, 256, 1088, mf.MF_EINVAL), (1, None, 256, 1088, mf.MF_EINVAL), (1, 3, 256, 1088, mf.MF_EINVAL),
                                              (1, 2, None, 1088, mf.MF_EINVAL), (1, 2, 128, 1088, mf.MF_EINVAL), (1, 2, 256, 1087, mf.MF_ENOMEM)):
        assert mf.lib.mf_w4_pack(C.byref(d), codes, scales, None, packed, C.c_size_t(room), None) == want


def test_cache_bytes():
    # per token and head D bytes of codes and 8 D / G of scales and offsets
    for d, g in ((64, 32), (64, 64), (128, 32), (128, 128), (256, 64)):
        assert _bytes(mf.lib.mf_kv4_cache_bytes, _cache(3, 48, 5, d, g)) == 3 * 48 * 5 * (d + 8 * d // g)
    # sizes past 32 bits
    assert _bytes(mf.lib.mf_kv4_cache_bytes, _cache(2 ** 31 - 1, 1024, 1024, 256, 32)) == (2 ** 31 - 1) * 2 ** 20 * 320


@pytest.mark.parametrize("cache,batch,args,want", [
    ({}, dict(n=-1), {}, mf.MF_EINVAL), ({}, dict(new=-1), {}, mf.MF_EINVAL), ({}, dict(rows=-1), {}, mf.MF_EINVAL),
    ({}, dict(kv=65), {}, mf.MF_EINVAL), ({}, dict(n=2, stride=3), {}, mf.MF_EINVAL), ({}, dict(n=2 ** 20 + 1), {}, mf.MF_EUNSUPPORTED),
    ({}, dict(rows=2 ** 30 + 1), {}, mf.MF_EUNSUPPORTED), ({}, dict(start=None), {}, mf.MF_EINVAL), ({}, dict(lens=2049), {}, mf.MF_EINVAL),
    ({}, dict(table=None), {}, mf.MF_EINVAL), (dict(at=None), {}, {}, mf.MF_EINVAL), (dict(at=128), {}, {}, mf.MF_EINVAL),
    (dict(d=96), {}, {}, mf.MF_EUNSUPPORTED), (dict(page=20), {}, {}, mf.MF_EUNSUPPORTED), (dict(heads=1025), {}, {}, mf.MF_EUNSUPPORTED),
    ({}, {}, dict(dt=mf.MF_F32), mf.MF_EINVAL), ({}, {}, dict(heads=3), mf.MF_EINVAL), ({}, {}, dict(heads=0), mf.MF_EINVAL),
    ({}, {}, dict(heads=4098), mf.MF_EUNSUPPORTED), ({}, {}, dict(scale=0.0), mf.MF_EINVAL), ({}, {}, dict(scale=float("inf")), mf.MF_EINVAL),
    ({}, {}, dict(window=-1), mf.MF_EINVAL), ({}, {}, dict(q=None), mf.MF_EINVAL), ({}, {}, dict(out=2049), mf.MF_EINVAL),
    ({}, {}, dict(lse=2), mf.MF_EINVAL), ({}, {}, dict(oh=63), mf.MF_EINVAL), ({}, dict(rows=2, new=2), dict(os=255), mf.MF_EINVAL),
    ({}, {}, dict(s=-1), mf.MF_EINVAL), ({}, dict(rows=2 ** 30), dict(heads=4096), mf.MF_EUNSUPPORTED),
    ({}, dict(rows=0), {}, mf.MF_OK), ({}, dict(n=0), {}, mf.MF_OK), ({}, dict(new=0), {}, mf.MF_OK)])
def test_attention_refusals(cache, batch, args, want):
    c, b, a = _cache(**cache), _batch(**batch), _attn(**args)
    assert mf.lib.mf_kv4_attention(C.byref(c), C.byref(b), C.byref(a), None, 0, None) == want


def test_attention_workspace():
    c, a = _cache(), _attn()
    assert _bytes(mf.lib.mf_kv4_workspace_size, c, _batch(), a) == 0
    b = _batch(kv=60000, cols=4000, stride=4000)
    need = _bytes(mf.lib.mf_kv4_workspace_size, c, b, a)
    assert need > 0
    # a window leaves too little to split
    assert _bytes(mf.lib.mf_kv4_workspace_size, c, b, _attn(window=100)) == 0
    assert mf.lib.mf_kv4_attention(C.byref(c), C.byref(b), C.byref(a), None, need, None) == mf.MF_ENOMEM
    assert mf.lib.mf_kv4_attention(C.byref(c), C.byref(b), C.byref(a), 4096, need - 1, None) == mf.MF_ENOMEM
    assert mf.lib.mf_kv4_attention(C.byref(c), C.byref(b), C.byref(a), 4097, need, None) == mf.MF_EINVAL


@pytest.mark.parametrize("args,want", [
    (dict(dt=mf.MF_F32), mf.MF_EINVAL), (dict(cos=None), mf.MF_EINVAL), (dict(sin=None), mf.MF_EINVAL), (dict(n_pos=19), mf.MF_EINVAL),
    (dict(rot=8), mf.MF_EINVAL), (dict(rot=80), mf.MF_EINVAL), (dict(rot=24), mf.MF_EUNSUPPORTED), (dict(cos=4097), mf.MF_EINVAL),
    (dict(k=None), mf.MF_EINVAL), (dict(v=2049), mf.MF_EINVAL), (dict(k_s=-1), mf.MF_EINVAL), (dict(heads=-1), mf.MF_EINVAL),
    (dict(q=1024, heads=4), mf.MF_EINVAL), (dict(q=1024, qo=2048, heads=0), mf.MF_EINVAL), (dict(q=1024, qo=2048, heads=4097), mf.MF_EUNSUPPORTED),
    (dict(q=1024, qo=2048, heads=4, cos=None, sin=None), mf.MF_EINVAL), (dict(q=1024, qo=2048, heads=4, o_h=63), mf.MF_EINVAL)])
def test_append_refusals(args, want):
    c, b, a = _cache(), _batch(), _append(**args)
    assert mf.lib.mf_kv4_append(C.byref(c), C.byref(b), C.byref(a), None) == want


def test_read_refusals():
    c, b = _cache(), _batch()
    assert mf.lib.mf_kv4_read(C.byref(c), C.byref(b), 5, 1024, 2048, None) == mf.MF_EINVAL
    assert mf.lib.mf_kv4_read(C.byref(c), C.byref(b), mf.MF_F32, 1026, 2048, None) == mf.MF_EINVAL
    assert mf.lib.mf_kv4_read(C.byref(c), C.byref(b), mf.MF_BF16, 1025, 2048, None) == mf.MF_EINVAL
    assert mf.lib.mf_kv4_read(C.byref(c), C.byref(b), mf.MF_BF16, None, None, None) == mf.MF_OK
