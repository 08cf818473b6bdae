"""Outputs that lie over a call's inputs, or over one another, are refused on the host; ones beside them are not
(no GPU is needed, none is touched: calls that pass are stopped by their workspace)."""
import ctypes as C

import pytest

from paper_2609_02109_amd import mf, serve

BF = mf.MF_BF16
X, Y, Z, CODES, SCALES, WEIGHT = 1 << 20, 2 << 20, 3 << 20, 4 << 20, 5 << 20, 6 << 20


def _row(rows=4, n=64, x=X, xs=64, codes=CODES, cs=64, scales=SCALES):
    return serve.Rows8Args(BF, rows, n, x, xs, codes, cs, scales)


# rows of 64 values: 128 bytes of x, 64 of codes, four of them 512 and 256, scales 16
@pytest.mark.parametrize("codes,cs", [(Y, 64), (Y + 511, 64), (Y - 255, 64), (Y + 128, 64), (Y, 128), (Y + 1, 128), (Y + 127, 128), (Y - 600, 1000)])
def test_codes_over_the_second_input(codes, cs):
    r = _row(codes=codes, cs=cs)
    assert mf.lib.mf_gate8(C.byref(serve.Gate8Args(r, Y, 64)), None) == mf.MF_EINVAL
    assert mf.lib.mf_norm8(C.byref(serve.Norm8Args(r, Y, 64, Z, 64, WEIGHT, 1e-6)), None) == mf.MF_EINVAL
    assert mf.lib.mf_norm8(C.byref(serve.Norm8Args(r, Z, 64, Y, 64, WEIGHT, 1e-6)), None) == mf.MF_EINVAL   # the sum: two outputs
    assert mf.lib.mf_norm8(C.byref(serve.Norm8Args(r, Y, 64, Y, 64, WEIGHT, 1e-6)), None) == mf.MF_EINVAL


def test_codes_between_rows_that_are_wider():
    # the second input's rows 256 bytes apart, the codes' too, in its second half: over the next row from 65 bytes on
    for at, want in ((Y + 127, mf.MF_EINVAL), (Y + 193, mf.MF_EINVAL), (Y + 256 - 63, mf.MF_EINVAL)):
        r = _row(codes=at, cs=256)
        assert mf.lib.mf_gate8(C.byref(serve.Gate8Args(r, Y, 128)), None) == want


@pytest.mark.parametrize("at", [-12, 0, 8, 508])
def test_scales_over_anything(at):
    for base in (X, CODES):
        r = _row(scales=base + (at if base == X else min(at, 252)))
        assert mf.lib.mf_rows8(C.byref(r), None) == mf.MF_EINVAL
        assert mf.lib.mf_gate8(C.byref(serve.Gate8Args(r, Y, 64)), None) == mf.MF_EINVAL
        assert mf.lib.mf_norm8(C.byref(serve.Norm8Args(r, None, 0, None, 0, WEIGHT, 1e-6)), None) == mf.MF_EINVAL
    r = _row(scales=Y + at)
    assert mf.lib.mf_gate8(C.byref(serve.Gate8Args(r, Y, 64)), None) == mf.MF_EINVAL
    for res, total in ((Y, Z), (Z, Y)):
        assert mf.lib.mf_norm8(C.byref(serve.Norm8Args(r, res, 64, total, 64, WEIGHT, 1e-6)), None) == mf.MF_EINVAL


def test_outputs_over_the_weight():
    for r, total in ((_row(codes=WEIGHT + 127), Z), (_row(codes=WEIGHT - 255), Z), (_row(scales=WEIGHT - 12), Z), (_row(), WEIGHT), (_row(), WEIGHT - 510)):
        assert mf.lib.mf_norm8(C.byref(serve.Norm8Args(r, Y, 64, total, 64, WEIGHT, 1e-6)), None) == mf.MF_EINVAL


@pytest.mark.parametrize("dt,size", [(mf.MF_F32, 4), (BF, 2)])
def test_values_over_what_they_are_made_of(dt, size):
    call = lambda out, cs=64, os=64: mf.lib.mf_rows8_values(dt, 4, 64, CODES, cs, SCALES, out, os, None)
    for out in (CODES, CODES + 252, CODES - 4 * 64 * size + size, SCALES, SCALES + 12, SCALES - 4 * 64 * size + size):
        assert call(out) == mf.MF_EINVAL
    assert call(CODES + 64, cs=64 * size, os=64) == mf.MF_EINVAL   # rows of 64 codes, results of the next rows' codes


def _w8(y=Y, bias=None, scales=None, x=X, rows=6, n=64, k=256, packed=Z, ys=64):
    return serve.W8Args(serve.W8Desc(n, k, BF), packed, x, scales, bias, y, rows, k, ys)


def test_products_over_what_they_are_made_of():
    # packed: 4 tiles of 4 records, and 64 scales
    size = 4 * 4 * 1024 + 256
    for a in (_w8(bias=Y), _w8(bias=Y + 766), _w8(bias=Y - 126), _w8(scales=Y), _w8(scales=Y + 764), _w8(scales=Y - 20), _w8(y=Z), _w8(y=Z + size - 2), _w8(y=Z - 766),
              _w8(y=X + 3070)):
        assert mf.lib.mf_w8_matmul(C.byref(a), 7 << 20, 1 << 20, None) == mf.MF_EINVAL
    # the workspace, which holds the rows' codes and scales (6 x 256 and 6 x 4 bytes)
    for a in (_w8(x=(7 << 20) + 1558), _w8(y=7 << 20), _w8(bias=(7 << 20) + 100)):
        assert mf.lib.mf_w8_matmul(C.byref(a), 7 << 20, 1 << 20, None) == mf.MF_EINVAL


def test_products_beside_what_they_are_made_of():
    """These pass, and are stopped by a workspace that is not there."""
    size = 4 * 4 * 1024 + 256
    for a in (_w8(), _w8(bias=Y + 768), _w8(bias=Y - 128), _w8(y=Z + size), _w8(y=Z - 768), _w8(y=X + 6 * 512), _w8(y=X - 768),
              _w8(x=Y + 128, ys=320, y=Y),          # columns of one buffer: rows of 640 bytes, 128 of results before 512 of x
              _w8(bias=Y + 128, ys=256)):           # between the rows of results
        if a.x_stride == 256 and a.d_x == Y + 128:
            a.x_stride = 320
        assert mf.lib.mf_w8_matmul(C.byref(a), None, 0, None) == mf.MF_ENOMEM


def test_weights_laid_out_over_themselves():
    d = serve.W8Desc(16, 128, BF)   # 2048 bytes of codes and 64 of scales, as laid out too
    for codes, scales, packed in ((X, Y, X), (X + 2048, Y, X), (X, Y, X + 1792), (X, Y + 2108, Y), (X, Y, Y)):
        assert mf.lib.mf_w8_pack(C.byref(d), codes, scales, packed, C.c_size_t(2112), None) == mf.MF_EINVAL


# ------------------------------------------------------------------ the caches

PAGES, STARTS, LENS, TABLE, COS, SIN = 16 << 20, 32 << 20, 33 << 20, 34 << 20, 35 << 20, 36 << 20
CACHES = [(mf.lib.mf_kv4_append, mf.lib.mf_kv4_read, mf.lib.mf_kv4_attention, lambda: serve.Cache(4, 16, 2, 64, 64, PAGES), 4 * 2 * (16 * 64 + 128)),
          (mf.lib.mf_kv8_append, mf.lib.mf_kv8_read, mf.lib.mf_kv8_attention, lambda: serve.Cache8(4, 16, 2, 64, PAGES), 4 * 2 * (32 * 64 + 8))]
kinds = pytest.mark.parametrize("kind", [0, 1], ids=["4-bit", "8-bit"])


def _batch(rows=3, n=1, cols=4, kv=20):
    return serve.Batch(n, rows, kv, rows, STARTS, LENS, TABLE, cols, cols)


def _append(kind, rows=3, k=X, ks=(128, 64), v=Y, vs=(128, 64), q=Z, qs=(256, 64), out=CODES, os=(256, 64), heads=4):
    call, _, _, cache, _ = CACHES[kind]
    a = serve.AppendArgs(BF, k, v, *ks, *vs, COS, SIN, 64, 64, 0, heads, q, out, *qs, *os)
    return call(C.byref(cache()), C.byref(_batch(rows)), C.byref(a), None)


@kinds
@pytest.mark.parametrize("kw", [
    dict(out=X), dict(out=Y), dict(out=X - 1534), dict(out=Y + 766), dict(out=COS + 2), dict(out=SIN), dict(out=COS + 20 * 32 * 4 - 2), dict(out=PAGES),
    dict(out=STARTS), dict(out=LENS), dict(out=TABLE), dict(out=Z + 2), dict(out=Z + 512), dict(out=Z, os=(512, 64)), dict(out=Z, os=(64, 192)),
    # one buffer of columns, 4 heads of q, 2 of k, 2 of v: the output over some of k's
    dict(q=Z, qs=(512, 64), k=Z + 512, ks=(512, 64), v=Z + 768, vs=(512, 64), out=Z + 128, os=(512, 64)),
    # the pages over what is read
    dict(k=PAGES), dict(v=PAGES + 64), dict(q=PAGES), dict(k=PAGES - 2)])
def test_append_over_what_it_reads(kind, kw):
    assert _append(kind, **kw) == mf.MF_EINVAL


def _attn(kind, rows=3, q=X, qs=(256, 64), out=Y, os=(256, 64), lse=None, heads=4, ws=None, room=0, kv=20, cols=4):
    _, _, call, cache, _ = CACHES[kind]
    a = serve.AttnArgs(BF, heads, q, out, lse, *qs, *os, 0.125, 0)
    return call(C.byref(cache()), C.byref(_batch(rows, cols=cols, kv=kv)), C.byref(a), ws, room, None)


@kinds
def test_attention_over_what_it_reads(kind):
    size = CACHES[kind][4]
    for kw in (dict(out=X + 2), dict(out=X + 512), dict(out=X - 1534), dict(out=X, os=(512, 64)), dict(out=X, os=(64, 192)), dict(out=PAGES), dict(out=PAGES + size - 2),
               dict(out=STARTS), dict(out=LENS + 2), dict(out=TABLE + 14), dict(lse=X), dict(lse=Y + 1532), dict(lse=PAGES), dict(lse=TABLE), dict(q=PAGES, out=PAGES)):
        assert _attn(kind, **kw) == mf.MF_EINVAL, kw


@kinds
def test_attention_beside_what_it_reads(kind):
    """These pass, and are stopped by a workspace that is not there."""
    size, long = CACHES[kind][4], dict(kv=60000, cols=4000, rows=1)
    for kw in (dict(), dict(out=X), dict(out=X, os=(777, 64)), dict(out=X + 512), dict(out=PAGES + size), dict(out=PAGES - 512), dict(lse=X + 512), dict(lse=Y + 512),
               dict(qs=(256, 192), out=X + 128, os=(256, 192)), dict(qs=(256, 192), out=X + 256, os=(256, 192)), dict(out=LENS + 4)):
        assert _attn(kind, **long, **kw) == mf.MF_ENOMEM, kw
    three = dict(kv=60000, cols=4000, rows=3)
    # rows inside heads, and columns of one buffer
    for kw in (dict(qs=(64, 192), os=(64, 192)), dict(qs=(512, 64), out=X + 512, os=(512, 64)), dict(out=X, os=(256, 64)), dict(qs=(768, 192), out=X + 128, os=(768, 192))):
        assert _attn(kind, **three, **kw) == mf.MF_ENOMEM, kw
    assert _attn(kind, **long, ws=X, room=1 << 30) == mf.MF_EINVAL
    assert _attn(kind, **long, ws=Y - 256, room=1 << 30) == mf.MF_EINVAL


@kinds
def test_read_over_what_it_reads(kind):
    _, call, _, cache, size = CACHES[kind]
    c, b = cache(), _batch()
    for ty, el in ((mf.MF_F32, 4), (BF, 2)):
        most = 3 * 2 * 64 * el
        for k, v in ((PAGES, X), (X, PAGES + size - 4), (X, PAGES - most + 4), (STARTS, X), (X, LENS), (TABLE + 12, None), (X, X), (X, X + most - 4), (X + most - 4, X)):
            assert call(C.byref(c), C.byref(b), ty, k, v, None) == mf.MF_EINVAL


# ------------------------------------------------------------- 4-bit products

def _w4(y=Y, bias=None, x=X, rows=3, n=64, k=256, packed=Z, ys=64, xs=None):
    return serve.W4Args(serve.W4Desc(n, k, 64, BF), packed, x, bias, y, rows, k if xs is None else xs, ys)


def test_4_bit_products_over_what_they_are_made_of():
    # packed: 4 tiles of 2 records of 1024 bytes of codes and 128 of scales
    size = 4 * 2 * (1024 + 128)
    for a in (_w4(y=X), _w4(y=X + 1534), _w4(y=X - 382), _w4(bias=Y), _w4(bias=Y + 382), _w4(bias=Y - 126), _w4(y=Z), _w4(y=Z + size - 2), _w4(y=Z - 382),
              _w4(y=X + 128, ys=256), _w4(y=X + 512, ys=512)):
        assert mf.lib.mf_w4_matmul(C.byref(a), 7 << 20, 1 << 20, None) == mf.MF_EINVAL
    nb = C.c_size_t(0)
    many = dict(n=4096, k=8192, rows=40, x=1 << 30, y=2 << 30, packed=3 << 30, ys=4096)
    a = _w4(**many)
    assert mf.lib.mf_w4_workspace_size(C.byref(a), C.byref(nb)) == mf.MF_OK and nb.value > 0
    for at in (1 << 30, (2 << 30) + 256, 3 << 30, (2 << 30) - nb.value // 512 * 256):
        assert mf.lib.mf_w4_matmul(C.byref(a), at, nb.value, None) == mf.MF_EINVAL


def test_4_bit_weights_laid_out_over_themselves():
    d = serve.W4Desc(16, 128, 64, BF)   # 1024 bytes of codes, 64 of scales, 32 of zero points; 1152 laid out
    for codes, scales, zeros, packed in ((X, Y, None, X), (X + 1150, Y, None, X), (X, Y, None, Y), (X, Y + 1150, Z, Y), (X, Y, Z, Z), (X, Y, Z - 30, Z)):
        assert mf.lib.mf_w4_pack(C.byref(d), codes, scales, zeros, packed, C.c_size_t(1152), None) == mf.MF_EINVAL
