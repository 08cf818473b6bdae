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
