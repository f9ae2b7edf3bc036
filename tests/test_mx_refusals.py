"""What the microscaled operators refuse, before any device work (no GPU).
Pointers are made up: a refused call reads none of them."""
import ctypes
import os

import pytest

from paper_2505_14260_amd import msd

if not os.path.exists(msd.LIB_PATH):
    pytest.skip("libmsd.so not built", allow_module_level=True)

A, B, C, D, E, G = (0x10000000 * (i + 1) for i in range(6))
SRC, DST = 0x100000000, 0x200000000


def q(rows=4, cols=64, layout=msd.MX_ROWS, terms=2, codes=A, scales=B):
    return msd.Mx(codes, scales, rows, cols, layout, terms)


W = dict(layout=msd.MX_WEIGHT, terms=1)


def refused(call):
    with pytest.raises(msd.MSDError) as e:
        call()
    assert e.value.code == msd.MSD_ERR_INVALID_ARG and str(e.value).strip()


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(rows=(1 << 23) + 1), dict(cols=0), dict(cols=-5), dict(cols=(1 << 20) + 1),
    dict(rows=1 << 20, cols=1 << 20), dict(layout=2), dict(layout=-1), dict(terms=0), dict(terms=3),
    dict(layout=msd.MX_WEIGHT, terms=2), dict(codes=None), dict(scales=None), dict(codes=A + 8),
    dict(scales=B + 4)], ids=str)
def test_bad_quantised_matrix(bad):
    m = q(**bad)
    ld = max(m.cols, 1)
    if not {"codes", "scales"} & set(bad):
        refused(lambda: msd.msd_mx_bytes(m))
    refused(lambda: msd.msd_mx_quantize(SRC, msd.F32, ld, m, None))
    refused(lambda: msd.msd_mx_dequantize(m, DST, msd.F32, ld, None))
    refused(lambda: msd.msd_mx_resid_norm(SRC, ld, None, 0, None, 0, msd.F32, G, 1e-5, m, None))
    refused(lambda: msd.msd_mx_swiglu(SRC, ld, DST, ld, msd.F32, m, None))
    refused(lambda: msd.msd_mx_product(m, q(**W, cols=ld), DST, msd.F32, 4, None))


def test_null_quantised_matrix():
    n = ctypes.c_size_t()
    lib = msd.lib()
    assert lib.msd_mx_bytes(None, ctypes.byref(n), ctypes.byref(n)) == msd.MSD_ERR_INVALID_ARG
    assert lib.msd_mx_quantize(SRC, 0, 64, None, None) == msd.MSD_ERR_INVALID_ARG
    assert lib.msd_mx_product(q(), None, DST, 0, 64, None) == msd.MSD_ERR_INVALID_ARG
    assert msd.msd_last_error(None)


@pytest.mark.parametrize("p, t, ld", [
    (None, msd.F32, 64), (SRC, 3, 64), (SRC, -1, 64), (SRC, msd.F32, 63), (SRC + 2, msd.F32, 64),
    (SRC + 1, msd.BF16, 64), (SRC, msd.F32, 1 << 60)], ids=str)
def test_bad_float_matrix(p, t, ld):
    refused(lambda: msd.msd_mx_quantize(p, t, ld, q(), None))
    refused(lambda: msd.msd_mx_dequantize(q(), p, t, ld, None))
    refused(lambda: msd.msd_mx_swiglu(p, ld, DST, 64, t, q(), None))
    refused(lambda: msd.msd_mx_swiglu(DST, 64, p, ld, t, q(), None))
    refused(lambda: msd.msd_mx_resid_norm(p, ld, None, 0, None, 0, t, G, 1e-5, q(), None))
    if p is not None:
        refused(lambda: msd.msd_mx_resid_norm(DST, 64, p, ld, None, 0, t, G, 1e-5, q(), None))
        refused(lambda: msd.msd_mx_resid_norm(DST, 64, None, 0, p, ld, t, G, 1e-5, q(), None))
    refused(lambda: msd.msd_mx_product(q(), q(rows=64, codes=C, scales=D, **W), p, t, ld, None))


def test_norm_and_swiglu_want_two_terms_in_rows():
    for m in (q(terms=1), q(**W)):
        refused(lambda: msd.msd_mx_swiglu(SRC, 64, DST, 64, msd.F32, m, None))
        refused(lambda: msd.msd_mx_resid_norm(SRC, 64, None, 0, None, 0, msd.F32, G, 1e-5, m, None))
    refused(lambda: msd.msd_mx_resid_norm(SRC, 8193, None, 0, None, 0, msd.F32, G, 1e-5,
                                          q(cols=8193), None))
    for eps in (-1e-5, float("inf"), float("nan")):
        refused(lambda: msd.msd_mx_resid_norm(SRC, 64, None, 0, None, 0, msd.F32, G, eps, q(), None))
    for g in (None, G + 1):
        refused(lambda: msd.msd_mx_resid_norm(SRC, 64, None, 0, None, 0, msd.F32, g, 1e-5, q(), None))


def test_product_shapes():
    w = q(rows=32, codes=C, scales=D, **W)
    refused(lambda: msd.msd_mx_product(q(cols=63), w, DST, msd.F32, 32, None))
    refused(lambda: msd.msd_mx_product(w, w, DST, msd.F32, 32, None))
    refused(lambda: msd.msd_mx_product(q(), q(codes=C, scales=D), DST, msd.F32, 32, None))
    refused(lambda: msd.msd_mx_product(q(), w, DST, msd.F32, 31, None))
    big = dict(rows=1 << 20, cols=32)
    refused(lambda: msd.msd_mx_product(q(**big), q(codes=C, scales=D, **W, **big), DST, msd.F32,
                                       1 << 20, None))


def test_overlaps():
    m = q()   # a tile of 1 KB and its scales in 256 bytes, of two terms
    nc, ns = msd.msd_mx_bytes(m)
    assert (nc, ns) == (2 * 1024, 2 * 256)
    refused(lambda: msd.msd_mx_quantize(A + nc - 4, msd.F32, 64, m, None))
    refused(lambda: msd.msd_mx_quantize(SRC, msd.F32, 64, q(scales=A + nc - 16), None))
    refused(lambda: msd.msd_mx_dequantize(m, B + ns - 16, msd.F32, 64, None))
    refused(lambda: msd.msd_mx_swiglu(SRC, 64, A, 64, msd.F32, m, None))
    # the sum may be an operand itself, not a shifted or otherwise strided one
    refused(lambda: msd.msd_mx_resid_norm(SRC, 64, DST, 64, SRC + 4, 64, msd.F32, G, 1e-5, m, None))
    refused(lambda: msd.msd_mx_resid_norm(SRC, 64, DST, 64, DST, 65, msd.F32, G, 1e-5, m, None))
    refused(lambda: msd.msd_mx_resid_norm(SRC, 64, DST, 64, G - 16, 64, msd.F32, G, 1e-5, m, None))
    refused(lambda: msd.msd_mx_resid_norm(SRC, 64, None, 0, A + 256, 64, msd.F32, G, 1e-5, m, None))
    w = q(rows=32, codes=C, scales=D, **W)
    refused(lambda: msd.msd_mx_product(m, w, A + 256, msd.F32, 32, None))
    refused(lambda: msd.msd_mx_product(m, w, D, msd.F32, 32, None))


@pytest.mark.parametrize("rows, cols, layout, terms, want", [
    # tiles of 16 rows x 128 columns; scales of four columns of tiles together
    (1, 1, msd.MX_ROWS, 1, (1024, 256)), (3, 128, msd.MX_ROWS, 2, (2048, 512)),
    (17, 513, msd.MX_ROWS, 2, (2 * 2 * 5 * 1024, 2 * 2 * 2 * 256)),
    (1, 1, msd.MX_WEIGHT, 1, (1024, 256)), (17, 640, msd.MX_WEIGHT, 1, (2 * 5 * 1024, 2 * 2 * 256)),
    (16, 256, msd.MX_WEIGHT, 1, (2 * 1024, 256)), (0, 64, msd.MX_ROWS, 2, (0, 0)),
    (152064, 3584, msd.MX_WEIGHT, 1, (9504 * 28 * 1024, 9504 * 7 * 256))])
def test_sizes(rows, cols, layout, terms, want):
    assert msd.msd_mx_bytes(q(rows, cols, layout, terms)) == want


def test_tensor_checks():
    torch = pytest.importorskip("torch")
    from paper_2505_14260_amd import mx
    m = mx.MX(4, 64, device="cpu")
    x = torch.zeros(4, 64)
    g = torch.ones(64, dtype=torch.bfloat16)
    w = mx.MX(8, 64, layout="weight", device="cpu")
    for call in (lambda: mx.MX(4, 64, layout="tiles"), lambda: mx.quantize(x[:3], m),
                 lambda: mx.quantize(x.t().contiguous().t(), m), lambda: mx.quantize(x.double(), m),
                 lambda: mx.dequantize(m, torch.zeros(64, 4)),
                 lambda: mx.resid_norm(x, x.bfloat16(), g, 1e-5, None, m),
                 lambda: mx.resid_norm(x, x, g.float(), 1e-5, None, m),
                 lambda: mx.resid_norm(x, x, g[:32], 1e-5, None, m),
                 lambda: mx.swiglu(x, x.half(), m),
                 lambda: mx.product(m, w, torch.zeros(4, 9)),
                 # right in all but that they are not on a GPU
                 lambda: mx.quantize(x, m), lambda: mx.dequantize(m, x),
                 lambda: mx.resid_norm(x, x, g, 1e-5, None, m), lambda: mx.swiglu(x, x, m),
                 lambda: mx.product(m, w, torch.zeros(4, 8))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(msd.MSDError):
        mx.MX(4, 64, layout="weight", terms=2, device="cpu")


def test_draft_sizes_and_refusals():
    d = msd.ModelDesc(2, 128, 4, 2, 64, 300 // 8 * 8, 515, 1e4, 1e-5)

    def weight(n, k):
        return -(-n // 16) * (-(-k // 128) * 1024 + -(-k // 512) * 256)
    F = 296
    want = (weight(128, 256) + weight(512, 128) + weight(128, 256) + weight(-(-F // 16) * 16 + F, 128)
            + weight(128, F) + weight(515, 128))
    assert msd.msd_draft_mx_bytes(d) == want
    refused(lambda: msd.msd_draft_mx_bytes(msd.ModelDesc(2, 128, 4, 3, 64, 296, 515, 1e4, 1e-5)))
    refused(lambda: msd.msd_set_draft_mx(None, 0x1000))
    assert msd.lib().msd_draft_mx_bytes(ctypes.byref(d), None) == msd.MSD_ERR_INVALID_ARG
