"""Host-side checks of include/da_training.h that need no GPU: symbols, and arguments that are refused before any device work."""
import ctypes
import os
import re

import pytest

from paper_2202_08556_amd import binding as da

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
i64, vp, f32, size = ctypes.c_int64, ctypes.c_void_p, ctypes.c_float, ctypes.c_size_t
SIZES = (size(), size(), size())
OUT = [ctypes.byref(s) for s in SIZES]
P = vp(4096)                                                 # an address that no refused call looks at
ODD = vp(4097)
INVALID, UNSUPPORTED = da.DA_ERR_INVALID_ARG, da.DA_ERR_UNSUPPORTED


def lib():
    return ctypes.CDLL(os.path.join(ROOT, "paper_2202_08556_amd", "libdaspmm.so"))


def test_header_symbols_are_exported():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "da_training.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(da_\w+)\s*\(", text))
    assert names == set(da.TRAINING_EXPORTS)
    for n in names:
        assert getattr(lib(), n) is not None


# ---------------------------------------------------------------------------------------------
def rms(dtype=0, rows=10, C=8, x=P, ldx=8, res=P, ldr=8, w=P, param=0, eps=1e-6, total=P, y=P):
    return lib().da_rms_norm(dtype, i64(rows), i64(C), x, i64(ldx), res, i64(ldr), w, param, f32(eps), total, y, None)


def rms_e4m3(dtype=0, rows=10, C=8, x=P, ldx=8, eps=1e-6, q=P, scale=P):
    return lib().da_rms_norm_e4m3(dtype, i64(rows), i64(C), x, i64(ldx), None, i64(0), None, 0, f32(eps), None, q, scale, None)


def rms_back(dtype=0, rows=10, C=8, s=P, lds=8, dy=P, ldy=8, dsum=P, ldd=8, param=0, eps=1e-6, dx=P, dw=P, ws=P, bytes=1 << 24):
    return lib().da_rms_norm_backward(dtype, i64(rows), i64(C), s, i64(lds), dy, i64(ldy), dsum, i64(ldd), None, param, f32(eps), dx, dw,
                                      ws, size(bytes), None)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), UNSUPPORTED), (dict(param=7), UNSUPPORTED), (dict(rows=-1), INVALID), (dict(C=-1), INVALID), (dict(rows=2 ** 31), UNSUPPORTED),
    (dict(C=2 ** 20 + 1, ldx=2 ** 21, ldr=2 ** 21), UNSUPPORTED), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(ldx=7), INVALID), (dict(ldr=7), INVALID), (dict(x=None), INVALID), (dict(y=None), INVALID), (dict(total=None), INVALID),
    (dict(rows=0, x=None, y=None, total=None), da.DA_OK), (dict(C=0, ldx=0, ldr=0, x=None, y=None, total=None), da.DA_OK)])
def test_rms_norm(change, status):
    assert rms(**change) == status


@pytest.mark.parametrize("change,status", [(dict(scale=None), INVALID), (dict(q=None), INVALID), (dict(ldx=3), INVALID),
                                           (dict(rows=0, x=None, q=None, scale=None), da.DA_OK)])
def test_rms_norm_e4m3(change, status):
    assert rms_e4m3(**change) == status


@pytest.mark.parametrize("change,status", [
    (dict(s=None), INVALID), (dict(lds=7), INVALID), (dict(ldy=7), INVALID), (dict(ldd=7), INVALID), (dict(ws=None), INVALID),
    (dict(bytes=16), INVALID), (dict(ws=ODD), INVALID), (dict(dx=None, dw=None), da.DA_OK), (dict(C=0, lds=0, ldy=0, ldd=0), da.DA_OK)])
def test_rms_norm_backward(change, status):
    assert rms_back(**change) == status


# ---------------------------------------------------------------------------------------------
def ce_sizes(dtype=0, rows=10, d=8, V=5):
    return lib().da_linear_cross_entropy_sizes(dtype, i64(rows), i64(d), i64(V), *OUT)


def ce(dtype=0, rows=10, d=8, V=5, x=P, ldx=8, w=P, b=P, param=0, target=P, reduction=2, loss=P, stats=P, ws=P, bytes=1 << 30):
    return lib().da_linear_cross_entropy(dtype, i64(rows), i64(d), i64(V), x, i64(ldx), w, b, param, target, 1, reduction, loss, stats, ws,
                                         size(bytes), None)


def ce_back(dtype=0, rows=10, d=8, V=5, x=P, ldx=8, w=P, b=P, param=0, reduction=2, stats=P, dloss=P, stride=1, dx=P, dw=P, db=P, ws=P,
            bytes=1 << 40):
    return lib().da_linear_cross_entropy_backward(dtype, i64(rows), i64(d), i64(V), x, i64(ldx), w, b, param, reduction, stats, dloss,
                                                  i64(stride), dx, dw, db, ws, size(bytes), None)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=3), UNSUPPORTED), (dict(rows=-1), INVALID), (dict(d=-1), INVALID), (dict(V=-1), INVALID), (dict(rows=2 ** 26 + 1), UNSUPPORTED),
    (dict(d=2 ** 22 + 1), UNSUPPORTED), (dict(V=2 ** 22 + 1), UNSUPPORTED), (dict(rows=2 ** 26, V=2 ** 22), UNSUPPORTED),
    (dict(rows=0), da.DA_OK), (dict(V=0), da.DA_OK), (dict(d=0), da.DA_OK), (dict(rows=2 ** 26, d=1, V=2), da.DA_OK)])
def test_cross_entropy_sizes(change, status):
    assert ce_sizes(**change) == status
    if status == da.DA_OK:
        rows = change.get("rows", 10)
        assert SIZES[0].value >= 16 + 16 * rows and SIZES[1].value > 0 and SIZES[2].value > 0


@pytest.mark.parametrize("change,status", [
    (dict(ldx=7), INVALID), (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(param=9), UNSUPPORTED), (dict(target=None), INVALID),
    (dict(reduction=3), INVALID), (dict(reduction=-1), INVALID), (dict(loss=None), INVALID), (dict(stats=None), INVALID),
    (dict(stats=ODD), INVALID), (dict(ws=None), INVALID), (dict(bytes=16), INVALID), (dict(d=300, ldx=300, bytes=64), INVALID), (dict(ws=ODD), INVALID)])
def test_cross_entropy(change, status):
    assert ce(**change) == status


@pytest.mark.parametrize("change,status", [
    (dict(ldx=7), INVALID), (dict(x=None), INVALID), (dict(stride=-1), INVALID), (dict(dloss=None), INVALID), (dict(reduction=5), INVALID),
    (dict(b=None, param=9), UNSUPPORTED), (dict(bytes=64), INVALID), (dict(V=300, bytes=1024), INVALID), (dict(stats=None), INVALID), (dict(dx=None, dw=None, db=None), da.DA_OK)])
def test_cross_entropy_backward(change, status):
    assert ce_back(**change) == status


# ---------------------------------------------------------------------------------------------
GOOD = (3.4445, -4.775, 2.0315)


def orth(dtype=0, batch=1, rows=8, cols=8, g=P, ldg=8, stride=64, coefficients=GOOD * 5, eps=1e-7, out=P, ws=P, bytes=1 << 30, steps=None):
    c = (ctypes.c_float * len(coefficients))(*coefficients) if coefficients is not None else None
    steps = len(coefficients) // 3 if steps is None else steps
    return lib().da_orthogonalise(dtype, i64(batch), i64(rows), i64(cols), g, i64(ldg), i64(stride), steps, c, f32(eps), out, ws, size(bytes), None)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), UNSUPPORTED), (dict(batch=-1), INVALID), (dict(rows=-1), INVALID), (dict(batch=65536), UNSUPPORTED),
    (dict(rows=2 ** 17 + 1), UNSUPPORTED), (dict(cols=2 ** 17 + 1, ldg=2 ** 18), UNSUPPORTED), (dict(rows=2 ** 17, cols=2 ** 17, ldg=2 ** 17, batch=500), UNSUPPORTED),
    (dict(steps=-1), INVALID), (dict(steps=65), UNSUPPORTED), (dict(coefficients=None, steps=5), INVALID), (dict(ldg=7), INVALID),
    (dict(stride=-64), INVALID), (dict(eps=-1.0), INVALID), (dict(g=None), INVALID), (dict(out=None), INVALID), (dict(rows=80, cols=80, ldg=80, ws=None), INVALID),
    (dict(rows=80, cols=80, ldg=80, bytes=64), INVALID), (dict(rows=80, cols=80, ldg=80, ws=ODD), INVALID),
    # values that grow from step to step, or are none
    (dict(coefficients=(200.0, 0.0, 0.0)), INVALID), (dict(coefficients=(3.0, 0.0, 0.0) * 5), INVALID),
    (dict(coefficients=(float("nan"), 0.0, 0.0)), INVALID), (dict(coefficients=(1.0, float("inf"), 0.0)), INVALID),
    (dict(coefficients=(0.0, 9000.0, -9000.0)), da.DA_ERR_INVALID_ARG),
    (dict(batch=0), da.DA_OK), (dict(rows=0), da.DA_OK), (dict(cols=0, ldg=0), da.DA_OK)])
def test_orthogonalise(change, status):
    assert orth(**change) == status and (status == da.DA_OK or da.da_spmm_last_error())
