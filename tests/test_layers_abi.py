"""Host-side checks of include/da_layers.h that need no GPU: symbols, and arguments that are refused before any device work."""
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


def lib():
    return ctypes.CDLL(os.path.join(ROOT, "paper_2202_08556_amd", "libdaspmm.so"))


def test_header_symbols_are_exported():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "da_layers.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(da_\w+)\s*\(", text))
    assert names == set(da.LAYER_EXPORTS)
    for n in names:
        assert getattr(lib(), n) is not None


def norm_sizes(dtype=0, rows=10, samples=1, ragged=0, channels=8, groups=2, train=1):
    return lib().da_group_norm_sizes(dtype, i64(rows), i64(samples), ragged, i64(channels), i64(groups), train, *OUT)


def norm(dtype=0, rows=10, samples=1, offsets=None, channels=8, groups=2, x=P, ldx=8, param=0, eps=1e-5, act=0, y=P, ws=P, ws_bytes=1 << 20):
    return lib().da_group_norm(dtype, i64(rows), i64(samples), offsets, i64(channels), i64(groups), x, i64(ldx), None, None, param,
                               f32(eps), act, y, None, ws, size(ws_bytes), None)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), da.DA_ERR_UNSUPPORTED), (dict(rows=-1), da.DA_ERR_INVALID_ARG), (dict(groups=3), da.DA_ERR_INVALID_ARG),
    (dict(groups=0), da.DA_ERR_INVALID_ARG), (dict(channels=2 ** 21, groups=1), da.DA_ERR_UNSUPPORTED),
    (dict(rows=2 ** 31), da.DA_ERR_UNSUPPORTED), (dict(samples=-5), da.DA_ERR_INVALID_ARG)])
def test_group_norm_sizes(change, status):
    assert norm_sizes() == da.DA_OK
    assert norm_sizes(**change) == status and da.da_spmm_last_error()


@pytest.mark.parametrize("change,status", [
    (dict(act=9), da.DA_ERR_INVALID_ARG), (dict(act=-1), da.DA_ERR_INVALID_ARG), (dict(eps=-1.0), da.DA_ERR_INVALID_ARG),
    (dict(eps=float("nan")), da.DA_ERR_INVALID_ARG), (dict(ldx=7), da.DA_ERR_INVALID_ARG), (dict(x=None), da.DA_ERR_INVALID_ARG),
    (dict(y=None), da.DA_ERR_INVALID_ARG), (dict(samples=0), da.DA_ERR_INVALID_ARG), (dict(samples=3), da.DA_ERR_INVALID_ARG),
    (dict(param=4), da.DA_ERR_UNSUPPORTED), (dict(rows=100000, ws=None), da.DA_ERR_INVALID_ARG),
    (dict(rows=100000, ws_bytes=16), da.DA_ERR_INVALID_ARG), (dict(rows=100000, ws=vp(4097)), da.DA_ERR_INVALID_ARG),
    (dict(rows=0, samples=0, x=None, y=None), da.DA_OK), (dict(channels=0, ldx=0, x=None, y=None), da.DA_OK)])
def test_group_norm(change, status):
    assert norm(**change) == status


@pytest.mark.parametrize("sizes", [(0, 0, 0, 0), (1, 0, 8, 8), (1, 8, 0, 8), (1, 8, 8, 0), (5, 1, 1, 1), (1, 4096, 12288, 4096),
                                   (100003, 64, 256, 64), (2 ** 20, 2 ** 10, 2 ** 12, 2 ** 10)], ids=str)
@pytest.mark.parametrize("dtype", [0, 1])
def test_gated_workspace_of_any_size(sizes, dtype):
    assert lib().da_gated_workspace(dtype, *map(i64, sizes), *OUT[:2]) == da.DA_OK


def gated(rows=4, d=8, h=8, dout=8, x=P, ldx=8, wg=P, wu=P, wd=P, act=2, y=P, u=None, v=None, a=P, ws=None, ws_bytes=0, dtype=0):
    return lib().da_gated(dtype, i64(rows), i64(d), i64(h), i64(dout), x, i64(ldx), wg, wu, wd, act, y, u, v, a, ws, size(ws_bytes), None)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=7), da.DA_ERR_UNSUPPORTED), (dict(rows=-1), da.DA_ERR_INVALID_ARG), (dict(h=2 ** 31), da.DA_ERR_UNSUPPORTED),
    (dict(rows=2 ** 30, h=2 ** 20), da.DA_ERR_UNSUPPORTED), (dict(act=5), da.DA_ERR_INVALID_ARG), (dict(ldx=4), da.DA_ERR_INVALID_ARG),
    (dict(x=None), da.DA_ERR_INVALID_ARG), (dict(wu=None), da.DA_ERR_INVALID_ARG), (dict(y=None), da.DA_ERR_INVALID_ARG),
    (dict(a=None), da.DA_ERR_INVALID_ARG), (dict(u=P), da.DA_ERR_INVALID_ARG), (dict(ws=None), da.DA_ERR_INVALID_ARG),
    (dict(rows=0, x=None, y=None, a=None), da.DA_OK)])
def test_gated(change, status):
    assert gated(**change) == status


def distill(dtype=0, rows=3, classes=41, best=5, z=P, ldz=41, index=P, top=P, top_dtype=0, T=1.0, loss=P):
    return lib().da_distill(dtype, i64(rows), i64(classes), i64(best), z, i64(ldz), index, 0, top, top_dtype, f32(T), loss, None, None,
                            size(0), None)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=3), da.DA_ERR_UNSUPPORTED), (dict(top_dtype=3), da.DA_ERR_UNSUPPORTED), (dict(best=1025), da.DA_ERR_UNSUPPORTED),
    (dict(classes=2 ** 31 - 1, ldz=2 ** 31), da.DA_ERR_UNSUPPORTED), (dict(rows=-3), da.DA_ERR_INVALID_ARG),
    (dict(ldz=40), da.DA_ERR_INVALID_ARG), (dict(T=0.0), da.DA_ERR_INVALID_ARG), (dict(T=float("inf")), da.DA_ERR_INVALID_ARG),
    (dict(T=float("nan")), da.DA_ERR_INVALID_ARG), (dict(z=None), da.DA_ERR_INVALID_ARG), (dict(index=None), da.DA_ERR_INVALID_ARG),
    (dict(loss=None), da.DA_ERR_INVALID_ARG), (dict(rows=1, classes=10 ** 6, ldz=10 ** 6), da.DA_ERR_INVALID_ARG),   # no workspace
    (dict(rows=0, z=None, index=None, top=None, loss=None), da.DA_OK)])
def test_distill(change, status):
    assert distill(**change) == status


def test_python_refuses_what_is_not_on_the_gpu():
    import torch
    from paper_2202_08556_amd import layers
    x = torch.zeros(4, 8)
    for call in (lambda: layers.group_norm(x, 2), lambda: layers.gated_feed_forward(x, x.t(), x.t(), x),
                 lambda: layers.distill_loss(x, torch.zeros(4, 2, dtype=torch.int32), x[:, :2])):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("rows", [0, 1, 3, 10 ** 6])
@pytest.mark.parametrize("classes", [0, 1, 41, 8192, 65537, 2 ** 31 - 2 ** 16 - 1])
def test_distill_workspace_of_any_size(rows, classes):
    assert lib().da_distill_workspace(i64(rows), i64(classes), OUT[0]) == da.DA_OK
    pieces = SIZES[0].value // (8 * rows) if rows else 0
    assert pieces * 8192 <= max(classes, 8192)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("best", [0, 5, 1024])
def test_distill_of_no_rows_and_no_classes(dtype, best):
    assert distill(dtype=dtype, rows=0, classes=0, best=best, ldz=0, z=None, index=None, top=None, loss=None) == da.DA_OK
    assert lib().da_distill_backward(dtype, i64(3), i64(0), i64(best), None, i64(0), P, 0, P, 0, f32(1.0), None, None, i64(1), None,
                                     None) == da.DA_OK


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,channels,groups", [(1, 8008, 1001), (1, 65528, 8191), (3, 65535, 65535), (100, 8008, 1001), (10 ** 6, 65535, 65535),
                                                  (10 ** 6, 983025, 65535)])
def test_group_norm_workspace_of_rows_of_many_groups(rows, channels, groups, dtype):
    """Sums of dw and db: two numbers of 32 bits for every number of x at most, and no more than 1 GB."""
    assert norm_sizes(dtype=dtype, rows=rows, samples=rows, channels=channels, groups=groups) == da.DA_OK
    assert 0 < SIZES[2].value <= min(8 * rows * channels + 16, 2 ** 30)
