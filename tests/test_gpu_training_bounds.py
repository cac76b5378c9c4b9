"""The C entry points of include/da_training.h write to their outputs, statistics and workspaces, of the sizes that they report, and to
nothing else: everything lies between numbers that have to stay as they are.  Sizes from a seed, over all ways that a call may take."""
import ctypes
import random

import pytest
import torch

from paper_2202_08556_amd import binding as da

pytestmark = pytest.mark.gpu
GUARD, MARK = 4096, 0x5A
i64, vp, f32, size = ctypes.c_int64, ctypes.c_void_p, ctypes.c_float, ctypes.c_size_t


class Room:
    """Memory of `bytes` between two guards."""

    def __init__(self, bytes):
        self.bytes = max(int(bytes), 16)
        self.all = torch.full((self.bytes + 2 * GUARD,), MARK, dtype=torch.uint8, device="cuda")

    def ptr(self):
        return vp(self.all.data_ptr() + GUARD)

    def whole(self):
        end = (self.bytes + 15) // 16 * 16                   # the guard behind begins at the next 16 bytes
        return bool((self.all[:GUARD] == MARK).all()) and bool((self.all[GUARD + end:] == MARK).all())


def ptr(t):
    return vp(t.data_ptr()) if t is not None else None


def sizes_of(f, *args, count):
    out = [size() for _ in range(count)]
    assert f(*args, *[ctypes.byref(s) for s in out]) == da.DA_OK
    return [s.value for s in out]


def lib():
    return da._lib


def check(rooms):
    torch.cuda.synchronize()
    for name, r in rooms.items():
        assert r.whole(), name


def ce_shape(rng):
    kind = rng.choice(["narrow", "tall", "few", "general", "general"])
    if kind == "narrow":
        return rng.randint(1, 9000), rng.randint(0, 256), rng.randint(1, 128)
    if kind == "tall":
        return rng.randint(17, 5000), rng.randint(257, 900), rng.randint(1, 64)
    if kind == "few":
        return rng.randint(1, 16), rng.randint(1, 1500), rng.randint(1, 9000)
    return rng.randint(17, 6000), rng.randint(1, 500), rng.randint(65, 2500)


@pytest.mark.parametrize("seed", range(40))
def test_cross_entropy(seed):
    rng = random.Random(seed)
    rows, d, V = ce_shape(rng)
    dtype = rng.choice([0, 1])
    reduction = rng.choice([0, 1, 2])
    print(dict(rows=rows, d=d, V=V, dtype=dtype, reduction=reduction), flush=True)
    t = torch.float32 if dtype == 0 else torch.bfloat16
    n = t.itemsize
    torch.manual_seed(seed)
    ldx = d + rng.choice([0, 3])
    x, w, b = torch.randn(rows, ldx, device="cuda").to(t), torch.randn(d, V, device="cuda").to(t), torch.randn(V, device="cuda").to(t)
    target = torch.randint(-V, V, (rows,), device="cuda")
    keep, fwd, bwd = sizes_of(lib().da_linear_cross_entropy_sizes, dtype, i64(rows), i64(d), i64(V), count=3)
    stream = vp(torch.cuda.current_stream().cuda_stream)
    r = dict(loss=Room(4 * (rows if reduction == 0 else 1)), stats=Room(keep), forward=Room(fwd), backward=Room(bwd), dx=Room(rows * d * n),
             dw=Room(d * V * n), db=Room(V * n))
    common = (dtype, i64(rows), i64(d), i64(V), ptr(x), i64(ldx), ptr(w), ptr(b), dtype)
    assert lib().da_linear_cross_entropy(*common, ptr(target), 1, reduction, r["loss"].ptr(), r["stats"].ptr(), r["forward"].ptr(), size(fwd), stream) == 0
    check(r)
    dloss = torch.rand(rows, device="cuda")
    assert lib().da_linear_cross_entropy_backward(*common, reduction, r["stats"].ptr(), ptr(dloss), i64(1), r["dx"].ptr(), r["dw"].ptr(), r["db"].ptr(),
                                                  r["backward"].ptr(), size(bwd), stream) == 0
    check(r)


@pytest.mark.parametrize("seed", range(30))
def test_cross_entropy_of_some_rows(seed, monkeypatch):
    """... of 1 to 70 rows of a large weight."""
    monkeypatch.setitem(globals(), "ce_shape", lambda rng: (rng.randint(1, 70), rng.choice([rng.randint(1, 64), rng.randint(257, 2000)]), rng.randint(65, 5000)))
    test_cross_entropy(seed)


@pytest.mark.parametrize("seed", range(25))
def test_orthogonalise(seed):
    rng = random.Random(seed)
    batch = rng.choice([1, 1, 2, 5])
    rows, cols = (rng.randint(1, 64), rng.randint(1, 512)) if seed % 3 == 0 else (rng.randint(65, 900), rng.randint(65, 1500))
    if rng.random() < 0.5:
        rows, cols = cols, rows
    dtype, steps = rng.choice([0, 1]), rng.choice([0, 1, 3])
    print(dict(batch=batch, rows=rows, cols=cols, dtype=dtype, steps=steps), flush=True)
    t = torch.float32 if dtype == 0 else torch.bfloat16
    ld = cols + rng.choice([0, 5])
    g = torch.randn(batch, rows, ld, device="cuda").to(t)
    need, = sizes_of(lib().da_orthogonalise_workspace, dtype, i64(batch), i64(rows), i64(cols), steps, count=1)
    c = (ctypes.c_float * (3 * steps))(*(3.4445, -4.775, 2.0315) * steps)
    r = dict(out=Room(batch * rows * cols * t.itemsize), workspace=Room(need))
    assert lib().da_orthogonalise(dtype, i64(batch), i64(rows), i64(cols), ptr(g), i64(ld), i64(rows * ld), steps, c, f32(1e-7), r["out"].ptr(),
                                  r["workspace"].ptr(), size(need), vp(torch.cuda.current_stream().cuda_stream)) == 0
    check(r)


@pytest.mark.parametrize("seed", range(25))
def test_rms_norm(seed):
    rng = random.Random(seed)
    C = round(2 ** rng.uniform(0, 15.5))
    rows = rng.randint(1, max(1, min(3000, 2000000 // C)))
    dtype = rng.choice([0, 1])
    print(dict(rows=rows, C=C, dtype=dtype), flush=True)
    t = torch.float32 if dtype == 0 else torch.bfloat16
    n, ld = t.itemsize, C + rng.choice([0, 1])
    x, res, dy, dsum = (torch.randn(rows, ld, device="cuda").to(t) for _ in range(4))
    w = torch.randn(C, device="cuda").to(t)
    need, = sizes_of(lib().da_rms_norm_workspace, dtype, i64(rows), i64(C), count=1)
    stream = vp(torch.cuda.current_stream().cuda_stream)
    r = dict(total=Room(rows * C * n), y=Room(rows * C * n), q=Room(rows * C), scale=Room(rows * 4), dx=Room(rows * C * n), dw=Room(C * n),
             workspace=Room(need))
    common = (dtype, i64(rows), i64(C), ptr(x), i64(ld), ptr(res), i64(ld), ptr(w), dtype, f32(1e-6), r["total"].ptr())
    assert lib().da_rms_norm(*common, r["y"].ptr(), stream) == 0
    assert lib().da_rms_norm_e4m3(*common, r["q"].ptr(), r["scale"].ptr(), stream) == 0
    assert lib().da_rms_norm_backward(dtype, i64(rows), i64(C), ptr(x), i64(ld), ptr(dy), i64(ld), ptr(dsum), i64(ld), ptr(w), dtype, f32(1e-6),
                                      r["dx"].ptr(), r["dw"].ptr(), r["workspace"].ptr(), size(need), stream) == 0
    check(r)
