"""rms_norm and rms_norm_e4m3 against their formulas in 64 bits, forward and backward.

Tolerances, with e = 2^-24 and u half a step of the result's type (0 more for float32, whose e is counted).  A sum of n squares
is off by K e relative, K = 64 + n / 1024 (a lane's numbers one after the other, then pairs); r by (K / 2 + 4) e; y = s r w
by (K / 2 + 8) e and u.  The mean of dy w s r is off by (K + 8) e of the mean M of its magnitudes, so dx by
(K + 12) e r (|dy w| + |s r| M) + 2 e |dsum| and u; dw by (K / 2 + 8 + L) e of the sum of |dy s r|, L = 128 + rows / 64
additions, and u.  The sum is x + residual rounded once.  e4m3: the scale is off by (K / 2 + 10) e; q scale by
half a step of q: 2^-4 of it, or 2^-10 of the scale where q is below 2^-6."""
import math

import pytest
import torch

from paper_2202_08556_amd import layers

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
U = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}
SIZES = [(1, 1), (1, 4096), (3, 5), (7, 16), (300, 24), (1, 128), (1000, 128), (517, 602), (70, 1000), (33, 1024), (9, 2048), (5, 4100), (3, 8192),
         (2, 16384), (2, 16400), (3, 33000), (100, 3), (20000, 8), (2, 100003)]


def make(rows, C, dtype, seed=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed + rows * 7 + C)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")          # noqa: E731
    x, res = (r(rows, C) * scale).to(dtype), (2 * r(rows, C) * scale).to(dtype)
    return x, res, (1 + 0.2 * r(C)).to(dtype), r(rows, C).to(dtype), r(rows, C).to(dtype)


def check(x, w, res, dy, dsum, eps=1e-6):
    dt, C, rows = x.dtype, x.shape[-1], x.numel() // max(1, x.shape[-1])
    leaves = [t.detach().requires_grad_(True) for t in (x, w, res) if t is not None]
    it = iter(leaves)
    X, W, R = (next(it) if t is not None else None for t in (x, w, res))
    out = layers.rms_norm(X, W, residual=R, eps=eps)
    y, s = out if res is not None else (out, x)
    assert y.shape == x.shape and y.dtype == dt and s.shape == x.shape and s.dtype == dt
    grads = torch.autograd.grad((y, s) if res is not None else y, leaves, (dy, dsum) if res is not None else dy)
    torch.cuda.synchronize()
    d = lambda t: t.detach().double().cpu()                             # noqa: E731
    if res is not None:
        exact = d(x) + d(res)
        assert ((d(s) - exact).abs() <= exact.abs() * (U[dt] + 2 * E)).all()
    S, G = d(s), d(dy)
    Wd = d(w) if w is not None else torch.ones(C, dtype=torch.float64)
    K = 64 + C / 1024
    r = 1 / (S.square().mean(-1, keepdim=True) + eps).sqrt()
    want = S * r * Wd
    assert ((d(y) - want).abs() <= want.abs() * ((K / 2 + 8) * E + U[dt]) + 1e-44).all()
    xh, e = S * r, G * Wd
    M = (e * xh).abs().mean(-1, keepdim=True)
    more = d(dsum) if res is not None else torch.zeros_like(S)
    dx = r * (e - xh * (e * xh).mean(-1, keepdim=True)) + more
    tol = (K + 12) * E * r * (e.abs() + xh.abs() * M) + 2 * E * more.abs()
    got = dict(zip([n for n, t in (("x", x), ("w", w), ("res", res)) if t is not None], grads))
    for name in ("x", "res"):
        if name in got:
            assert ((d(got[name]) - dx).abs() <= tol * (1 + U[dt]) + dx.abs() * U[dt] + 1e-38).all(), name
    if w is not None:
        dw = (G * xh).flatten(0, -2).sum(0) if S.dim() > 1 else G * xh
        tw = ((G * xh).abs().flatten(0, -2).sum(0) if S.dim() > 1 else (G * xh).abs()) * (K / 2 + 8 + 128 + rows / 64) * E
        assert got["w"].dtype == w.dtype
        assert ((d(got["w"]) - dw).abs() <= tw * (1 + U[w.dtype]) + dw.abs() * (U[w.dtype] + E)).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("rows,C", SIZES)
def test_forward_and_backward(rows, C, dtype):
    x, res, w, dy, dsum = make(rows, C, dtype)
    check(x, w, res, dy, dsum)
    check(x, None if C % 3 == 0 else w, None, dy, None)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("rows,C", SIZES)
def test_eight_bits(rows, C, dtype):
    x, res, w, _, _ = make(rows, C, dtype, seed=1)
    with torch.no_grad():
        q, scale, s = layers.rms_norm_e4m3(x, w, residual=res)
        q0, scale0 = layers.rms_norm_e4m3(x)
    assert q.dtype == torch.float8_e4m3fn and q.shape == x.shape and scale.shape == x.shape[:1] and scale.dtype == torch.float32
    K = 64 + C / 1024
    for Q, sc, S, W in ((q, scale, s, w), (q0, scale0, x, torch.ones_like(w))):
        S, W = S.double().cpu(), W.double().cpu()
        y = S / (S.square().mean(-1, keepdim=True) + 1e-6).sqrt() * W
        sc, Q = sc.double().cpu()[:, None], Q.cpu().double()
        want = y.abs().amax(-1, keepdim=True) / 448
        assert ((sc - want).abs() <= want * (K / 2 + 10) * E).all()
        half = torch.maximum(y.abs() * 2.0 ** -4, sc * 2.0 ** -10)
        assert ((Q * sc - y).abs() <= half * (1 + 2.0 ** -3) + y.abs() * (K + 20) * E).all()
        assert Q.abs().max() <= 448


def test_rows_of_zeros_and_large_numbers():
    x = torch.zeros(4, 96, device="cuda")
    x[1] = 3e18                                              # the squares' sum is a float
    x[2, 5] = 1e-30
    w = torch.linspace(0.5, 2, 96, device="cuda")
    y = layers.rms_norm(x, w)
    q, scale = layers.rms_norm_e4m3(x, w)
    assert torch.equal(y[0], torch.zeros_like(y[0])) and torch.allclose(y[1], w, rtol=1e-5) and torch.isfinite(y).all()
    assert scale[0] == 0 and scale[3] == 0 and not q[0].float().any() and torch.isfinite(q.float()).all()
    x[3, 7] = float("nan")
    y, (q, scale) = layers.rms_norm(x, w), layers.rms_norm_e4m3(x, w)
    assert y[3].isnan().all() and scale[3].isnan() and q[3].float().isnan().all()
    assert y[:3].isfinite().all() and scale[:3].isfinite().all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_strides_and_types(dtype):
    wide = torch.randn(50, 200, device="cuda").to(dtype)
    x, res = wide[:, 3:73], wide[:, 101:171]                 # rows 200 apart, at odd addresses
    _, _, w, dy, dsum = make(50, 70, dtype)
    check(x, w, res, dy, dsum)
    check(x.t().contiguous().t(), w, res, dy, dsum)          # columns that are not neighbours
    check(x, w.float() if dtype == torch.bfloat16 else w.bfloat16(), res, dy, dsum)
    check(x.reshape(5, 10, 70), w, res.reshape(5, 10, 70), dy.view(5, 10, 70), dsum.view(5, 10, 70))
    check(x[7].clone(), w, res[7].clone(), dy[7], dsum[7])   # one axis
    check(x, w, res, torch.ones((), device="cuda", dtype=dtype).expand(50, 70), dsum)


def test_one_gradient_of_two():
    x, res, w, dy, dsum = make(40, 70, torch.float32)
    for pick in (0, 1):
        leaves = [t.clone().requires_grad_(True) for t in (x, res, w)]
        out = layers.rms_norm(leaves[0], leaves[2], residual=leaves[1])
        got = torch.autograd.grad(out[pick], leaves, (dy, dsum)[pick], allow_unused=True)
        L = [t.detach().double().requires_grad_(True) for t in (x, res, w)]
        s = L[0] + L[1]
        ref = ((s * torch.rsqrt(s.square().mean(-1, keepdim=True) + 1e-6) * L[2]), s)[pick]
        want = torch.autograd.grad(ref, L, (dy, dsum)[pick].double(), allow_unused=True)
        for a, b in zip(got, want):
            # 64 + 12 roundings of numbers of the order of 10; a weight that is not used has gradient 0
            b = torch.zeros_like(a) if b is None else b
            assert torch.allclose(a.double(), b.double(), rtol=1e-4, atol=1e-4)


def test_only_what_is_asked_for():
    x, res, w, dy, _ = make(64, 128, torch.float32)
    for need in ((True, False, False), (False, True, False), (False, False, True)):
        leaves = [t.clone().requires_grad_(n) for t, n in zip((x, res, w), need)]
        y, _ = layers.rms_norm(leaves[0], leaves[2], residual=leaves[1])
        y.backward(dy)
        assert [t.grad is not None for t in leaves] == list(need)


def test_differences():
    """The gradient along a direction is what the loss changes by; central differences in steps of 2^-7 are off by the third
    derivative's 2^-14 and by 2^-17 of the loss's terms."""
    x, res, w, dy, dsum = make(3, 40, torch.float32, seed=5)
    f = lambda a, b, c: sum((t * k).double().sum() for t, k in zip(layers.rms_norm(a, c, residual=b), (dy, dsum)))      # noqa: E731
    leaves = [t.clone().requires_grad_(True) for t in (x, res, w)]
    grads = torch.autograd.grad(f(*leaves), leaves)
    for i, t in enumerate((x, res, w)):
        v = torch.randn_like(t)
        h = 2.0 ** -7
        plus, minus = ([a + s * h * v if k == i else a for k, a in enumerate((x, res, w))] for s in (1, -1))
        slope = float((f(*plus) - f(*minus)) / (2 * h))
        scale = float(sum((k.abs()).sum() for k in (dy, dsum)))
        assert abs(slope - float((grads[i] * v).double().sum())) <= scale * 2.0 ** -9


def test_graph_and_streams():
    x, res, w, dy, dsum = make(300, 256, torch.bfloat16)
    X, R, W = (t.clone().requires_grad_(True) for t in (x, res, w))

    def step():
        y, s = layers.rms_norm(X, W, residual=R)
        return (y, s, *torch.autograd.grad((y, s), (X, R, W), (dy, dsum)))

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        want = [t.clone() for t in step()]
        step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for k in range(3):
        if k:
            with torch.no_grad():
                X.copy_(torch.randn_like(X))
            want = [t.clone() for t in step()]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k


@pytest.mark.parametrize("rows,C", [(530000, 4096), (140000, 16400)])
def test_many_numbers(rows, C):
    """Offsets beyond 32 bits: the last rows are what they are by themselves."""
    x = torch.empty(rows, C, device="cuda", dtype=torch.bfloat16).normal_()
    w = torch.randn(C, device="cuda")
    X = x.detach().requires_grad_(True)
    y, s = layers.rms_norm(X, w, residual=x)
    dx, = torch.autograd.grad((y, s), X, (x, x))
    few = x[-100:].clone().requires_grad_(True)
    y1, s1 = layers.rms_norm(few, w, residual=x[-100:])
    dx1, = torch.autograd.grad((y1, s1), few, (x[-100:], x[-100:]))
    # one row may be dealt to another number of lanes: the sum of squares in another order, and one rounding to bfloat16 more or less
    for a, b in ((y, y1), (s, s1), (dx, dx1)):
        assert torch.allclose(a[-100:].float(), b.float(), rtol=2.0 ** -7, atol=2.0 ** -9)
    with torch.no_grad():
        q, scale = layers.rms_norm_e4m3(x, w)
        q1, scale1 = layers.rms_norm_e4m3(x[-100:], w)
    assert torch.allclose(scale[-100:], scale1, rtol=1e-5) and torch.allclose(q[-100:].float(), q1.float(), rtol=0.13, atol=2.0 ** -8)


def test_refusals():
    x, res, w, dy, _ = make(8, 16, torch.float32)
    with pytest.raises(ValueError):
        layers.rms_norm(x, w[:8])
    with pytest.raises(ValueError):
        layers.rms_norm(x, w, residual=res[:1])              # not broadcast
    with pytest.raises(TypeError):
        layers.rms_norm(x, w, residual=res.bfloat16())
    with pytest.raises(TypeError):
        layers.rms_norm(x.half(), w)
    with pytest.raises(ValueError):
        layers.rms_norm(x.cpu(), w.cpu())
    with pytest.raises(ValueError):
        layers.rms_norm(x, w.cpu())
    with pytest.raises(da_error()):
        layers.rms_norm(x, w, eps=-1.0)
    with pytest.raises(ValueError):
        layers.rms_norm_e4m3(x.requires_grad_(True), w)
    y = layers.rms_norm(x, w)
    g, = torch.autograd.grad(y, x, dy, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(g.sum(), x)
    y, s = layers.rms_norm(x, w, residual=res)
    s.detach().mul_(2.0)                                     # the sum is read again backward
    with pytest.raises(RuntimeError):
        y.backward(dy)


def da_error():
    from paper_2202_08556_amd import binding
    return binding.DaSpmmError


def test_empty():
    for shape in ((0, 16), (5, 0), (0, 0)):
        x, w = torch.zeros(shape, device="cuda", requires_grad=True), torch.ones(shape[1], device="cuda", requires_grad=True)
        y, s = layers.rms_norm(x, w, residual=x.detach())
        dx, dw = torch.autograd.grad(y, (x, w), torch.zeros_like(y))
        assert y.shape == shape and dx.shape == shape and not dw.any()
        with torch.no_grad():
            q, scale = layers.rms_norm_e4m3(x)
        assert q.shape == shape and not scale.any()


def test_module():
    m = layers.RMSNorm(48).cuda()
    x = torch.randn(5, 48, device="cuda")
    y, s = m(x, residual=x)
    assert torch.equal(s, 2 * x) and torch.equal(y, layers.rms_norm(2 * x, m.weight)) and math.isclose(m.eps, 1e-6)
