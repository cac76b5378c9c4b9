"""linear_cross_entropy on every way that its sizes can take: masks, bad numbers, numbers of very different size, strides, refused and
partial gradients, graphs.  Each test says which kernels the call launches, so that sizes cannot move to another way unseen.

Tolerances as in the tests of the formula, but for each row by itself: what its results are off by follows from its own numbers, its
own factor and the weight, never from other rows.  With bfloat16 dz has the 11 bits of fp16 for dx and dw.  Pairs of halves keep 2^-35 of a row's largest x (2^-36 and a bit for the
row's scale), 2^-39 of its factor for dz, 2^-39 of the largest w; a row adds to dw with an error of 2^-37 of the largest product of
a row's x and its factor."""
import pytest
import torch

from paper_2202_08556_amd import layers

from .gpu_util import kernels_of

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
U = {torch.float32: E, torch.bfloat16: 2.0 ** -8}
F32, BF16 = torch.float32, torch.bfloat16

# rows, inner positions, classes; what the backward pass launches
WAYS = {
    "narrow": ((100, 32, 60), "ce_narrow_kernel"),
    "tall": ((100, 300, 60), "ce_tall_weight_kernel"),
    "few": ((3, 32, 700), "ce_few_products_kernel"),
    "some": ((15, 32, 700), "ce_some_products_kernel"),
    "some_more": ((31, 32, 700), "ce_some_products_kernel"),
    "packed": ((200, 32, 700), "plane_kernel"),
    "packed_wide": ((300, 200, 2100), "plane_kernel"),       # several tiles both ways
}
EACH = pytest.mark.parametrize("way", list(WAYS))
TYPES = pytest.mark.parametrize("dtype", [F32, BF16], ids=str)


def make(way, dtype, share=1.0, seed=0, bias=True):
    rows, d, V = WAYS[way][0]
    g = torch.Generator(device="cuda").manual_seed(seed + rows + 3 * d + 7 * V)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")          # noqa: E731
    x, w = r(rows, d).to(dtype), (2 * d ** -0.5 * r(d, V)).to(dtype)
    b = (0.3 * r(V)).to(dtype) if bias else None
    t = torch.randint(0, V, (rows,), generator=g, device="cuda")
    t = torch.where(torch.rand(rows, generator=g, device="cuda") < share, t, -1)
    return x, w, b, t, torch.rand(rows, generator=g, device="cuda") + 0.1


def run(x, w, b, t, g, reduction="none"):
    """(loss, dx, dw, db or nothing)"""
    leaves = [v.detach().requires_grad_(True) for v in (x, w, b) if v is not None]
    loss = layers.linear_cross_entropy(leaves[0], leaves[1], t, bias=leaves[2] if b is not None else None, reduction=reduction)
    return (loss.detach(), *torch.autograd.grad(loss, leaves, g if reduction == "none" else g.flatten()[0]))


def takes(way, *args, **kw):
    kernels = kernels_of(lambda: run(*args, **kw))
    ours = {k for k in kernels if "ce_" in k or "plane_kernel" in k}
    assert any(WAYS[way][1] in k for k in ours), (way, ours)
    others = {k for _, k in WAYS.values()} - {WAYS[way][1]}
    assert not any(o in k for o in others for k in ours), (way, ours)


def formula(x, w, b, t, g):
    """Results and tolerances in 64 bits on the CPU, row by row; g: factors of the rows."""
    dtype, rows = x.dtype, x.shape[0]
    f = lambda a: a.detach().cpu().double()                              # noqa: E731
    d, V = w.shape
    t = t.cpu()
    keep = ((t >= 0) & (t < V)).nonzero()[:, 0]
    X, W, g, t = f(x)[keep], f(w), f(g)[keep], t[keep]
    halves = dtype == F32
    extra = 2.0 ** -20 if halves else 0.0
    xm, wm, gm = X.abs().amax(1, keepdim=True), W.abs().max(), g.abs()[:, None]
    z = torch.mm(X, W) + (f(b) if b is not None else 0)
    err = ((d / 16 + 16) * E + extra) * torch.mm(X.abs(), W.abs()) + 2 * E * z.abs().masked_fill(z.isinf(), 0)
    if halves:
        err = err + 2.0 ** -34 * d * xm * wm
    D = err.amax(1, keepdim=True)
    K = 64 + V / 1024
    lse = z.logsumexp(1, keepdim=True)
    loss, t_loss = (lse - z.gather(1, t[:, None]))[:, 0], (2 * D + (K + 4 * lse.abs()) * E)[:, 0]
    p = (z - lse).exp()
    away = (z - lse).abs().masked_fill(z.isinf(), 0)
    one = torch.zeros_like(p).scatter_(1, t[:, None], 1.0)
    dz = g[:, None] * (p - one)
    # an error e of a logit is a factor exp(e) of p; and p, computed or not, is between 0 and 1, but for the rounding of z - lse where
    # z is the largest logit and lse above it: whatever the logits are off by, p is off by 1 and a little at most
    t_p = torch.nan_to_num(p * torch.expm1(2 * D + (K + 4 * away) * E), nan=1.0, posinf=1.0).clamp(max=1.0) + 2.0 ** -20 * p
    t_sum = gm * (t_p + 4 * E * (p + one))                   # db adds what has not been rounded as an operand
    t_dz = t_sum + dz.abs() * (2.0 ** -22 if halves else 2.0 ** -11) + 2.0 ** -39 * gm         # pairs, or one fp16 number
    dx, t_dx = torch.mm(dz, W.t()), torch.mm(t_dz, W.abs().t()) + ((V / 16 + 16) * E + extra) * torch.mm(dz.abs(), W.abs().t())
    dw, t_dw = torch.mm(X.t(), dz), torch.mm(X.abs().t(), t_dz) + ((rows / 16 + 80) * E + extra) * torch.mm(X.abs().t(), dz.abs())
    t_dx = t_dx + 2.0 ** -38 * V * gm * wm                   # the weight's numbers far below the largest, or those of its line
    t_dw = t_dw + 2.0 ** -37 * rows * (xm * gm).max()
    db, t_db = dz.sum(0), t_sum.sum(0) + (rows / 16 + 80) * E * dz.abs().sum(0)
    place = lambda v: torch.zeros(rows, *v.shape[1:], dtype=v.dtype).index_copy(0, keep, v)             # noqa: E731
    return [(place(loss), place(t_loss), E), (place(dx), place(t_dx), U[dtype]), (dw, t_dw, U[dtype])] + \
        ([(db, t_db, U[b.dtype])] if b is not None else [])


def check(x, w, b, t, g):
    got = run(x, w, b, t, g)
    for name, a, (want, tol, u) in zip(("loss", "dx", "dw", "db"), got, formula(x, w, b, t, g)):
        a = a.cpu().double()
        room = tol * (1 + u) + want.abs() * u + 2.0 ** -126
        off = (a - want).abs()
        assert (off <= room).all(), (name, float((off / room).max()), (off / room).argmax().item())
    return got


@EACH
@TYPES
def test_plain(way, dtype):
    args = make(way, dtype, share=0.8)
    takes(way, *args)
    check(*args)


@EACH
@pytest.mark.parametrize("reduction", ["none", "sum"])
def test_bias_in_32_bits_beside_bfloat16(way, reduction):
    """The gradient of a float32 bias is a sum in 32 bits of numbers in 32 bits, also where dz is rounded for the other products."""
    x, w, b, t, g = make(way, BF16, share=0.8)
    b = b.float()
    if reduction == "none":
        check(x, w, b, t, g)
        return
    db = run(x, w, b, t, g, reduction="sum")[3]
    want, tol, u = formula(x, w, b, t, g[0].expand(x.shape[0]))[3]
    assert u == E and ((db.cpu().double() - want).abs() <= tol * (1 + u) + want.abs() * 2 * E).all()


@EACH
@TYPES
def test_masked_classes(way, dtype):
    """A bias of -inf, or of the type's lowest value, takes a class out, whole waves and tiles of them too; one that leaves only the
    target gives loss 0."""
    x, w, b, t, g = make(way, dtype)
    V = w.shape[1]
    left = V // 7
    t = t % left
    for low in (float("-inf"), torch.finfo(dtype).min):
        masked = b.clone()
        masked[left:] = low
        takes(way, x, w, masked, t, g)
        loss, dx, dw, db = run(x, w, masked, t, g)
        want = formula(x, w[:, :left], b[:left], t, g)       # the others are not there at all
        for name, a, (ref, tol, u) in zip(("loss", "dx", "dw", "db"), (loss, dx, dw[:, :left], db[:left]), want):
            # the scale of w is that of all classes: 2^-34 of its largest number
            more = 2.0 ** -34 * float(x.abs().max()) * float(w.abs().max()) * x.shape[1] * (1 + float(w.abs().max()) * V)
            assert ((a.cpu().double() - ref).abs() <= tol * (1 + u) + ref.abs() * u + more).all(), (name, low)
        assert not dw[:, left:].any() and not db[left:].any()
    masked = torch.full_like(b, float("-inf"))
    masked[left - 1] = 0
    rows = x.shape[0]
    loss, dx, dw, db = run(x, w, masked, torch.full_like(t, left - 1), g)
    assert torch.equal(loss, torch.zeros(rows, device="cuda")) and not dx.any() and not dw.any() and not db.any()
    assert (run(x, w, masked, torch.full_like(t, left), g)[0] == float("inf")).all()


@EACH
@TYPES
def test_bad_rows_stay_by_themselves(way, dtype):
    """NaN and infinities in labelled rows: those rows' loss and dx are none, the others' are the same bits."""
    x, w, b, t, g = make(way, dtype)
    takes(way, x, w, b, t, g)
    want = run(x, w, b, t, g)
    bad = [0, 2] if x.shape[0] < 14 else [1, 13]
    x = x.clone()
    x[bad[0], 3], x[bad[1], 0] = float("nan"), float("inf")
    got = run(x, w, b, t, g)
    rest = torch.ones(x.shape[0], dtype=torch.bool, device="cuda")
    rest[bad] = False
    assert torch.equal(got[0][rest], want[0][rest]) and torch.equal(got[1][rest], want[1][rest])
    assert not torch.isfinite(got[0][~rest]).any() and not torch.isfinite(got[1][~rest]).any()


@EACH
@TYPES
def test_infinite_weights(way, dtype):
    """Rows without a target get no gradient whatever the weight holds."""
    x, w, b, t, g = make(way, dtype)
    t[: (x.shape[0] + 1) // 2] = -1
    w = w.clone()
    w[5, 7], w[6, 40] = float("inf"), float("nan")
    takes(way, x, w, b, t, g)
    loss, dx, dw, db = run(x, w, b, t, g)
    assert not loss[t < 0].any() and not dx[t < 0].any()
    assert torch.isnan(loss[t >= 0]).all() and torch.isnan(dx[t >= 0]).any(1).all()
    t[:] = -1
    loss, dx, dw, db = run(x, w, b, t, g)
    assert not loss.any() and not dx.any() and not dw.any() and not db.any()


@EACH
@TYPES
def test_rows_of_very_different_size(way, dtype):
    """What a row's loss and gradient are off by does not depend on other rows."""
    x, w, b, t, g = make(way, dtype)
    rows = x.shape[0]
    size = torch.logspace(-6, 1, rows, device="cuda").to(dtype)
    takes(way, x * size[:, None], w, b, t, g)
    check(x * size[:, None], w, b, t, g * torch.logspace(-5, 0, rows, device="cuda"))
    for k in (1e8, 1e12, 1e25):                              # one number, and one row's factor, far beyond the others
        y, f = x.clone(), g.clone()
        y[0, 0] = k
        check(y, w, b, t, g)
        f[rows // 2] = k
        check(x, w, b, t, f)
        check(y, w, b, t, f / k)
    check(x, w, b, t, g * torch.logspace(-20, 0, rows, device="cuda"))
    check(x * torch.logspace(-20, 0, rows, device="cuda")[:, None].to(dtype), w, b, t, g * torch.logspace(0, -20, rows, device="cuda"))
    f = g.clone()
    f[::2] = 0.0
    check(x, w, b, t, f)
    check(x, w, b, t, f * 0)
    y = x.clone()
    y[1::2] = 0.0
    check(y, w, b, t, g)


@EACH
@TYPES
def test_weights_of_very_different_size(way, dtype):
    """The weight has one scale, or one for each line with bfloat16, and numbers of it keep 2^-39 of the largest under one."""
    x, w, b, t, g = make(way, dtype)
    d, V = w.shape
    check(x, w * torch.logspace(-4, 0, V, device="cuda").to(dtype), b, t, g)
    check(x, w * torch.logspace(-4, 0, d, device="cuda").to(dtype)[:, None], b, t, g)
    for k in (1e-20, 1e20, 1e-35, 1e33):                     # logits as they were, between numbers that are far from 1
        check(x * k, w / k, b, t, g)
    check(x * 0, w, b, t, g)
    check(x, w * 0, b, t, g)


@EACH
@TYPES
@pytest.mark.parametrize("reduction", ["sum", "mean"])
def test_rows_of_very_different_size_reduced(way, dtype, reduction):
    x, w, b, t, g = make(way, dtype, share=0.7)
    rows = x.shape[0]
    t[0] = 3
    x = x * torch.logspace(6, -8, rows, device="cuda")[:, None].to(dtype)
    takes(way, x, w, b, t, g, reduction=reduction)
    got = run(x, w, b, t, g, reduction=reduction)
    count = int((t >= 0).sum()) if reduction == "mean" else 1
    want = formula(x, w, b, t, (g[0] / count).expand(rows))
    assert abs(float(got[0]) - float(want[0][0].sum()) / count) <= float(want[0][1].sum()) / count + 4 * E * abs(float(got[0]))
    for name, a, (ref, tol, u) in zip(("dx", "dw", "db"), got[1:], want[1:]):
        assert ((a.cpu().double() - ref).abs() <= tol * (1 + u) + ref.abs() * (u + 2 * E) + 2.0 ** -126).all(), name


@EACH
@TYPES
def test_strides_types_and_axes(way, dtype):
    x, w, b, t, g = make(way, dtype, share=0.9)
    rows, d = x.shape
    wide = torch.randn(rows, 2 * d + 7, device="cuda").to(dtype)
    part = wide[:, 5:5 + d]                                  # rows far apart at odd addresses
    takes(way, part, w, b, t, g)
    want = check(part, w, b, t, g)
    for same in ((part, w.t().contiguous().t(), b, t, g),    # a transposed weight
                 (wide.repeat(2, 1)[:rows, 5:5 + d], w, b, torch.stack([t, t], 1)[:, 0], torch.stack([g, g], 1)[:, 1])):
        assert all(torch.equal(p, q) for p, q in zip(run(*same), want))
    check(x, w, b.float() if dtype == BF16 else b.bfloat16(), t, g)
    leaf = part.reshape(1, rows, 1, d).detach().requires_grad_(True)
    loss = layers.linear_cross_entropy(leaf, w, t.view(1, rows, 1).to(torch.int32), bias=b, reduction="none")
    assert loss.shape == (1, rows, 1) and torch.equal(loss.flatten(), want[0])
    assert torch.equal(torch.autograd.grad(loss, leaf, g.view(1, rows, 1))[0].view(rows, d), want[1])
    one = run(part, w, b, t, torch.ones((), device="cuda").expand(rows))         # one number for all rows
    assert all(torch.equal(p, q) for p, q in zip(one, run(part, w, b, t, torch.ones(rows, device="cuda"))))


@EACH
def test_differences(way):
    """The gradient along a direction is what the loss changes by: central differences in steps of 2^-6 are off by the third
    derivative's 2^-13 and 2^-15 of the losses (float32)."""
    x, w, b, t, g = make(way, F32, share=0.8)
    f = lambda *a: (layers.linear_cross_entropy(a[0], a[1], t, bias=a[2], reduction="none") * g).double().sum()       # noqa: E731
    leaves = [v.clone().requires_grad_(True) for v in (x, w, b)]
    grads = torch.autograd.grad(f(*leaves), leaves)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for i, v in enumerate((x, w, b)):
        dirn = torch.randn(v.shape, generator=gen, device="cuda") / v.numel() ** 0.5
        h = 2.0 ** -6
        p, m = ([a + s * h * dirn if k == i else a for k, a in enumerate((x, w, b))] for s in (1, -1))
        slope = float((f(*p) - f(*m)) / (2 * h))
        assert abs(slope - float((grads[i] * dirn).double().sum())) <= float(g.sum()) * 2.0 ** -9


@EACH
@TYPES
def test_only_what_is_asked_for(way, dtype):
    x, w, b, t, g = make(way, dtype, share=0.8)
    want = run(x, w, b, t, g)[1:]
    for need in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 0), (1, 0, 1), (0, 1, 1)):
        leaves = [v.clone().requires_grad_(bool(n)) for v, n in zip((x, w, b), need)]
        layers.linear_cross_entropy(leaves[0], leaves[1], t, bias=leaves[2], reduction="none").backward(g)
        assert all(torch.equal(v.grad, q) if n else v.grad is None for v, n, q in zip(leaves, need, want))


@EACH
@TYPES
@pytest.mark.parametrize("reduction", ["mean", "none"])
def test_graph_replayed(way, dtype, reduction):
    """A captured step, replayed on other inputs, factors and numbers of labelled rows, with work of its own between the replays."""
    x, w, b, t, g = make(way, dtype, share=0.5)
    X, W, B = (v.clone().requires_grad_(True) for v in (x, w, b))

    def step():
        loss = layers.linear_cross_entropy(X, W, t, bias=B, reduction=reduction)
        return (loss, *torch.autograd.grad(loss, (X, W, B), g if reduction == "none" else g[0]))

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for k, share in enumerate((1.0, 0.2, 0.0, 0.6, 1.0)):
        x, _, _, t2, g2 = make(way, dtype, share=share, seed=k + 1)
        with torch.no_grad():
            X.copy_(x * (torch.logspace(-6, 3, x.shape[0], device="cuda")[:, None] if k == 3 else 1.0))
        t.copy_(t2)
        g.copy_(g2 * torch.logspace(0, -9, g2.numel(), device="cuda") if k >= 3 else g2)
        graph.replay()
        torch.cuda.synchronize()
        mine = [v.clone() for v in got]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(mine, got)), share
        assert all(torch.equal(p, q) for p, q in zip(mine, step())), share


@EACH
def test_refusals(way):
    x, w, b, t, g = make(way, F32)
    L = layers.linear_cross_entropy
    for bad in ((x, w.t(), t), (x, w, t[:-1]), (x[:, :8], w, t), (x.cpu(), w, t), (x, w.cpu(), t), (x, w, t.cpu()), (x, w[0], t)):
        with pytest.raises(ValueError):
            L(*bad)
    for bad in ((x.half(), w.half(), t), (x.bfloat16(), w, t), (x, w, t.float()), (x, w, t.to(torch.int16))):
        with pytest.raises(TypeError):
            L(*bad)
    with pytest.raises(ValueError):
        L(x, w, t, bias=b[:2])
    x.requires_grad_(True)
    dx, = torch.autograd.grad(L(x, w, t), x, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(dx.sum(), x)
    w2 = w.clone().requires_grad_(True)
    loss = L(x, w2, t)
    with torch.no_grad():
        w2.mul_(2.0)
    with pytest.raises(RuntimeError):
        loss.backward()
