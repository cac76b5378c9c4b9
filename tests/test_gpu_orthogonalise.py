"""orthogonalise against its formula in 64 bits.

Tolerance: the relative error (Frobenius) of the same formula in float32 with torch's products, times 8, plus half a step of
the result's type.  The kernels' operands are pairs with 22 bits where float32 has 24, which makes each rounding four times as
large, and leave out the product of the second halves, once more as much; sums are in 32 bits in both.  How such errors grow from
step to step is the same.  A floor of 2^-20 covers matrices on which float32 makes next to no error (one row or column)."""
import pytest
import torch

from paper_2202_08556_amd import optim

pytestmark = pytest.mark.gpu
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def formula(g, dtype, steps=5, coefficients=optim.COEFFICIENTS, eps=1e-7):
    X = g.detach().to(dtype)
    tall = X.shape[-2] > X.shape[-1]
    X = X.mT.contiguous() if tall else X
    X = X / (g.detach().double().square().sum((-2, -1), keepdim=True).sqrt() + eps).to(dtype)
    triples = [coefficients] * steps if not hasattr(coefficients[0], "__len__") else coefficients
    for a, b, c in triples:
        A = X @ X.mT.contiguous()
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.mT.contiguous() if tall else X


def check(g, **kw):
    got = optim.orthogonalise(g, **kw)
    assert got.shape == g.shape and got.dtype == g.dtype and got.is_contiguous()
    want, plain = formula(g, torch.float64, **kw), formula(g, torch.float32, **kw)
    norm = want.flatten(-2).norm(dim=-1)
    off, off32 = ((t.double() - want).flatten(-2).norm(dim=-1) for t in (got, plain))
    assert torch.isfinite(got).all()
    assert (off <= 8 * off32 + (U[g.dtype] + 2.0 ** -20) * norm).all(), (off / norm, off32 / norm)
    return got


def momentum(B, r, c, dtype, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed + B + 3 * r + 7 * c)
    k = max(1, min(r, c) // 8)
    n = lambda *s: torch.randn(*s, generator=gen, device="cuda")          # noqa: E731
    g = 1e-3 * ((n(B, r, k).double() @ n(B, k, c).double()).float() / k ** 0.5 + 0.3 * n(B, r, c))
    return g.to(dtype)


SIZES = [(1, 1, 1), (1, 1, 7), (1, 5, 1), (1, 16, 16), (1, 64, 256), (1, 65, 129), (1, 63, 64), (3, 40, 100), (2, 100, 40), (1, 200, 1000), (1, 1187, 602),
         (12, 256, 1024), (48, 64, 64), (1, 130, 5000), (1, 5000, 130), (40, 250, 300), (1, 2100, 2200), (1, 300, 9000), (5, 1, 64), (70, 128, 512),
         (600, 64, 512), (3, 512, 64), (2, 64, 513), (2, 33, 470), (7, 500, 17), (1, 64, 65)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("B,r,c", SIZES)
def test_formula(B, r, c, dtype):
    check(momentum(B, r, c, dtype))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_large(dtype):
    check(momentum(1, 4100, 4200, dtype))                    # tiles of 256 for all three products


def test_singular_values():
    g = momentum(2, 96, 400, torch.float32)
    s = torch.linalg.svdvals(optim.orthogonalise(g).double().cpu())
    first = torch.linalg.svdvals(g.double().cpu())
    some = first > 0.01 * first.square().sum(-1, keepdim=True).sqrt()
    assert (s[some] > 0.6).all() and (s < 1.3).all()


@pytest.mark.parametrize("scale", [1e-38, 1e-25, 1e15, 1e36])
def test_scales(scale):
    """Squares that are no floats; the result does not depend on the scale (eps 0)."""
    g = momentum(1, 48, 96, torch.float32)
    g = g / g.abs().max()
    check(g * scale, eps=0.0)


def test_coefficients_and_steps():
    g = momentum(2, 60, 100, torch.float32)
    check(g, steps=0)
    check(g.transpose(1, 2), steps=0)
    assert torch.equal(optim.orthogonalise(g, steps=0, coefficients=[]), optim.orthogonalise(g, steps=0))
    check(g, steps=1)
    check(g, steps=8, coefficients=(1.5, -0.5, 0.0))
    check(g, steps=3, coefficients=[(4.0, -6.0, 3.0), (3.0, -3.2, 1.2), (1.9, -1.3, 0.4)])
    check(g, steps=2, coefficients=(0.0, 0.0, 0.0))
    check(g, steps=2, coefficients=(-2.0, 1.0, 0.0))
    check(g, steps=1, coefficients=(100.0, 0.0, 0.0))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_strides(dtype):
    wide = momentum(3, 70, 200, dtype)
    check(wide[:, :, 3:90])                                  # rows 200 apart, at odd addresses
    check(wide[:, ::2])
    check(wide[::2])
    check(wide[1])
    check(wide[1].t())
    check(wide[:, :64].transpose(1, 2))
    check(wide.view(3, 1, 70, 200).expand(3, 2, 70, 200))
    check(wide[:1].expand(4, 70, 200))


def test_zeros_and_bad_numbers():
    g = torch.zeros(4, 40, 70, device="cuda")
    g[1] = torch.randn(40, 70, device="cuda")
    g[2, 3, 5] = float("nan")
    g[3, 3, 5] = 2.0                                         # rank one
    out = optim.orthogonalise(g)
    assert not out[0].any() and torch.isfinite(out[1]).all() and out[2].isnan().all()
    check(g[3:])
    assert not torch.equal(out[3], torch.zeros_like(out[3]))


def test_empty():
    for shape in ((0, 4, 5), (2, 0, 5), (2, 4, 0)):
        assert optim.orthogonalise(torch.zeros(shape, device="cuda")).shape == shape


def test_refusals():
    g = torch.randn(8, 16, device="cuda")
    with pytest.raises(ValueError):
        optim.orthogonalise(g.cpu())
    with pytest.raises(ValueError):
        optim.orthogonalise(g[0])
    with pytest.raises(TypeError):
        optim.orthogonalise(g.half())
    with pytest.raises(ValueError):
        optim.orthogonalise(g, steps=-1)
    with pytest.raises(ValueError):
        optim.orthogonalise(g, steps=3, coefficients=[(1.0, 0.0, 0.0)])
    with pytest.raises(ValueError):
        optim.orthogonalise(g.clone().requires_grad_(True))
    from paper_2202_08556_amd import binding
    with pytest.raises(binding.DaSpmmError):
        optim.orthogonalise(g, coefficients=(3.0, 0.0, 0.0))
    with pytest.raises(ValueError):
        optim.OrthogonalMomentum([torch.nn.Parameter(torch.zeros(4, device="cuda"))])


def test_graph_and_streams():
    g = momentum(2, 200, 300, torch.bfloat16)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        optim.orthogonalise(g)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = optim.orthogonalise(g)
    for k in range(3):
        g.copy_(momentum(2, 200, 300, torch.bfloat16, seed=k))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, optim.orthogonalise(g)), k


def test_optimizer():
    """A step against its formula; weights of one shape go together and come to the same numbers as by themselves."""
    torch.manual_seed(0)
    shapes = [(64, 96), (64, 96), (96, 40), (3, 20, 30)]
    make = lambda: [torch.nn.Parameter(torch.randn(*s, device="cuda", generator=torch.Generator("cuda").manual_seed(i))) for i, s in enumerate(shapes)]     # noqa: E731
    params = make()
    opt = optim.OrthogonalMomentum(params, lr=0.1, momentum=0.9, weight_decay=0.01)
    want, kept = [p.detach().double() for p in params], [torch.zeros_like(p, dtype=torch.float64) for p in params]
    for step in range(3):
        for i, p in enumerate(params):
            p.grad = torch.randn(p.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(10 * step + i))
            kept[i] = 0.9 * kept[i] + p.grad.double()
            turned = formula(p.grad.double() + 0.9 * kept[i], torch.float64)
            want[i] = want[i] * (1 - 0.1 * 0.01) - 0.1 * max(1.0, p.shape[-2] / p.shape[-1]) ** 0.5 * turned
        opt.step()
    for p, w in zip(params, want):
        # three updates with entries below 1.3, each off by 1e-5 of its norm at most, times 0.1
        assert float((p.detach().double() - w).norm()) <= 3 * 0.1 * 1e-4 * float(w.numel()) ** 0.5 + 1e-6 * float(w.norm())
