"""orthogonalise of bfloat16 matrices is the formula's result with one rounding: nothing before it has fewer digits than float32's way.

Tolerance: with d the error before the rounding and r the distance of the exact result to the nearest bfloat16 number, a rounded number
is off by r(exact + d) + |d| <= r(exact) + 2 |d|.  d is what the float32 tests allow: 8 times the error of the formula in float32, and
2^-20 (Frobenius norms)."""
import pytest
import torch

from paper_2202_08556_amd import optim

from .gpu_util import kernels_of
from .test_gpu_orthogonalise import formula, momentum

pytestmark = pytest.mark.gpu


def check(g):
    got = optim.orthogonalise(g)
    want, plain = formula(g, torch.float64), formula(g, torch.float32)
    norms = lambda t: t.flatten(-2).norm(dim=-1)                        # noqa: E731
    rounding = norms(want.to(torch.bfloat16).double() - want)
    d = 8 * norms(plain.double() - want) + 2.0 ** -20 * norms(want)
    off = norms(got.double() - want)
    assert (off <= rounding + 2 * d).all(), (off / norms(want), rounding / norms(want), d / norms(want))


def signs(B, r, c, seed):
    """Numbers of one magnitude: what is lost of one of them is lost of all, and does not average out."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=gen, device="cuda").sign()              # noqa: E731
    return (n(B, r, 1) * n(B, 1, c)).to(torch.bfloat16)


SIZES = [(1, 71, 497), (1, 217, 269), (3, 125, 301), (1, 497, 71), (1, 300, 300), (12, 256, 1024), (1, 700, 2200), (1, 2100, 900), (1, 64, 256), (2, 300, 40)]


@pytest.mark.parametrize("B,r,c", SIZES)
def test_momentum(B, r, c):
    check(momentum(B, r, c, torch.bfloat16))


@pytest.mark.parametrize("B,r,c", SIZES)
def test_numbers_alike(B, r, c):
    g = signs(B, r, c, seed=r + c)
    check(g)
    check(g * torch.randn(g.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).sign())


@pytest.mark.parametrize("B,r,c", SIZES)
def test_few_directions(B, r, c):
    gen = torch.Generator(device="cuda").manual_seed(r + c)
    n = lambda *s: torch.randn(*s, generator=gen, device="cuda")         # noqa: E731
    one = n(B, r, 1) * n(B, 1, c)
    check((one + 1e-3 * n(B, r, c)).to(torch.bfloat16))
    check(torch.rand(B, r, c, generator=gen, device="cuda").to(torch.bfloat16))
    one = n(B, r, c) * 1e-3
    one[:, 0, 0] = 100.0
    check(one.to(torch.bfloat16))


def test_large():
    check(momentum(1, 2048, 4096, torch.bfloat16))           # tiles of 256


def test_repeats():
    """Parts of a sum are added in their order, whichever block comes last: the same bits every time."""
    junk = torch.randn(2000, 2000, device="cuda")
    for g in (momentum(12, 256, 1024, torch.bfloat16), momentum(1, 1000, 3000, torch.bfloat16), momentum(1, 1187, 602, torch.float32)):
        first = optim.orthogonalise(g)
        for _ in range(5):
            junk @ junk
            assert torch.equal(optim.orthogonalise(g), first)


def test_sizes_are_those_of_the_packed_products():
    for size, packed in (((1, 71, 497), True), ((1, 300, 300), True), ((1, 64, 256), False)):
        names = kernels_of(lambda: optim.orthogonalise(momentum(*size, torch.bfloat16)))
        assert any("plane_kernel" in n for n in names) == packed and any("orth_small_kernel" in n for n in names) != packed
