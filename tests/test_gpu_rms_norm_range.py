"""rms_norm of rows at the end of float32's range: the squares' sum over many channels is no float, and neither is that of numbers that
were brought down by too little."""
import pytest
import torch

from paper_2202_08556_amd import layers

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("channels", [96, 4096, 16384, 16500, 131072, 1 << 20])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_rows_of_the_largest_numbers(channels, dtype):
    """All numbers are +-2^127: y is their sign times the weight.  A sum of C equal squares in chains of C / 1024 (a lane's) and a
    few steps that join them is off by (C / 1024 + 32) 2^-24 at most, y by half of that, three roundings more and that to its type;
    dw is a sum of three such rows."""
    g = torch.Generator(device="cuda").manual_seed(channels)
    sign = torch.where(torch.rand(3, channels, generator=g, device="cuda") < 0.5, -1.0, 1.0)
    sign[2] *= 2.0 ** -130                                   # ... and one of small ones
    x = (sign * 2.0 ** 127).to(dtype).requires_grad_(True)
    w = (torch.rand(channels, generator=g, device="cuda") + 0.5).to(dtype).requires_grad_(True)
    y = layers.rms_norm(x, w, eps=0.0)
    dw, = torch.autograd.grad(y, w, sign.sign().to(dtype))
    off = (channels / 1024 + 32) * 2.0 ** -25 + 4 * 2.0 ** -24 + (2.0 ** -8 if dtype == torch.bfloat16 else 0.0)
    want = sign.sign().double() * w.detach().double()
    assert ((y.detach().double() - want).abs() <= off * want.abs()).all()
    assert ((dw.double() - 3.0).abs() <= 3.0 * off).all()
    with torch.no_grad():
        q, scale = layers.rms_norm_e4m3(x, w, eps=0.0)
    # e4m3: half a step, 2^-4 of the number, or 2^-10 of the scale below its normal numbers
    tol = want.abs() * (2.0 ** -4 + off) + scale[:, None].double() * 2.0 ** -10
    assert ((q.float().double() * scale[:, None].double() - want).abs() <= tol).all()
