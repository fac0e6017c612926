"""Layer norm of rows far from zero: what is left after the mean has its digits.

x is given in fp32, so x - mean can be had to 2^-24 of itself however large the mean; a mean that is off by a few roundings of its own
size would show in every y.  Tolerance of y: 1e-5 of the row's largest value as in the layer's own test (two roundings of x - mean
and mean, rstd, two products, one sum: eight of 2^-24 = 5e-7, and the sums behind the statistics, relative to a variance that is a sum of
squares).  dx is computed with the mean as fp32 holds it, off by 2^-24 of the offset over the deviation."""
import pytest
import torch

from paper_2501_05370_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF = torch.float32, torch.bfloat16


@pytest.mark.parametrize("offset", [0.0, 30.0, -1e3, 1e5, 3e6])
@pytest.mark.parametrize("d", [16, 100, 1024, 1001, 4096, 12288, 12289, 16384, 40000])
def test_rows_far_from_zero(d, offset):
    gen = torch.Generator().manual_seed(d)
    R = 7
    x = (torch.randn(R, d, generator=gen, dtype=torch.float64) + offset).float()
    w, b = (1 + 0.2 * torch.randn(d, generator=gen)), torch.randn(d, generator=gen)
    y, mean, rstd = torch.empty(R, d, device="cuda"), torch.empty(R, device="cuda"), torch.empty(R, device="cuda")
    B.sdden_layernorm_forward(x.cuda(), w.cuda(), b.cuda(), 1e-5, y, mean, rstd)
    x64 = x.double()
    m = x64.mean(1, keepdim=True)
    r = ((x64 - m).square().mean(1, keepdim=True) + 1e-5) ** -0.5
    want = (x64 - m) * r * w.double() + b.double()
    assert bool(((y.double().cpu() - want).abs() <= 1e-5 * want.abs().amax(1, keepdim=True)).all())
    assert bool(((mean.double().cpu() - m[:, 0]).abs() <= 2.0 ** -23 * m[:, 0].abs() + 1e-6).all())
    assert bool(((rstd.double().cpu() / r[:, 0] - 1).abs() <= 1e-5).all())


def test_rows_of_one_value():
    """Nothing is left of them: y is the bias, whatever the value and however many of it are added up."""
    for d in (3, 1000, 4100, 20000):
        x = torch.tensor([0.1, -7.3, 1e6 / 3, 2.0 ** -40], device="cuda")[:, None].expand(4, d).contiguous()
        b = torch.randn(d, device="cuda")
        y = torch.empty_like(x)
        B.sdden_layernorm_forward(x, None, b, 1e-5, y)
        assert bool(((y - b).abs() <= 1e-5).all())
