"""The gates' functions and their derivatives value by value, far into the tails, through the block's own entry points.

One hidden unit with u = 1 and dA = 1:  Y = f(g), dX = (f'(g), f(g)).  hidden, dG and dU are rounded to bf16 once (2^-8 of the
value; the outputs are those values themselves).  Before that the exponential carries its argument's rounding (relative, 1.5 |g| or
0.75 g^2 units of 2^-24 for e^-g and e^(-g^2 / 2)), erfc's argument likewise (g^2 units) and a handful of operations one each."""
import pytest
import torch

from paper_2501_05370_amd import binding as B

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def run(g, act):
    """g [R] of bf16 values -> Y[:, 0], dX[:, 0], dX[:, 1] in fp64."""
    R, d, H = g.numel(), 8, 8
    x = torch.zeros(R, d, dtype=BF, device="cuda")
    x[:, 0], x[:, 1] = g, 1
    wg, wu, wd, dy = (torch.zeros(s, dtype=BF, device="cuda") for s in ((H, d), (H, d), (d, H), (R, d)))
    wg[0, 0] = wu[0, 1] = wd[0, 0] = 1
    dy[:, 0] = 1
    y, hidden, gates, dx = torch.empty_like(x), torch.empty(R, H, dtype=BF, device="cuda"), torch.empty(2, R, H, device="cuda"), torch.empty_like(x)
    ws = torch.empty(B.sdden_gated_workspace_bytes(R, d, H), dtype=torch.uint8, device="cuda")
    B.sdden_gated_forward(x, wg, wu, wd, y, hidden, gates=gates, act=act)
    B.sdden_gated_backward(dy, x, wg, wu, wd, gates, hidden, dx, None, None, None, ws, act=act)
    return [t.double().cpu() for t in (y[:, 0], dx[:, 0], dx[:, 1])]


@pytest.mark.parametrize("R", [40, 3000])
def test_gelu(R):
    g = torch.linspace(-12, 8, R).to(BF)
    y, df, f = run(g.cuda(), B.SDDEN_GELU)
    v = g.double()
    P, p = torch.erfc(-v * 0.5 ** 0.5) / 2, torch.exp(-v * v / 2) / (2 * torch.pi) ** 0.5
    tol = 2.0 ** -8 + (2 * v * v + 16) * 2.0 ** -24
    for got in (y, f):
        assert bool(((got - v * P).abs() <= tol * (v * P).abs()).all())
    assert bool(((df - (P + v * p)).abs() <= 2.0 ** -8 * (P + v * p).abs() + (2 * v * v + 16) * 2.0 ** -24 * (P + v.abs() * p)).all())


@pytest.mark.parametrize("R", [40, 3000])
def test_silu(R):
    g = torch.linspace(-80, 40, R).to(BF)
    y, df, f = run(g.cuda(), B.SDDEN_SILU)
    v = g.double()
    s = torch.sigmoid(v)
    tol = 2.0 ** -8 + (2 * v.abs() + 16) * 2.0 ** -24
    for got in (y, f):
        assert bool(((got - v * s).abs() <= tol * (v * s).abs()).all())
    want = s + v * s * (1 - s)
    assert bool(((df - want).abs() <= 2.0 ** -8 * want.abs() + (2 * v.abs() + 16) * 2.0 ** -24 * (s + (v * s * (1 - s)).abs())).all())
