"""The layers at the ends of what a call takes: rows wider than one launch's workgroups."""
import pytest
import torch

from paper_2501_05370_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF = torch.float32, torch.bfloat16


@pytest.mark.parametrize("d", [(1 << 25) + 5, (1 << 27) + 40])
def test_weight_gradients_of_the_widest_rows(d):
    """From 2^25 columns on the workgroups that add the partial rows up walk the columns (a launch holds fewer than 2^27 of them at 32
    columns each).  A term dy (x - mean) rstd carries three roundings and the sum of the two rows one."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    R = 2
    x, dy = (torch.randn(R, d, generator=gen, device="cuda").to(BF) for _ in range(2))
    mean, rstd = torch.tensor([0.25, -0.5], device="cuda"), torch.tensor([1.5, 0.75], device="cuda")
    dx, dw, db = torch.empty(R, d, dtype=BF, device="cuda"), torch.full((d,), float("nan"), device="cuda"), torch.full((d,), float("nan"), device="cuda")
    ws = torch.empty(B.sdden_layernorm_workspace_bytes(R, d), dtype=torch.uint8, device="cuda")
    B.sdden_layernorm_backward(dy, x, None, mean, rstd, dx, dw, db, ws)
    terms = (x.double() - mean.double()[:, None]) * rstd.double()[:, None] * dy.double()
    assert bool(((dw.double() - terms.sum(0)).abs() <= 4 * 2.0 ** -24 * terms.abs().sum(0)).all())
    assert bool(((db.double() - dy.double().sum(0)).abs() <= 2.0 ** -24 * dy.double().abs().sum(0)).all())
    assert bool(dx.isfinite().all())
