"""The gradients of a whole training step (norm, gated block, residual) against its formulas and against differences in fp64.

The comparison is by norm: LIMIT is derived beside the fp64 step, whose CPU tests show that every gradient with a term missing, doubled
or exchanged is several limits off.  The products' fp32 sums (up to 4600 roundings of 2^-24 of the sum of |terms|, which is
at most sqrt(4600) of the sum's norm: 0.019 if all went one way, and they go either way) stay far inside it."""
import pytest
import torch

from _layer_step import LIMIT, gradients, loss, problem, shares
from paper_2501_05370_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF = torch.float32, torch.bfloat16
ACT = {"silu": B.SDDEN_SILU, "gelu": B.SDDEN_GELU}
STEPS = [(1, 64, 128, "silu"), (24, 64, 96, "gelu"), (64, 136, 264, "silu"), (130, 136, 264, "gelu"), (700, 264, 520, "silu"),
         (4600, 520, 1032, "silu"), (1100, 1032, 2056, "gelu")]


def kernels(p, act):
    h, c, w, b, Wg, Wu, Wd = p
    R, d = h.shape
    H = Wg.shape[0]
    dev = lambda t, ty: t.to(ty).cuda()
    empty = lambda *n, t=F32: torch.empty(*n, dtype=t, device="cuda")
    hg, cg, cb, wt, bt = dev(h, F32), dev(c, F32), dev(c, BF), dev(w, F32), dev(b, F32)
    ws = [dev(t, BF) for t in (Wg, Wu, Wd)]
    x, mean, rstd, y = empty(R, d, t=BF), empty(R), empty(R), empty(R, d)
    hidden, gates, dx, dh, dw, db = empty(R, H, t=BF), empty(2, R, H), empty(R, d, t=BF), empty(R, d), empty(d), empty(d)
    dws = [empty(H, d), empty(H, d), empty(d, H)]
    scratch = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
    B.sdden_layernorm_forward(hg, wt, bt, 1e-5, x, mean, rstd)
    B.sdden_gated_forward(x, *ws, y, hidden, gates=gates, act=ACT[act], res=hg)
    B.sdden_gated_backward(cb, x, *ws, gates, hidden, dx, *dws, scratch(B.sdden_gated_workspace_bytes(R, d, H)), act=ACT[act])
    B.sdden_layernorm_backward(dx, hg, wt, mean, rstd, dh, dw, db, scratch(B.sdden_layernorm_workspace_bytes(R, d)), dres=cg)
    return [t.double().cpu() for t in (dh, dw, db, *dws)], dx.double().cpu(), y.double().cpu()


@pytest.mark.parametrize("R,d,H,act", STEPS)
def test_every_gradient_of_a_step(R, d, H, act):
    p = problem(R, d, H, R + d)
    got, dx, y = kernels(p, act)
    want = gradients(*p, act=act)
    far = shares(got, want, p[1])
    print(R, d, H, act, [f"{t:.4f}" for t in far], "limit", f"{LIMIT:.4f}")
    assert max(far) <= LIMIT
    # the norm's backward pass of the block's gradient as the block left it, element by element: fp32 only
    h, c, w = p[0], p[1], p[2]
    mean = h.mean(1, keepdim=True)
    r = ((h - mean).square().mean(1, keepdim=True) + 1e-5) ** -0.5
    xh, v = (h - mean) * r, dx * w
    dh = r * (v - v.mean(1, keepdim=True) - xh * (v * xh).mean(1, keepdim=True)) + c
    scale = r * v.abs().amax(1, keepdim=True) * (1 + xh.abs().amax(1, keepdim=True)) + c.abs()
    assert bool(((got[0] - dh).abs() <= 1e-5 * scale + 1e-7).all())
    # the value, whose gradients these are: sum(c y)
    assert abs(float((p[1] * y).sum() - loss(*p, act=act))) <= LIMIT * float(p[1].norm() * (y - h).norm()) + 1e-5 * float((p[1] * h).abs().sum())


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_slopes_along_the_right_gradient(act):
    """Central differences of the loss in fp64 along the right gradient v of each input: <got, v> is |v|^2 off by LIMIT of it at most
    (Cauchy-Schwarz), where a missing part would be missing with its own square."""
    p = problem(130, 136, 264, 5)
    got, _, _ = kernels(p, act)
    for at, g, v in zip((0, 2, 3, 4, 5, 6), got, gradients(*p, act=act)):
        if at == 0:                                  # the block's share alone: the residual's is exact, and larger
            v, g = v - p[1], g - p[1]
        t = 1e-4 / float(v.abs().max())
        moved = [list(p), list(p)]
        for m, s in zip(moved, (t, -t)):
            m[at] = p[at] + s * v
        slope = (loss(*moved[0], act=act) - loss(*moved[1], act=act)) / (2 * t)
        if at == 0:
            slope = slope - (p[1] * v).sum()
        square = float((v * v).sum())
        assert abs(float(slope) - square) <= 1e-4 * square
        assert abs(float((g * v).sum() - slope)) <= (LIMIT + 1e-4) * square
