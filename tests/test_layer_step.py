"""The fp64 step that the kernels' gradients are compared with: against automatic differentiation and differences, and that the
comparison finds a mistake where one is planted in it."""
import pytest
import torch

from _layer_step import LIMIT, MISTAKES, gradients, loss, problem, shares


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_formulas_against_differentiation(act):
    p = [t.requires_grad_() for t in problem(7, 24, 40, 1)]
    loss(*p, act=act).backward()
    want = [p[0].grad, p[2].grad, p[3].grad, p[4].grad, p[5].grad, p[6].grad]
    for g, w in zip(gradients(*[t.detach() for t in p], act=act), want):
        assert torch.allclose(g, w, rtol=1e-10, atol=1e-12)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_roundings_stay_within_the_limit(act):
    p = problem(130, 136, 264, 2)
    assert max(shares(gradients(*p, act=act, rounded=True), gradients(*p, act=act), p[1])) <= LIMIT


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("mistake", MISTAKES)
def test_mistakes_do_not(mistake, act):
    """Each moves the rows' gradient by several limits at least, roundings or not."""
    p = problem(130, 136, 264, 2)
    want = gradients(*p, act=act)
    for rounded in (False, True):
        assert shares(gradients(*p, act=act, mistake=mistake, rounded=rounded), want, p[1])[0] > 2 * LIMIT

