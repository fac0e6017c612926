"""The 4-bit network takes finite weights only: quantised, an infinity or a NaN would become an ordinary number."""
import numpy as np
import pytest

import workloads as W
from paper_2501_05370_amd import binding as B


@pytest.mark.parametrize("bits", [0x7FC0, 0xFFC1, 0x7F80, 0xFF80, 0x7F81])
@pytest.mark.parametrize("name,at", [("W1", (0, 0)), ("W1", (7, 11)), ("W2", (11, 11)), ("W3", (5, 7))])
def test_weights_that_are_not_finite_are_refused(name, at, bits):
    p = W.random_mlp(np.random.default_rng(0), 8, 12, 2)
    getattr(p, name)[at] = bits
    with pytest.raises(B.SDError, match=f"{name} has weights that are not finite"):
        B.Denoiser.sdden_mlp4_create(p, 32, 4, 4)


@pytest.mark.parametrize("where", ["largest", "embedding", "b2"])
def test_other_values_are_not(where):
    """The largest finite weights, and a NaN in what stays as it is, are taken (and fail only for want of a GPU, where there is none)."""
    p = W.random_mlp(np.random.default_rng(0), 8, 12, 2)
    if where == "largest":
        p.W2[0, :2] = 0x7F7F, 0xFF7F
    elif where == "embedding":
        p.W1[8:] = 0x7FC0
    else:
        p.b2 = np.full(12, np.nan)
    try:
        B.Denoiser.sdden_mlp4_create(p, 32, 4, 4).close()
    except B.SDError as e:
        assert "failed (-4)" in str(e)
