"""A call that fails leaves nothing behind for the next one to report."""
import numpy as np
import pytest
import torch

import workloads as W
from paper_2501_05370_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("what", ["gated", "mlp4", "mlp"])
def test_calls_after_one_that_ran_out_of_memory(what):
    """Room for 2^30 rows of 1024 values is refused by the device's allocator; a layer norm after it works and says so."""
    rng, rows = np.random.default_rng(0), 1 << 30
    with pytest.raises(B.SDError, match="memory"):
        if what == "gated":
            B.Denoiser.sdden_gated_create(W.random_gated(rng, 1024, 1024, 1, 2), 4, rows)
        elif what == "mlp4":
            B.Denoiser.sdden_mlp4_create(W.random_mlp(rng, 1024, 1024, 2), 32, 4, rows)
        else:
            B.Denoiser.sdden_mlp_create(W.random_mlp(rng, 1024, 1024, 2), 4, rows)
    x = torch.randn(3, 64, device="cuda")
    y = torch.empty_like(x)
    B.sdden_layernorm_forward(x, None, None, 1e-5, y)
    x64 = x.double()
    want = (x64 - x64.mean(1, keepdim=True)) / (x64.var(1, unbiased=False, keepdim=True) + 1e-5).sqrt()
    assert bool(((y.double() - want).abs() <= 1e-5 * want.abs().max()).all())


def test_the_gated_block_without_a_tensor_it_needs():
    """A missing tensor, or one of another shape, is named."""
    x, w, wd = torch.randn(4, 64, device="cuda").bfloat16(), torch.randn(16, 64, device="cuda").bfloat16(), torch.randn(64, 16, device="cuda").bfloat16()
    y, hidden, gates = torch.empty_like(x), torch.empty(4, 16, dtype=torch.bfloat16, device="cuda"), torch.empty(2, 4, 16, device="cuda")
    for name, args in (("Wg", (x, None, w, wd, y, hidden)), ("Wg", (x, w[0, 0], w, wd, y, hidden)), ("Wg", (x, w[0], w, wd, y, hidden)),
                       ("Wu", (x, w, None, wd, y, hidden)), ("Wd", (x, w, w, None, y, hidden)), ("Y", (x, w, w, wd, None, hidden)),
                       ("hidden", (x, w, w, wd, y, None)), ("X", (None, w, w, wd, y, hidden))):
        with pytest.raises(B.SDError, match=f"{name}:"):
            B.sdden_gated_forward(*args)
    ws = torch.empty(B.sdden_gated_workspace_bytes(4, 64, 16), dtype=torch.uint8, device="cuda")
    for name, args in (("Wg", (y, x, None, w, wd, gates, hidden)), ("dY", (None, x, w, w, wd, gates, hidden)), ("gates", (y, x, w, w, wd, None, hidden))):
        with pytest.raises(B.SDError, match=f"{name}:"):
            B.sdden_gated_backward(*args, torch.empty_like(x), None, None, None, ws)
