"""The networks of layers in the sampler's other roles: target of the efficient frozen drafter, target and draft at once, one chain."""
import dataclasses

import numpy as np
import pytest
import torch

import workloads as W

pytestmark = pytest.mark.gpu


def _config(kind, B):
    cfg = W.make_config("c4", B=B, d=200, H=136, K=5, T=24)
    rng = np.random.default_rng(4)
    return cfg, dataclasses.replace(cfg, params={"gated": W.random_gated(rng, 200, 136, 2, 16, 1), "mlp4": W.Q4MLPParams(cfg.params, 64)}[kind])


@pytest.mark.parametrize("B", [1, 30])
@pytest.mark.parametrize("kind", ["gated", "mlp4"])
@pytest.mark.parametrize("drafter", ["efficient_frozen", "efficient_frozen_last_accepted", "independent"])
def test_every_loop_gives_the_same_chains(kind, drafter, B):
    """Eager windows, several to a readback, and replayed graphs: the same bits; the independent drafter drafts with the other kind."""
    from paper_2501_05370_amd.runner import make_sampler
    plain, cfg = _config(kind, B)
    kw = dict(drafter=drafter)
    if drafter == "independent":
        kw["draft_params"] = W.Q4MLPParams(plain.params, 32) if kind == "gated" else W.random_gated(np.random.default_rng(5), 200, 64, 1, 8)
    ids = torch.arange(B, dtype=torch.int64, device="cuda")
    runs = []
    for loop in (dict(), dict(windows_per_sync=3), dict(graph=True)):
        smp = make_sampler(cfg, **kw)
        for _ in range(2):                                   # a second run of the same sampler starts afresh
            out, counters = smp.run(ids, **loop)
            runs.append((out.clone(), counters))
    assert runs[0][1][0] == B * cfg.T and bool(runs[0][0].isfinite().all())
    for out, counters in runs[1:]:
        assert torch.equal(out, runs[0][0]) and counters[:3] == runs[0][1][:3]


def test_target_as_its_own_draft():
    """The same gated network drafts for itself: what it drafts is what the target predicts, so every draft is accepted."""
    from paper_2501_05370_amd.runner import make_sampler
    _, cfg = _config("gated", 16)
    out, c = make_sampler(cfg, drafter="independent", draft_params=cfg.params).run(torch.arange(16, dtype=torch.int64, device="cuda"))
    assert c[0] == 16 * cfg.T and c[2] == 0 and bool(out.isfinite().all())
