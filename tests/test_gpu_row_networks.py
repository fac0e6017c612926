"""Denoisers made of the new layers: the MLP with 4-bit matrices and the residual gated network, against the fp64 oracle and
inside the samplers.

Tolerance 2e-2 of the row's scale, as for the bf16 MLP: bf16 rows and activations (2^-8 each, a handful one after the other),
fp32 sums; the 4-bit values themselves are the oracle's to the bit."""
import dataclasses

import numpy as np
import pytest
import torch

import workloads as W
from oracle import speculative as S
from oracle.denoisers import GatedDenoiser, MLPDenoiser, Q4MLPDenoiser

from _gpu import as_f32_f64, dev, f32, host, rel_err

pytestmark = pytest.mark.gpu
TOL = 2e-2


def check_rows(g, ref, d, T, sizes, reserved):
    """Masked rows stay as they are, results do not depend on the call's size, and agree with the oracle."""
    rng = np.random.default_rng(d)
    R = max(sizes)
    x = as_f32_f64(rng.standard_normal((R, d)))
    k = rng.integers(-2, T + 2, size=R).astype(np.int32)
    k[0] = T - 1
    live = (k >= 0) & (k < T)
    want = np.zeros((R, d))
    want[live] = ref(x[live], k[live])
    xg, kg = f32(x), dev(k, torch.int32)
    whole = torch.full((R, d), 777.0, device="cuda")
    g.sdden_eval(R, xg, kg, whole)
    got = host(whole)
    assert rel_err(got[live], want[live]) < TOL and np.all(got[~live] == 777.0)
    for r in sizes:
        out = torch.full((r, d), 777.0, device="cuda")
        g.sdden_eval(r, xg[:r], kg[:r], out)
        assert torch.equal(out, whole[:r]), r
        img = xg[:r].to(torch.bfloat16).view(torch.int16).contiguous()
        img[~dev(live[:r], torch.bool)] = 0x7fc0                     # masked rows carry NaN in the image
        out2 = torch.full((r, d), 777.0, device="cuda")
        g.sdden_eval_mirror(r, xg[:r], img, kg[:r], out2)
        assert torch.equal(out2, out), r
    # a device-side count: 3 of the chains of 4 rows
    r = min(R, 40)
    out = torch.full((r, d), 777.0, device="cuda")
    cnt = torch.tensor([3], dtype=torch.int32, device="cuda")
    g.sdden_set_active_count(cnt, 4)
    g.sdden_eval(r, xg[:r], kg[:r], out)
    g.sdden_set_active_count(None, 1)
    n = min(12, r)
    assert torch.equal(out[:n], whole[:n]) and bool((out[n:] == 777.0).all())
    out.fill_(777.0)
    g.sdden_eval(r, xg[:r], torch.full((r,), -1, dtype=torch.int32, device="cuda"), out)
    assert bool((out == 777.0).all())
    with pytest.raises(Exception, match="reserved"):
        g.sdden_eval(reserved + 1, torch.zeros(reserved + 1, d, device="cuda"),
                     torch.zeros(reserved + 1, dtype=torch.int32, device="cuda"), torch.zeros(reserved + 1, d, device="cuda"))


@pytest.mark.parametrize("d,H,E,group", [(256, 512, 16, 128), (200, 96, 8, 32), (37, 45, 0, 64), (1024, 384, 32, 256)])
def test_mlp_in_four_bits(d, H, E, group):
    from paper_2501_05370_amd.binding import Denoiser
    T = 21
    p = W.random_mlp(np.random.default_rng(3), d, H, E)
    g = Denoiser.sdden_mlp4_create(p, group, T, 300)
    check_rows(g, Q4MLPDenoiser(W.Q4MLPParams(p, group)), d, T, (1, 5, 16, 17, 33, 64, 65, 130, 300), 300)
    g.close()


@pytest.mark.parametrize("d,H,E,blocks,act", [(64, 128, 16, 3, 0), (200, 136, 8, 2, 1), (1032, 520, 0, 1, 0), (256, 512, 32, 2, 0)])
def test_gated_network(d, H, E, blocks, act):
    from paper_2501_05370_amd.binding import Denoiser
    T = 21
    p = W.random_gated(np.random.default_rng(5), d, H, blocks, E, act)
    g = Denoiser.sdden_gated_create(p, T, 700)
    check_rows(g, GatedDenoiser(p), d, T, (1, 2, 15, 16, 17, 33, 64, 129, 300, 700), 700)
    g.close()


def test_reserve_grows():
    from paper_2501_05370_amd.binding import Denoiser
    p, q = W.random_gated(np.random.default_rng(5), 64, 64, 1, 8), W.random_mlp(np.random.default_rng(3), 64, 64, 8)
    for g in (Denoiser.sdden_gated_create(p, 5, 2), Denoiser.sdden_mlp4_create(q, 32, 5, 2)):
        x, k = torch.randn(50, 64, device="cuda"), torch.zeros(50, dtype=torch.int32, device="cuda")
        a, b = torch.empty(2, 64, device="cuda"), torch.empty(50, 64, device="cuda")
        g.sdden_eval(2, x[:2], k[:2], a)
        torch.cuda.synchronize()
        g.sdden_reserve(50)
        g.sdden_eval(50, x, k, b)
        assert torch.equal(a, b[:2])


def _run(smp, B, **kw):
    out, counters = smp.run(torch.arange(B, dtype=torch.int64, device="cuda"), **kw)
    return out.clone(), counters


@pytest.mark.parametrize("kind", ["gated", "mlp4"])
def test_as_target_of_a_whole_run(kind):
    """Sampling from the first to the last step: all loops give the same bits, and a window agrees with the oracle's."""
    from paper_2501_05370_amd.runner import make_sampler
    cfg = W.make_config("c4", B=24, d=256, H=256, K=6, T=30)
    rng = np.random.default_rng(1)
    params = W.random_gated(rng, 256, 384, 2, 32) if kind == "gated" else W.Q4MLPParams(cfg.params, 64)
    cfg = dataclasses.replace(cfg, params=params)
    ref = GatedDenoiser(params) if kind == "gated" else Q4MLPDenoiser(params)
    out, counters = _run(make_sampler(cfg), cfg.B)
    assert counters[0] == cfg.B * cfg.T and bool(out.isfinite().all())
    for kw in (dict(windows_per_sync=3), dict(graph=True)):
        out2, counters2 = _run(make_sampler(cfg), cfg.B, **kw)
        assert torch.equal(out, out2) and counters2[:3] == counters[:3]
    smp = make_sampler(cfg)
    n = rng.integers(0, cfg.T, size=cfg.B)
    y = as_f32_f64(rng.standard_normal((cfg.B, cfg.d)))
    ids = np.arange(cfg.B, dtype=np.int64)
    b = smp.buf
    b.y.copy_(f32(y)); b.n.copy_(dev(n, torch.int32)); b.chain_id.copy_(dev(ids, torch.int64))
    smp.window(cfg.B)
    res, Ytil, Dq, D0, krow, _ = S.window(cfg.schedule, ref, y, n, ids, cfg.K, seed=cfg.seed)
    assert rel_err(host(b.D0), D0) < TOL and rel_err(host(b.Ytilde), Ytil) < TOL
    mask = np.zeros((cfg.B, cfg.K), dtype=bool)
    mask[:, 1:] = krow[:, :cfg.K - 1] >= 0
    assert rel_err(host(b.Dq)[mask], Dq[mask]) < 2 * TOL


def test_four_bit_draft_of_the_target():
    """The independent drafter with the target's own network in 4 bits: it has to draft better than a network that knows nothing of
    the target, and the chains end where the target's do on average."""
    from paper_2501_05370_amd.runner import make_sampler
    cfg = W.make_config("c4", B=32, d=256, H=256, K=6, T=40)
    drafts = {"other network": W.draft_params(cfg), "4 bits": W.Q4MLPParams(cfg.params, 32)}
    advance = {}
    for name, dp in drafts.items():
        out, c = _run(make_sampler(cfg, drafter="independent", draft_params=dp), cfg.B)
        assert c[0] == cfg.B * cfg.T and bool(out.isfinite().all())
        advance[name] = c[0] / c[1]
    print(f"mean advance per window: {advance}")
    assert advance["4 bits"] > advance["other network"]


def test_gated_network_as_draft():
    """A gated network whose blocks are switched off (zero last products) drafts as x + e_k, which the oracle predicts as well."""
    from paper_2501_05370_amd.runner import make_sampler
    cfg = W.make_config("c4", B=16, d=256, H=256, K=4, T=20)
    p = W.random_gated(np.random.default_rng(2), 256, 64, 1, 16)
    p.Wd[:] = 0
    smp = make_sampler(cfg, drafter="independent", draft_params=p)
    ref, refd = MLPDenoiser(cfg.params), GatedDenoiser(p)
    rng = np.random.default_rng(8)
    n = rng.integers(0, cfg.T, size=cfg.B)
    y, ids = as_f32_f64(rng.standard_normal((cfg.B, cfg.d))), np.arange(cfg.B, dtype=np.int64)
    b = smp.buf
    b.y.copy_(f32(y)); b.n.copy_(dev(n, torch.int32)); b.chain_id.copy_(dev(ids, torch.int64))
    smp.window(cfg.B)
    Ytil, mp, krow = S.draft_independent(cfg.schedule, refd, y, n, ids, cfg.K, cfg.seed)
    assert np.array_equal(host(b.krow), krow)
    assert rel_err(host(b.mp), mp) < 1e-5 and rel_err(host(b.Ytilde), Ytil) < 1e-5      # no bf16 on this path: x + e_k in fp32
    assert ref is not None
