"""Every form in which the layers' kernels are built: widths, type pairs, accesses and output sizes of the norm, tiles and few-row forms
of the gated block, rows, groups and widths of the 4-bit products.  Tolerances are those of the layers' own tests, whose checks run
here on more sizes; the rest is compared bit by bit, as a row's result does not depend on the call it is part of."""
import itertools

import numpy as np
import pytest
import torch

import test_gpu_layers as layers
import test_gpu_q4 as q4
import test_gpu_row_networks as networks
import workloads as W
from oracle.denoisers import Q4MLPDenoiser
from paper_2501_05370_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF = torch.float32, torch.bfloat16
PAIRS = list(itertools.product((F32, BF), (F32, BF)))


@pytest.mark.parametrize("tx,ty", PAIRS)
@pytest.mark.parametrize("d", [64, 200, 1016, 1024, 2048, 8192, 12296, 16384, 16392, 20000])
def test_norm_of_every_width_with_wide_accesses(d, tx, ty):
    layers.test_norm_forward_and_backward(5, d, 8, tx, ty, True)


@pytest.mark.parametrize("tx,ty", PAIRS)
@pytest.mark.parametrize("d,pad", [(63, 0), (1023, 2), (2048, 1), (4095, 0), (8191, 0), (12288, 3), (12289, 0), (16381, 0), (16385, 0)])
def test_norm_of_every_width_element_by_element(d, pad, tx, ty):
    layers.test_norm_forward_and_backward(3, d, pad, tx, ty, True)


@pytest.mark.parametrize("tx,ty", PAIRS)
@pytest.mark.parametrize("d", [192, 1024, 4096, 12288, 16384])
def test_norm_outputs_past_the_caches(d, tx, ty):
    """Outputs above 32 MiB are stored in another way than smaller ones: the same bits as in calls of a few rows."""
    R = (9 << 20) * 2 // d                                  # 36 MiB of bf16, 72 of fp32
    gen = torch.Generator(device="cuda").manual_seed(d)
    rnd = lambda *n: torch.randn(*n, generator=gen, device="cuda")
    x, dy, dres = rnd(R, d).to(tx), rnd(R, d).to(ty), rnd(R, d).to(tx)
    w, b = 1 + 0.2 * rnd(d), rnd(d)

    def go(rows):
        n = x[rows].shape[0]
        y, dx = torch.full((n + 1, d), float("nan"), dtype=ty, device="cuda"), torch.full((n + 1, d), float("nan"), dtype=tx, device="cuda")
        mean, rstd, dw, db = (torch.empty(k, device="cuda") for k in (n, n, d, d))
        ws = torch.empty(B.sdden_layernorm_workspace_bytes(n, d), dtype=torch.uint8, device="cuda")
        B.sdden_layernorm_forward(x[rows], w, b, 1e-5, y[:n], mean, rstd)
        B.sdden_layernorm_backward(dy[rows], x[rows], w, mean, rstd, dx[:n], dw, db, ws, dres=dres[rows])
        assert bool(y[n].isnan().all()) and bool(dx[n].isnan().all()), "behind the last row nothing is written"
        return y[:n], dx[:n], mean, rstd, dw, db

    whole = go(slice(None))
    assert whole[0].numel() * whole[0].element_size() > 32 << 20 and whole[1].numel() * whole[1].element_size() > 32 << 20
    step = -(-R // 5)
    for at in range(0, R, step):
        rows = slice(at, min(R, at + step))
        for big, small in zip(whole[:4], go(rows)):
            assert torch.equal(big[rows], small)
    mean, rstd, dw, db = whole[2:]
    terms = dy.double() * ((x.double() - mean.double()[:, None]) * rstd.double()[:, None])
    # a partial row adds up R / 1024 rows (d <= 1024: a wavefront's share of four) or R / 512 at most, the partial rows 32 + 32 more;
    # a term carries three roundings
    roundings = -(-R // 512) + 64 + 3
    assert bool(((dw.double() - terms.sum(0)).abs() <= roundings * 2.0 ** -24 * terms.abs().sum(0)).all())
    assert bool(((db.double() - dy.double().sum(0)).abs() <= roundings * 2.0 ** -24 * dy.double().abs().sum(0)).all())


# few rows of more than 4096 outputs (several workgroups to a CU), tiles of 128 x 128 with two and with four stages
@pytest.mark.parametrize("R,d,H,pad,name,ty,with_res,tw",
                         [(R, 72, 4104, 0, "silu", F32, True, BF) for R in (1, 8, 9, 16, 17, 32, 33, 64)]
                         + [(R, 4104, 72, 8, "gelu", BF, False, F32) for R in (1, 4, 5, 16, 17, 32, 33, 64)]
                         + [(300, 2056, 4096, 0, "silu", F32, True, BF), (600, 2056, 4096, 8, "silu", BF, True, F32), (1000, 4224, 64, 0, "gelu", BF, False, BF)])
def test_gated_block_of_every_form(R, d, H, pad, name, ty, with_res, tw):
    layers.test_gated_forward_and_backward(R, d, H, pad, name, ty, with_res, tw)


@pytest.mark.parametrize("d,H", [(520, 2312), (4104, 72), (2056, 4096)])
def test_a_row_of_the_gated_block_does_not_depend_on_the_call(d, H):
    """Few-row forms, tiles of 64, 128 and 256: one chain over k in all of them."""
    gen = torch.Generator(device="cuda").manual_seed(d)
    rnd = lambda *n, s=1.0: (torch.randn(*n, generator=gen, device="cuda") * s).to(BF)
    R = 4600
    x, dy, wg, wu, wd = rnd(R, d), rnd(R, d), rnd(H, d, s=d ** -0.5), rnd(H, d, s=d ** -0.5), rnd(d, H, s=H ** -0.5)
    res = torch.randn(R, d, generator=gen, device="cuda")

    def go(n):
        y, hidden, gates, dx = torch.empty(n, d, device="cuda"), torch.empty(n, H, dtype=BF, device="cuda"), torch.empty(2, n, H, device="cuda"), torch.empty(n, d, dtype=BF, device="cuda")
        ws = torch.empty(B.sdden_gated_workspace_bytes(n, d, H), dtype=torch.uint8, device="cuda")
        B.sdden_gated_forward(x[:n], wg, wu, wd, y, hidden, gates=gates, res=res[:n])
        B.sdden_gated_backward(dy[:n], x[:n], wg, wu, wd, gates, hidden, dx, None, None, None, ws)
        return y, hidden, gates[0], gates[1], dx

    whole = go(R)
    for n in (1, 4, 5, 8, 9, 16, 17, 32, 33, 64, 65, 127, 129, 300, 513, 600, 1000, 2000):
        for part, full in zip(go(n), whole):
            assert torch.equal(part, full[:n]), n


@pytest.mark.parametrize("K,N", [(1100, 200), (515, 8208)])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("t", [F32, BF])
def test_4_bit_products_of_every_form(t, group, K, N):
    q4.test_a_row_does_not_depend_on_the_call(K, N, group, t)
    for R in (4, 6, 11, 22, 40, 200):
        q4.test_product(R, K, N, group, t, F32, True, 0)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("d,H", [(72, 96), (40, 8192)])
def test_4_bit_network_of_few_rows(d, H, group):
    """fp32 rows that the first product rounds itself, at both ends of every form of it, and 512 tiles of columns."""
    p = W.random_mlp(np.random.default_rng(6), d, H, 4)
    g = B.Denoiser.sdden_mlp4_create(p, group, 21, 70)
    networks.check_rows(g, Q4MLPDenoiser(W.Q4MLPParams(p, group)), d, 21, (1, 4, 5, 8, 9, 16, 17, 24, 25, 32, 33, 64, 70), 70)
    g.close()
