"""The oracle of the 4-bit and the gated network, pinned on sizes that can be written out by hand."""
import math

import numpy as np

import workloads as W
from oracle.denoisers import GatedDenoiser, Q4MLPDenoiser, quantize4


def test_quantisation_levels():
    W4 = np.array([[7.0, -7.0, 0.0], [3.4, -3.5, 0.0], [0.5, 1.5, 0.0], [-7.0, 3.0, 0.0]])
    out = quantize4(W4, 4)
    # scale 1 in both columns; halves to even (-3.5 -> -4, 0.5 -> 0, 1.5 -> 2); a column of zeros stays
    assert np.array_equal(out, np.array([[7, -7, 0], [3, -4, 0], [0, 2, 0], [-7, 3, 0]], float))
    # groups have scales of their own, the last one may be shorter
    out = quantize4(np.array([[7.0], [1.0], [14.0]]), 2)
    assert np.array_equal(out[:, 0], [7, 1, 14])
    # at most 16 levels per group and an error of at most half a step plus the scale's own rounding (2^-8 of up to 7 steps)
    rng = np.random.default_rng(0)
    w = rng.standard_normal((64, 5))
    q = quantize4(w, 32)
    for g in range(2):
        step = np.abs(w[32 * g:32 * g + 32].astype(np.float32)).max(0) / 7
        assert np.all(np.abs(q - w)[32 * g:32 * g + 32] <= (0.5 + 8 * 2 ** -8) * step)
        assert all(len(np.unique(q[32 * g:32 * g + 32, c])) <= 16 for c in range(5))


def test_q4_network_is_the_mlp_on_quantised_weights():
    p = W.random_mlp(np.random.default_rng(1), 6, 4, 2)
    x, k = np.random.default_rng(2).standard_normal((3, 6)), np.array([0, 1, 5])
    f = W.bf16_bits_to_f64
    W1 = f(p.W1)
    h = np.empty((3, 4))
    for r in range(3):
        emb = [math.sin(k[r]), math.cos(k[r])]
        h[r] = x[r] @ quantize4(W1[:6], 32) + emb @ W1[6:] + p.b1
    h = h / (1 + np.exp(-h))
    h = h @ quantize4(f(p.W2), 32) + p.b2
    h = h / (1 + np.exp(-h))
    assert np.allclose(Q4MLPDenoiser(W.Q4MLPParams(p, 32))(x, k), h @ quantize4(f(p.W3), 32) + p.b3, rtol=1e-12)


def test_gated_network_by_hand():
    for act in (0, 1):
        p = W.random_gated(np.random.default_rng(3), 8, 8, 2, 2, act)
        x, k = np.random.default_rng(4).standard_normal((2, 8)), np.array([3, 0])
        f = W.bf16_bits_to_f64
        for r in range(2):
            h = x[r] + p.be + math.sin(k[r]) * f(p.We)[0] + math.cos(k[r]) * f(p.We)[1]
            for l in range(2):
                m = sum(h) / 8
                v = sum((t - m) ** 2 for t in h) / 8
                n = (h - m) / math.sqrt(v + p.eps) * p.norm_weight[l] + p.norm_bias[l]
                a = np.empty(8)
                for j in range(8):
                    g, u = f(p.Wg)[l, j] @ n, f(p.Wu)[l, j] @ n
                    a[j] = u * (g / (1 + math.exp(-g)) if act == 0 else g * 0.5 * (1 + math.erf(g / math.sqrt(2))))
                h = h + f(p.Wd)[l] @ a
            assert np.allclose(GatedDenoiser(p)(x[r:r + 1], k[r:r + 1])[0], h, rtol=1e-12)
