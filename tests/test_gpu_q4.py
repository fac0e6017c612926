"""Products of rows with 4-bit matrices against plain fp64 sums.

Tolerance: every product q x is exact in the fp32 sums (4 + 8 bits).  A term goes through at most 8 matrix instructions of its
group (4 that sum -8 x, 4 that sum q x, each rounding or cutting once, by at most 2^-23 of the sum of |terms|), one scaled add
per group of 128 k or less, and at most 24 adds of wavefronts and pieces, the bias and the scaling: ``roundings``.  The
terms are (q + 8) |x| s, as the -8 enters by itself.  An fp32 row is three bf16 pieces: exact.  bf16 outputs add 2^-8 of the value.
"""
import numpy as np
import pytest
import torch

from paper_2501_05370_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF = torch.float32, torch.bfloat16


def roundings(K, group):
    return 8 + -(-K // min(group, 128)) + 26


def matrix(rng, N, K, group):
    q = rng.integers(0, 16, size=(N, K), dtype=np.uint8)
    q[rng.random((N, K)) < 0.05] = 0
    padded = np.concatenate([q, np.full((N, K % 2), 15, np.uint8)], axis=1)      # the unused half byte holds anything
    packed = (padded[:, 0::2] | (padded[:, 1::2] << 4)).astype(np.uint8)
    groups = -(-K // group)
    scale = torch.from_numpy(rng.uniform(0.002, 0.05, size=(N, groups)) * rng.choice([-1.0, 1.0], size=(N, groups))).to(BF)
    W = (q.astype(np.float64) - 8) * np.repeat(scale.double().numpy(), group, axis=1)[:, :K]
    T = (q.astype(np.float64) + 8) * np.abs(np.repeat(scale.double().numpy(), group, axis=1)[:, :K])
    return packed, scale.view(torch.int16).numpy(), torch.from_numpy(W), torch.from_numpy(T)


CASES = [  # R, K, N, group, x, y, bias, pad
    (1, 1, 1, 32, F32, F32, True, 0), (1, 128, 16, 128, BF, BF, False, 0), (1, 129, 17, 32, F32, F32, True, 3),
    (2, 256, 40, 64, BF, F32, True, 0), (5, 1001, 333, 32, F32, F32, True, 0), (6, 1001, 33, 64, F32, BF, False, 1),
    (10, 640, 128, 128, F32, F32, True, 4), (11, 640, 128, 256, F32, F32, True, 4), (16, 2048, 64, 128, BF, BF, True, 8),
    (17, 2048, 72, 64, BF, F32, False, 0), (21, 384, 48, 32, F32, BF, True, 0), (22, 384, 48, 32, F32, BF, True, 0),
    (32, 500, 100, 500 // 4 // 32 * 128 or 128, BF, F32, True, 0), (33, 1024, 200, 1024, BF, BF, True, 0), (64, 4096, 112, 128, BF, F32, True, 0),
    (65, 130, 129, 64, BF, F32, True, 0), (42, 256, 256, 128, F32, F32, False, 0), (43, 255, 257, 32, F32, F32, True, 2),
    (128, 1024, 144, 128, BF, BF, False, 0), (129, 1023, 131, 32, BF, F32, True, 0), (300, 896, 320, 64, F32, BF, True, 0),
    (513, 384, 264, 128, BF, F32, True, 8), (1000, 96, 24, 32, BF, BF, True, 0),
]


@pytest.mark.parametrize("R,K,N,group,tx,ty,bias,pad", CASES)
def test_product(R, K, N, group, tx, ty, bias, pad):
    rng = np.random.default_rng(R * 1000003 + K * 101 + N)
    q, scale, W, T = matrix(rng, N, K, group)
    m = B.Q4Matrix.sdden_q4_create(q, scale, K, group)
    x = torch.full((R, K + pad), float("nan"), dtype=tx, device="cuda")[:, :K]
    x.copy_(torch.from_numpy(rng.standard_normal((R, K)) + 0.5))
    b = torch.from_numpy(rng.standard_normal(N)).float().cuda() if bias else None
    full = torch.full((R, N + pad), float("nan"), dtype=ty, device="cuda")
    y = full[:, :N]
    m.sdden_q4_eval(x, y, bias=b)
    xd = x.double().cpu()
    want = xd @ W.T + (0 if b is None else b.double().cpu())
    terms = xd.abs() @ T.T + (0 if b is None else b.double().cpu().abs())
    tol = roundings(K, group) * 2.0 ** -23 * terms + (2.0 ** -8 * want.abs() if ty is BF else 0) + 1e-30
    off = ((y.double().cpu() - want).abs() / tol).max()
    assert off <= 1, f"{float(off):.2f} of the bound"
    assert full[:, N:].isnan().all(), "between the rows nothing is written"
    y2 = torch.empty(R, N, dtype=ty, device="cuda")
    m.sdden_q4_eval(x, y2, bias=b)
    assert torch.equal(y, y2)
    m.close()


def test_every_level_and_scale_is_exact():
    """One-hot rows pick single weights out: (q - 8) s must come back to the bit."""
    K, N = 128, 32
    rng = np.random.default_rng(0)
    q, scale, W, _ = matrix(rng, N, K, 32)
    assert len(np.unique(q)) > 100
    m = B.Q4Matrix.sdden_q4_create(q, scale, K, 32)
    x = torch.eye(K, device="cuda")
    for R in (5, 20, 128):
        for t in (F32, BF):
            y = torch.empty(R, N, device="cuda")
            m.sdden_q4_eval(x[:R].to(t), y)
            assert torch.equal(y.double().cpu(), W.T[:R])


def test_rows_do_not_touch_each_other_and_none_is_fine():
    rng = np.random.default_rng(1)
    K, N = 200, 40
    q, scale, _, _ = matrix(rng, N, K, 64)
    m = B.Q4Matrix.sdden_q4_create(q, scale, K, 64)
    for R in (4, 70):
        for t in (F32, BF):
            x = torch.randn(R, K, device="cuda").to(t)
            y, y2 = torch.empty(R, N, device="cuda"), torch.empty(R, N, device="cuda")
            m.sdden_q4_eval(x, y)
            x[2, 7] = float("inf")
            x[1, 3] = float("nan")
            m.sdden_q4_eval(x, y2)
            keep = [i for i in range(R) if i not in (1, 2)]
            assert torch.equal(y[keep], y2[keep]) and y2[1].isnan().all() and y2[2].isnan().all()
    m.sdden_q4_eval(torch.empty(0, K, device="cuda"), torch.empty(0, N, device="cuda"))


def test_streams_and_graphs_share_a_matrix():
    rng = np.random.default_rng(2)
    K, N = 512, 96
    q, scale, _, _ = matrix(rng, N, K, 128)
    m = B.Q4Matrix.sdden_q4_create(q, scale, K, 128)
    sides = [torch.cuda.Stream() for _ in range(2)]
    xs = [torch.randn(R, K, device="cuda") for R in (3, 100)]
    ys = [torch.empty(x.shape[0], N, device="cuda") for x in xs]
    want = []
    for x in xs:
        y = torch.empty(x.shape[0], N, device="cuda")
        m.sdden_q4_eval(x, y)
        want.append(y)
    torch.cuda.synchronize()
    for s, x, y in zip(sides, xs, ys):
        with torch.cuda.stream(s):
            m.sdden_q4_eval(x, y)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ys, want))
    graphs = []
    for x, y in zip(xs, ys):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            m.sdden_q4_eval(x, y)
        graphs.append(g)
    for _ in range(3):
        for x in xs:
            x.normal_()
        want = []
        for x in xs:
            y = torch.empty(x.shape[0], N, device="cuda")
            m.sdden_q4_eval(x, y)
            want.append(y)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ys, want))


@pytest.mark.parametrize("K,N,group,t", [(1100, 200, 32, BF), (1100, 200, 128, F32), (515, 8208, 64, BF), (515, 8208, 128, F32)])
def test_a_row_does_not_depend_on_the_call(K, N, group, t):
    """Row counts at the edges of every kernel and of its rows per lane: the same bits as in one large call."""
    rng = np.random.default_rng(5)
    q, scale, _, _ = matrix(rng, N, K, group)
    m = B.Q4Matrix.sdden_q4_create(q, scale, K, group)
    x = torch.randn(600, K, device="cuda").to(t)
    whole = torch.empty(600, N, device="cuda")
    m.sdden_q4_eval(x, whole)
    for R in (1, 4, 5, 6, 8, 9, 10, 11, 16, 17, 21, 22, 24, 25, 32, 33, 42, 43, 64, 65, 128, 129, 192, 193, 300):
        y = torch.full((R, N), float("nan"), device="cuda")
        m.sdden_q4_eval(x[:R], y)
        assert torch.equal(y, whole[:R]), R
