"""4-bit matrices at the ends of what a call takes: the largest groups, more rows than one launch holds, the largest and smallest values."""
import numpy as np
import pytest
import torch

from paper_2501_05370_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF = torch.float32, torch.bfloat16


def test_a_group_longer_than_any_row():
    """One scale per row, however large the group: the same bits as with the smallest group that holds the row."""
    rng = np.random.default_rng(0)
    K, N = 1000, 48
    q = rng.integers(0, 256, size=(N, K // 2), dtype=np.uint8)
    s = torch.from_numpy(rng.uniform(0.01, 0.1, size=(N, 1))).to(BF).view(torch.int16).numpy()
    x = torch.from_numpy(rng.standard_normal((7, K))).float().cuda()
    got = []
    for group in (1024, 1 << 20, (1 << 31) - 128):
        m = B.Q4Matrix.sdden_q4_create(q, s, K, group)
        y = torch.empty(7, N, device="cuda")
        m.sdden_q4_eval(x, y)
        got.append(y)
        m.close()
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


@pytest.mark.parametrize("K,N,tx,R", [(3, 5, F32, 45_000_000), (1, 8, BF, (1 << 27) + 77)])
def test_more_rows_than_a_launch_holds(K, N, tx, R):
    """2^24 workgroups of 256 threads hold 44 040 171 fp32 rows of up to 1024 columns, or 2^27 bf16 ones: what is more goes into
    another launch.  The rows repeat, so every one of them must have the first ones' results."""
    rng = np.random.default_rng(3)
    q = rng.integers(0, 256, size=(N, (K + 1) // 2), dtype=np.uint8)
    s = torch.from_numpy(rng.uniform(0.01, 0.1, size=(N, 1))).to(BF).view(torch.int16).numpy()
    m = B.Q4Matrix.sdden_q4_create(q, s, K, 32)
    period = 1009
    some = torch.from_numpy(rng.standard_normal((period, K))).to(tx).cuda()
    x = some.repeat(-(-R // period), 1)[:R]
    want, y = torch.empty(period, N, dtype=BF, device="cuda"), torch.full((R + 1, N), float("nan"), dtype=BF, device="cuda")
    m.sdden_q4_eval(some, want)
    m.sdden_q4_eval(x, y[:R])
    whole = R // period * period
    assert torch.equal(y[:whole].view(-1, period, N), want.expand(whole // period, period, N))
    assert torch.equal(y[whole:R], want[:R - whole]) and y[R].isnan().all()
    m.close()


def test_the_range_of_the_rows():
    """Rows of values just below 2^116 with the signs and levels that make a group's unscaled sum largest, single values where 24 |x| is
    just below 2^128, and small fp32 values of 24 bits down to 2^-103.  Roundings as in the products' own test: 8 of a block's
    instructions, one scaled add, 26 of shares, pieces and bias, each 2^-23 of sum (q + 8) |x| s at most."""
    K, N = 128, 32
    rng = np.random.default_rng(4)
    q = rng.integers(0, 16, size=(N, K), dtype=np.uint8)
    q[0], q[1], q[2] = 15, 0, 8
    s = torch.full((N, 1), 2.0 ** -9, dtype=BF)
    m = B.Q4Matrix.sdden_q4_create(q[:, 0::2] | (q[:, 1::2] << 4), s.view(torch.int16).numpy(), K, 128)
    level = torch.from_numpy(q.astype(np.float64))
    full = 1 + torch.from_numpy(rng.integers(0, 1 << 23, size=K) | 1).double() * 2.0 ** -23      # 24 bits, the last one set
    rows = [torch.full((K,), 2.0 ** 116 * (1 - 2.0 ** -8)), -torch.full((K,), 2.0 ** 116 * (1 - 2.0 ** -8)), full * 2.0 ** 114,
            full * 2.0 ** -102, full * 2.0 ** -103]
    one = torch.zeros(K, dtype=torch.float64)
    one[77] = 2.0 ** 123 * 1.25
    rows += [one, -one]
    x = torch.stack([r.double() for r in rows])
    for R in (len(rows), 5, 40, 130):
        for t in (F32, BF):
            xt = x.repeat(-(-R // len(rows)), 1)[:R].to(t).cuda()
            y = torch.empty(R, N, device="cuda")
            m.sdden_q4_eval(xt, y)
            xd = xt.double().cpu()
            want, terms = xd @ (level - 8).T * 2.0 ** -9, xd.abs() @ (level + 8).T * 2.0 ** -9
            assert bool(((y.double().cpu() - want).abs() <= 35 * 2.0 ** -23 * terms).all()), (R, t)
    m.close()
