"""4-bit matrices at the ends of what a call takes: the largest groups."""
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
