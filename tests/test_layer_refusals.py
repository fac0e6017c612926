"""More of what the layer calls refuse on the host: buffers off their element type's alignment."""
import pytest

from paper_2501_05370_amd import binding as B

P = 1 << 20          # an aligned address that no refused call touches


def err():
    return B.load_library().sdden_last_error(None).decode()


@pytest.mark.parametrize("kw", [dict(mean=P + 2), dict(rstd=P + 1)])
def test_norm_forward_refuses_misaligned_statistics(kw):
    v = dict(mean=P, rstd=P)
    v.update(kw)
    rc = B.load_library().sdden_layernorm_forward(4, 64, P, 0, 64, P, P, 1e-5, P, 0, 64, v["mean"], v["rstd"], None)
    assert rc == -1 and "sdden_layernorm_forward" in err() and "aligned" in err()


@pytest.mark.parametrize("kw", [dict(mean=P + 1), dict(rstd=P + 2), dict(dw=P + 2), dict(db=P + 3), dict(w=P + 1), dict(dy=P + 2)])
def test_norm_backward_refuses_misaligned_buffers(kw):
    v = dict(dy=P, w=P, mean=P, rstd=P, dw=P, db=P)
    v.update(kw)
    rc = B.load_library().sdden_layernorm_backward(4, 64, v["dy"], 0, 64, P, 0, 64, v["w"], v["mean"], v["rstd"], None, 0, P, 64, v["dw"],
                                                   v["db"], P, 1 << 30, None)
    assert rc == -1 and "sdden_layernorm_backward" in err() and "aligned" in err()


@pytest.mark.parametrize("d", [1, 64, 1024])
def test_norm_workspace_of_any_number_of_rows(d):
    """1024 partial rows of two sums at most, up to the largest number that the argument holds."""
    for R in (5000, (1 << 30) - 1, 1 << 30, (1 << 31) - 3, (1 << 31) - 1):
        assert B.sdden_layernorm_workspace_bytes(R, d) == 1024 * d * 8
    assert [B.sdden_layernorm_workspace_bytes(R, d) // (8 * d) for R in (1, 4, 5, 8, 9)] == [1, 1, 2, 2, 3]
