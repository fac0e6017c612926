"""The layers on rows that lie gigabytes apart (offsets past 2^31 elements and 2^32 bytes) and on several streams at once."""
import numpy as np
import pytest
import torch

from paper_2501_05370_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF = torch.float32, torch.bfloat16


def far(rows, stride, width, dtype, gen):
    """`rows` rows of `width` random values, `stride` elements apart, and the same rows close together."""
    near = torch.randn(rows, width, generator=gen).to(dtype).cuda()
    base = torch.empty((rows - 1) * stride + width, dtype=dtype, device="cuda")
    wide = base.as_strided((rows, width), (stride, 1))
    wide.copy_(near)
    return wide, near


def test_norm_of_rows_far_apart():
    gen = torch.Generator().manual_seed(1)
    R, d, stride = 70, 1000, 40_000_000                       # 2.8e9 elements from the first to the last row
    x, xn = far(R, stride, d, BF, gen)
    w, b = torch.randn(d, generator=gen).cuda(), torch.randn(d, generator=gen).cuda()
    y, yn = x, torch.empty(R, d, dtype=BF, device="cuda")
    mean, rstd = torch.empty(R, device="cuda"), torch.empty(R, device="cuda")
    B.sdden_layernorm_forward(xn, w, b, 1e-5, yn, mean, rstd)
    out = torch.empty(R, d, dtype=BF, device="cuda")
    B.sdden_layernorm_forward(x, w, b, 1e-5, out)
    assert torch.equal(out, yn)
    dx, dxn = torch.empty(R, d, dtype=BF, device="cuda"), torch.empty(R, d, dtype=BF, device="cuda")
    dy = torch.randn(R, d, generator=gen).cuda()
    B.sdden_layernorm_backward(dy, x, w, mean, rstd, dx)
    B.sdden_layernorm_backward(dy, xn, w, mean, rstd, dxn)
    assert torch.equal(dx, dxn)
    B.sdden_layernorm_forward(xn, w, b, 1e-5, y)                # and written far apart
    assert torch.equal(y, yn)


@pytest.mark.parametrize("R", [40, 300])
def test_gated_block_of_rows_far_apart(R):
    gen = torch.Generator().manual_seed(2)
    d, H, stride = 64, 72, 1 << 23
    x, xn = far(R, stride, d, BF, gen)
    wg, wu = torch.randn(H, d, generator=gen).to(BF).cuda(), torch.randn(H, d, generator=gen).to(BF).cuda()
    wd = torch.randn(d, H, generator=gen).to(BF).cuda()
    res = []
    for rows in (x, xn):
        y, hid, gates = torch.empty(R, d, device="cuda"), torch.empty(R, H, dtype=BF, device="cuda"), torch.empty(2, R, H, device="cuda")
        B.sdden_gated_forward(rows, wg, wu, wd, y, hid, gates=gates)
        dx, dws = torch.empty(R, d, dtype=BF, device="cuda"), [torch.empty(s, device="cuda") for s in ((H, d), (H, d), (d, H))]
        ws = torch.empty(B.sdden_gated_workspace_bytes(R, d, H), dtype=torch.uint8, device="cuda")
        B.sdden_gated_backward(rows, rows, wg, wu, wd, gates, hid, dx, *dws, ws)
        res.append([y, hid, gates, dx] + dws)
    assert all(torch.equal(a, b) for a, b in zip(*res))


@pytest.mark.parametrize("R", [3, 40, 100])
def test_q4_product_of_rows_far_apart(R):
    gen = torch.Generator().manual_seed(3)
    K, N = 130, 40
    rng = np.random.default_rng(0)
    m = B.Q4Matrix.sdden_q4_create(rng.integers(0, 256, size=(N, K // 2), dtype=np.uint8),
                                   torch.rand(N, 2, generator=gen).to(BF).view(torch.int16).numpy(), K, 128)
    x, xn = far(R, 3_000_000_001 // (R - 1), K, BF, gen)       # an odd stride: rows of every alignment
    y, yn = torch.empty(R, N, device="cuda"), torch.empty(R, N, device="cuda")
    m.sdden_q4_eval(x, y)
    m.sdden_q4_eval(xn, yn)
    assert torch.equal(y, yn)


def test_two_steps_at_once_on_two_streams():
    """The same weights, rows and buffers of their own: two training steps that overlap give what they give alone."""
    gen = torch.Generator().manual_seed(4)
    R, d, H = 700, 264, 520
    wg, wu = ((torch.randn(H, d, generator=gen) * d ** -0.5).to(BF).cuda() for _ in range(2))
    wd = (torch.randn(d, H, generator=gen) * H ** -0.5).to(BF).cuda()
    w, b = torch.ones(d, device="cuda"), torch.zeros(d, device="cuda")

    def make(seed):
        g = torch.Generator().manual_seed(seed)
        s = dict(h=torch.randn(R, d, generator=g).cuda(), dy=torch.randn(R, d, generator=g).to(BF).cuda())
        s.update(x=torch.empty(R, d, dtype=BF, device="cuda"), mean=torch.empty(R, device="cuda"), rstd=torch.empty(R, device="cuda"),
                 y=torch.empty(R, d, device="cuda"), hid=torch.empty(R, H, dtype=BF, device="cuda"), gates=torch.empty(2, R, H, device="cuda"),
                 dx=torch.empty(R, d, dtype=BF, device="cuda"), dh=torch.empty(R, d, device="cuda"), dw=torch.empty(d, device="cuda"),
                 db=torch.empty(d, device="cuda"), dwg=torch.empty(H, d, device="cuda"), dwu=torch.empty(H, d, device="cuda"),
                 dwd=torch.empty(d, H, device="cuda"))
        s["ws"] = torch.empty(B.sdden_gated_workspace_bytes(R, d, H), dtype=torch.uint8, device="cuda")
        s["ws2"] = torch.empty(B.sdden_layernorm_workspace_bytes(R, d), dtype=torch.uint8, device="cuda")
        return s

    def step(s):
        B.sdden_layernorm_forward(s["h"], w, b, 1e-5, s["x"], s["mean"], s["rstd"])
        B.sdden_gated_forward(s["x"], wg, wu, wd, s["y"], s["hid"], gates=s["gates"], res=s["h"])
        B.sdden_gated_backward(s["dy"], s["x"], wg, wu, wd, s["gates"], s["hid"], s["dx"], s["dwg"], s["dwu"], s["dwd"], s["ws"])
        B.sdden_layernorm_backward(s["dx"], s["h"], w, s["mean"], s["rstd"], s["dh"], s["dw"], s["db"], s["ws2"])

    outs = ("y", "hid", "dx", "dh", "dw", "db", "dwg", "dwu", "dwd")
    alone = []
    for seed in (1, 2):
        s = make(seed)
        step(s)
        torch.cuda.synchronize()
        alone.append([s[k].clone() for k in outs])
    states, streams = [make(1), make(2)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, st in zip(states, streams):
            with torch.cuda.stream(st):
                step(s)
    torch.cuda.synchronize()
    for s, want in zip(states, alone):
        assert all(torch.equal(s[k], t) for k, t in zip(outs, want))


def test_more_rows_than_a_call_takes_are_refused():
    """The library's sizes are 32 bits wide: more must not be taken for what is left of them."""
    x = torch.empty((1 << 30) + 1, 1, dtype=BF, device="cuda")
    with pytest.raises(B.SDError, match="2\\^30"):
        B.sdden_layernorm_forward(x, None, None, 1e-5, x)
    with pytest.raises(B.SDError, match="2\\^30"):
        B.sdden_layernorm_forward(x.view(1, -1), None, None, 1e-5, x.view(1, -1))
