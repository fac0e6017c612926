"""What the layer calls refuse, on the host and before anything is enqueued: no GPU is needed."""
import ctypes

import pytest
import torch

from paper_2501_05370_amd import binding as B

P = 1 << 20          # an aligned address that no refused call touches


def err():
    return B.load_library().sdden_last_error(None).decode()


def norm_fwd(R=4, d=64, x=P, tx=0, xs=64, w=P, b=P, eps=1e-5, y=P, ty=0, ys=64, mean=P, rstd=P):
    return B.load_library().sdden_layernorm_forward(R, d, x, tx, xs, w, b, eps, y, ty, ys, mean, rstd, None)


@pytest.mark.parametrize("kw", [dict(R=-1), dict(d=0), dict(x=None), dict(y=None), dict(tx=2), dict(ty=-1), dict(xs=63), dict(ys=63),
                                dict(mean=None), dict(rstd=None), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
                                dict(x=P + 2), dict(y=P + 1, ty=1), dict(w=P + 2)])
def test_norm_forward_refuses(kw):
    assert norm_fwd(**kw) == -1 and "sdden_layernorm_forward" in err()


def norm_bwd(R=4, d=64, dy=P, ty=0, dys=64, x=P, tx=0, xs=64, w=P, mean=P, rstd=P, dres=None, drs=0, dx=P, dxs=64, dw=P, db=P, ws=P,
             n=1 << 30):
    return B.load_library().sdden_layernorm_backward(R, d, dy, ty, dys, x, tx, xs, w, mean, rstd, dres, drs, dx, dxs, dw, db, ws, n, None)


@pytest.mark.parametrize("kw", [dict(R=-1), dict(d=-3), dict(dy=None), dict(x=None), dict(dx=None), dict(mean=None), dict(rstd=None),
                                dict(ty=3), dict(tx=3), dict(dys=1), dict(xs=1), dict(dxs=1), dict(dres=P, drs=63), dict(dx=P + 2),
                                dict(dres=P + 1, drs=64), dict(ws=P + 2)])
def test_norm_backward_refuses(kw):
    assert norm_bwd(**kw) == -1 and "sdden_layernorm_backward" in err()


def test_sizes_beyond_the_range_are_refused():
    big = (1 << 30) + 1
    assert norm_fwd(R=big) == -5 and norm_fwd(d=big, xs=big, ys=big) == -5 and norm_bwd(R=big) == -5
    assert gated_fwd(R=big) == -5 and gated_bwd(R=big) == -5


def test_norm_backward_needs_its_workspace():
    need = B.sdden_layernorm_workspace_bytes(4, 64)
    assert need > 0 and B.sdden_layernorm_workspace_bytes(0, 64) == 0 and B.sdden_layernorm_workspace_bytes(4, 0) == 0
    assert norm_bwd(n=need - 1) == -3 and norm_bwd(ws=None) == -3 and norm_bwd(db=None, ws=None) == -3 and str(need) in err()


def gated_fwd(R=4, d=64, H=128, act=0, x=P, xs=64, wg=P, wu=P, wd=P, res=None, y=P, ty=1, ys=64, hid=P, gates=None):
    return B.load_library().sdden_gated_forward(R, d, H, act, x, xs, wg, wu, wd, res, y, ty, ys, hid, gates, None)


@pytest.mark.parametrize("kw,rc", [(dict(R=-1), -1), (dict(d=0), -1), (dict(H=0), -1), (dict(act=2), -1), (dict(x=None), -1),
                                   (dict(wg=None), -1), (dict(wu=None), -1), (dict(wd=None), -1), (dict(y=None), -1), (dict(hid=None), -1),
                                   (dict(ty=2), -1), (dict(d=60), -5), (dict(H=100), -5), (dict(xs=56), -1), (dict(xs=68), -1),
                                   (dict(ys=56), -1), (dict(ys=70), -1), (dict(xs=1 << 24), -1), (dict(ys=1 << 24), -1),
                                   (dict(x=P + 8), -1), (dict(y=P + 2), -1), (dict(wd=P + 4), -1), (dict(res=P + 8), -1),
                                   (dict(hid=P + 8), -1), (dict(gates=P + 8), -1),
                                   (dict(R=2 ** 31 - 1, d=1 << 20, xs=1 << 20, ys=1 << 20, H=1 << 20), -5)])
def test_gated_forward_refuses(kw, rc):
    assert gated_fwd(**kw) == rc and "sdden_gated_forward" in err()


def gated_bwd(R=4, d=64, H=128, act=0, dy=P, dys=64, x=P, xs=64, wg=P, wu=P, wd=P, gates=P, hid=P, dx=P, dxs=64, dwg=P, dwu=P, dwd=P, tw=0,
              ws=P, n=1 << 30):
    return B.load_library().sdden_gated_backward(R, d, H, act, dy, dys, x, xs, wg, wu, wd, gates, hid, dx, dxs, dwg, dwu, dwd, tw, ws, n, None)


@pytest.mark.parametrize("kw,rc", [(dict(act=-1), -1), (dict(dy=None), -1), (dict(gates=None), -1), (dict(hid=None), -1), (dict(d=12), -5),
                                   (dict(dwg=None), -1), (dict(dwd=None), -1), (dict(dx=None, dwg=None, dwu=None, dwd=None), -1),
                                   (dict(dys=60), -1), (dict(dxs=60), -1), (dict(tw=5), -1), (dict(ws=P + 8), -1), (dict(dx=P + 8), -1),
                                   (dict(n=4 * 128 * 4 - 1), -3), (dict(ws=None), -3)])
def test_gated_backward_refuses(kw, rc):
    assert gated_bwd(**kw) == rc and "sdden_gated_backward" in err()


def test_binding_refuses_tensors_that_are_not_on_the_device():
    x, w = torch.randn(4, 64), torch.ones(64)
    with pytest.raises(B.SDError, match="x:"):
        B.sdden_layernorm_forward(x, w, w, 1e-5, x)
    with pytest.raises(B.SDError, match="X:"):
        B.sdden_gated_forward(x, x, x, x, x, x)


def test_errors_are_kept_per_thread():
    import threading
    assert norm_fwd(d=0) == -1
    seen = []
    t = threading.Thread(target=lambda: seen.append((gated_fwd(H=0), err())))
    t.start()
    t.join()
    assert seen[0][0] == -1 and "gated" in seen[0][1] and "layernorm" in err()


def q4_create(N=4, K=64, group=32, q=P, s=P, out=True):
    h = ctypes.c_void_p()
    return B.load_library().sdden_q4_create(N, K, group, q, s, ctypes.byref(h) if out else None)


@pytest.mark.parametrize("kw,rc", [(dict(N=0), -1), (dict(K=0), -1), (dict(q=None), -1), (dict(s=None), -1), (dict(out=False), -1),
                                   (dict(group=0), -5), (dict(group=-128), -5), (dict(group=16), -5), (dict(group=96), -5),
                                   (dict(group=200), -5), (dict(N=(1 << 20) + 1), -5), (dict(K=(1 << 20) + 1), -5)])
def test_q4_create_refuses(kw, rc):
    assert q4_create(**kw) == rc and "sdden_q4_create" in err()


def test_q4_calls_without_a_matrix():
    lib = B.load_library()
    assert lib.sdden_q4_eval(None, 1, P, 0, 64, None, P, 0, 64, None) == -1 and "sdden_q4_eval" in err()
    assert lib.sdden_q4_destroy(None) == -1


def test_q4_binding_checks_shapes():
    import numpy as np
    q, s = np.zeros((4, 33), np.uint8), np.zeros((4, 3), np.uint16)
    for bad in (dict(q=q, scale=s, K=64, group=32), dict(q=q, scale=s, K=65, group=64), dict(q=q.astype(np.int8), scale=s, K=65, group=32),
                dict(q=q, scale=s.astype(np.float32), K=65, group=32), dict(q=q, scale=s, K=65, group=0), dict(q=q[0], scale=s, K=65, group=32)):
        with pytest.raises(B.SDError, match="sdden_q4_create"):
            B.Q4Matrix.sdden_q4_create(**bad)


def _ptrs(n):
    import numpy as np
    a = np.zeros(64 * 64, np.uint16)
    f = np.zeros(64 * 64, np.float32)
    return a, f


@pytest.mark.parametrize("kw,rc", [(dict(d=0), -1), (dict(H=-1), -1), (dict(E=3), -1), (dict(T=0), -1), (dict(Rmax=0), -1), (dict(group=48), -5),
                                   (dict(group=0), -5), (dict(d=(1 << 20) + 1), -5), (dict(null=True), -1)])
def test_mlp4_create_refuses(kw, rc):
    a, f = _ptrs(1)
    v = dict(d=8, H=8, E=2, group=32, T=4, Rmax=4, null=False)
    v.update(kw)
    h = ctypes.c_void_p()
    w = None if v["null"] else a.ctypes.data
    assert B.load_library().sdden_mlp4_create(v["d"], v["H"], v["E"], v["group"], w, f.ctypes.data, a.ctypes.data, f.ctypes.data,
                                              a.ctypes.data, f.ctypes.data, v["T"], v["Rmax"], ctypes.byref(h)) == rc
    assert "sdden_mlp4_create" in err()


@pytest.mark.parametrize("kw,rc", [(dict(d=12), -5), (dict(H=20), -5), (dict(E=1), -1), (dict(blocks=0), -1), (dict(act=2), -1),
                                   (dict(eps=float("nan")), -1), (dict(T=0), -1), (dict(Rmax=-1), -1), (dict(null=True), -1)])
def test_gated_create_refuses(kw, rc):
    a, f = _ptrs(1)
    v = dict(d=8, H=8, E=2, blocks=1, act=0, eps=1e-5, T=4, Rmax=4, null=False)
    v.update(kw)
    h = ctypes.c_void_p()
    w = None if v["null"] else a.ctypes.data
    assert B.load_library().sdden_gated_create(v["d"], v["H"], v["E"], v["blocks"], v["act"], a.ctypes.data, f.ctypes.data, f.ctypes.data,
                                               f.ctypes.data, v["eps"], w, a.ctypes.data, a.ctypes.data, v["T"], v["Rmax"], ctypes.byref(h)) == rc
    assert "sdden_gated_create" in err()


def test_network_bindings_check_shapes():
    import numpy as np
    import workloads as W
    p = W.random_mlp(np.random.default_rng(0), 8, 8, 2)
    p.W2 = p.W2[:4]
    with pytest.raises(B.SDError, match="mlp4"):
        B.Denoiser.sdden_mlp4_create(p, 32, 4, 4)
    g = W.random_gated(np.random.default_rng(0), 8, 16, 2, 2)
    g.norm_bias = g.norm_bias[:1]
    with pytest.raises(B.SDError, match="gated"):
        B.Denoiser.sdden_gated_create(g, 4, 4)
