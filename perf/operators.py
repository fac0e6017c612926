"""Calls of the layers that row networks are made of, with sizes of the repository's own configurations and generic ones.

Three operators, each as a user's program calls it:

  norm    layer norm over the last axis of R rows, forward, or forward and backward with the gradients of weight and bias
  gated   the gated feed-forward block  Y = (f(X Wg^T) * (X Wu^T)) Wd^T,  forward, or a training step's forward and
          backward with the gradients of the rows and of the three weights
  q4      rows times a matrix kept in 4 bits with one scale per group of inputs, plus a bias

``run`` computes them in elementary torch operations in 32 bits, or, with ``own``, by the library's calls.
"""
from types import SimpleNamespace

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


# ---------------------------------------------------------------------------------------------- the listed cases
def listed():
    return [
        # one chain's window start: a single row as wide as the image configuration's states; latency
        dict(name="norm_one_row", op="norm", train=False, R=1, d=12288, x="f32", y="bf16", pad=0),
        # the batched call of 480 chains with 16 drafts each: fp32 states in, rows for the first product out
        dict(name="norm_batch", op="norm", train=False, R=7680, d=12288, x="f32", y="bf16", pad=0),
        # a training step over many rows of a usual width
        dict(name="norm_train", op="norm", train=True, R=16384, d=4096, x="bf16", y="bf16", pad=0),
        # odd width, ragged rows, rows that lie apart: nothing is aligned to 16 bytes
        dict(name="norm_train_odd", op="norm", train=True, R=2049, d=1001, x="f32", y="f32", pad=5),
        # one chain through the block at the image configuration's widths: reading 302 MB of weights
        dict(name="gated_one_row", op="gated", train=False, act="silu", R=1, d=12288, H=4096, pad=0),
        # the batched call of the same configuration
        dict(name="gated_batch", op="gated", train=False, act="silu", R=7680, d=12288, H=4096, pad=0),
        # a training step, forward and backward
        dict(name="gated_train", op="gated", train=True, act="silu", R=8192, d=4096, H=11008, pad=0),
        # a small network's training step at sizes that fill no tile
        dict(name="gated_train_ragged", op="gated", train=True, act="gelu", R=777, d=520, H=1352, pad=8),
        # one chain's first product with a 4-bit draft of the image configuration, fp32 state
        dict(name="q4_one_row", op="q4", R=1, K=12288, N=4096, group=128, x="f32", y="bf16"),
        # a few chains' last product: fp32 predictions
        dict(name="q4_few_rows", op="q4", R=19, K=4096, N=12288, group=64, x="bf16", y="f32"),
        # all chains of the image configuration
        dict(name="q4_batch", op="q4", R=512, K=4096, N=12288, group=128, x="bf16", y="f32"),
        # a small odd matrix: latency and ends inside a group, a tile and a byte
        dict(name="q4_odd", op="q4", R=5, K=1001, N=333, group=32, x="f32", y="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "gated", "gated", "gated", "q4", "q4", "q4"])
    if op == "norm":
        train = rng.random() < 0.6
        d = _log(rng, 16, 16384)
        R = _log(rng, 1, 16384)
        R = max(1, min(R, (16384 * 4096 if train else 7680 * 12288) // (2 * d)))
        return dict(op="norm", train=train, R=R, d=d, x=rng.choice(["f32", "bf16"]), y=rng.choice(["f32", "bf16"]), pad=rng.choice([0, 0, 3, 8]))
    if op == "gated":
        train = rng.random() < 0.5
        d, H = 8 * _log(rng, 8, 1536), 8 * _log(rng, 8, 1536)
        R = _log(rng, 1, 8192)
        R = max(1, min(R, (8192 * 4096 * 11008 if train else 7680 * 12288 * 4096) // (d * H)))
        return dict(op="gated", train=train, act=rng.choice(["silu", "gelu"]), R=R, d=d, H=H, pad=rng.choice([0, 0, 8, 24]))
    K, N = _log(rng, 32, 12288), _log(rng, 16, 12288)
    R = max(1, min(_log(rng, 1, 512), 512 * 4096 * 12288 // (K * N)))
    return dict(op="q4", R=R, K=K, N=N, group=rng.choice([32, 64, 128, 256]), x=rng.choice(["f32", "bf16"]), y=rng.choice(["f32", "bf16"]))


# ---------------------------------------------------------------------------------------------- inputs
def _rows(gen, R, d, pad, dtype):
    """R rows of d normal values, `pad` values apart in memory."""
    full = torch.randn(R, d + pad, generator=gen, device="cuda").to(dtype)
    return full[:, :d]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, R = case["op"], case["R"]
    s = SimpleNamespace(case=dict(case))
    empty = lambda *n, t=torch.float32: torch.empty(*n, dtype=t, device="cuda")
    if op == "norm":
        d, tx, ty = case["d"], TYPES[case["x"]], TYPES[case["y"]]
        # rows of a residual stream: an offset and a scale of their own each
        s.x = _rows(gen, R, d, case["pad"], torch.float32)
        s.x.mul_(torch.rand(R, 1, generator=gen, device="cuda") * 3 + 0.3).add_(torch.randn(R, 1, generator=gen, device="cuda"))
        full = torch.empty(R, d + case["pad"], dtype=tx, device="cuda")
        full[:, :d] = s.x
        s.x = full[:, :d]
        s.w = 1 + 0.2 * torch.randn(d, generator=gen, device="cuda")
        s.b = 0.2 * torch.randn(d, generator=gen, device="cuda")
        s.y = empty(R, d, t=ty)
        if case["train"]:
            s.dy = _rows(gen, R, d, case["pad"], ty)
            s.dres = _rows(gen, R, d, 0, tx)              # the gradient that comes around the block, on the residual path
            s.mean, s.rstd = empty(R), empty(R)
            s.dx, s.dw, s.db = empty(R, d, t=tx), empty(d), empty(d)
    elif op == "gated":
        d, H, bf = case["d"], case["H"], torch.bfloat16
        s.x = _rows(gen, R, d, case["pad"], bf)
        s.wg, s.wu = ((torch.randn(H, d, generator=gen, device="cuda") * d ** -0.5).to(bf) for _ in range(2))
        s.wd = (torch.randn(d, H, generator=gen, device="cuda") * H ** -0.5).to(bf)
        s.y, s.hidden = empty(R, d, t=bf), empty(R, H, t=bf)
        if case["train"]:
            s.dy = _rows(gen, R, d, case["pad"], bf)
            s.gates = empty(2, R, H)
            s.dx, s.dwg, s.dwu, s.dwd = empty(R, d, t=bf), empty(H, d, t=bf), empty(H, d, t=bf), empty(d, H, t=bf)
    else:
        K, N, g = case["K"], case["N"], case["group"]
        s.x = _rows(gen, R, K, 0, TYPES[case["x"]])
        groups = -(-K // g)
        w = torch.randn(N, groups * g, generator=gen, device="cuda").view(N, groups, g)
        s.scale = (w.abs().amax(2) / 7.5).to(torch.bfloat16)
        q = (torch.round(w / s.scale.float().unsqueeze(2)) + 8).clamp_(0, 15).view(N, groups * g)[:, :K + K % 2].to(torch.uint8)
        s.q = (q[:, 0::2] | (q[:, 1::2] << 4)).contiguous()          # [N, ceil(K / 2)], the even input in the low half
        s.scale = (s.scale.float() * K ** -0.5).to(torch.bfloat16).contiguous()
        s.bias = torch.randn(N, generator=gen, device="cuda")
        s.y = empty(R, N, t=TYPES[case["y"]])
    if own:
        from paper_2501_05370_amd import binding
        s.lib = binding
        scratch = lambda n: torch.empty(max(1, n), dtype=torch.uint8, device="cuda")
        if op == "norm" and case["train"]:
            s.ws = scratch(binding.sdden_layernorm_workspace_bytes(R, case["d"]))
        elif op == "gated":
            s.act = {"silu": binding.SDDEN_SILU, "gelu": binding.SDDEN_GELU}[case["act"]]
            if case["train"]:
                s.ws = scratch(binding.sdden_gated_workspace_bytes(R, case["d"], case["H"]))
        elif op == "q4":     # the handle that holds the weights in the kernels' order
            s.net = binding.Q4Matrix.sdden_q4_create(s.q.cpu().numpy(), s.scale.view(torch.int16).cpu().numpy(), case["K"], case["group"])
    return s


# ---------------------------------------------------------------------------------------------- one pass
def _norm_plain(s):
    c = s.case
    x = s.x.float()
    mean = x.mean(1, keepdim=True)
    xc = x - mean
    rstd = 1.0 / torch.sqrt((xc * xc).mean(1, keepdim=True) + EPS)
    xh = xc * rstd
    y = (xh * s.w + s.b).to(TYPES[c["y"]])
    if not c["train"]:
        return [y]
    dy = s.dy.float()
    g = dy * s.w
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) + s.dres.float()
    return [y, dx.to(TYPES[c["x"]]), (dy * xh).sum(0), dy.sum(0)]


def _act(g, act):
    """f(g) and f'(g)."""
    if act == "silu":
        t = 1.0 / (1.0 + torch.exp(-g))
        return g * t, t * (1.0 + g * (1.0 - t))
    t = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
    return g * t, t + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))


def _gated_plain(s):
    c, bf = s.case, torch.bfloat16
    x, wg, wu, wd = (t.float() for t in (s.x, s.wg, s.wu, s.wd))
    g, u = x @ wg.t(), x @ wu.t()
    f, df = _act(g, c["act"])
    a = f * u
    y = (a @ wd.t()).to(bf)
    if not c["train"]:
        return [y]
    dy = s.dy.float()
    da = dy @ wd
    dg, du = da * u * df, da * f
    dx = dg @ wg + du @ wu
    return [y] + [t.to(bf) for t in (dx, dg.t() @ x, du.t() @ x, dy.t() @ a)]


def _q4_plain(s):
    c = s.case
    w = torch.stack([s.q & 15, s.q >> 4], 2).view(c["N"], -1)[:, :c["K"]].float() - 8
    w = w * s.scale.float().repeat_interleave(c["group"], 1)[:, :c["K"]]
    return [(s.x.float() @ w.t() + s.bias).to(TYPES[c["y"]])]


def run(s):
    c = s.case
    if not own:
        return {"norm": _norm_plain, "gated": _gated_plain, "q4": _q4_plain}[c["op"]](s)
    lib = s.lib
    if c["op"] == "norm":
        if not c["train"]:
            lib.sdden_layernorm_forward(s.x, s.w, s.b, EPS, s.y)
            return [s.y]
        lib.sdden_layernorm_forward(s.x, s.w, s.b, EPS, s.y, s.mean, s.rstd)
        lib.sdden_layernorm_backward(s.dy, s.x, s.w, s.mean, s.rstd, s.dx, s.dw, s.db, s.ws, dres=s.dres)
        return [s.y, s.dx, s.dw, s.db]
    if c["op"] == "gated":
        if not c["train"]:
            lib.sdden_gated_forward(s.x, s.wg, s.wu, s.wd, s.y, s.hidden, act=s.act)
            return [s.y]
        lib.sdden_gated_forward(s.x, s.wg, s.wu, s.wd, s.y, s.hidden, gates=s.gates, act=s.act)
        lib.sdden_gated_backward(s.dy, s.x, s.wg, s.wu, s.wd, s.gates, s.hidden, s.dx, s.dwg, s.dwu, s.dwd, s.ws, act=s.act)
        return [s.y, s.dx, s.dwg, s.dwu, s.dwd]
    s.net.sdden_q4_eval(s.x, s.y, bias=s.bias)
    return [s.y]


# ---------------------------------------------------------------------------------------------- what a pass needs
def work(case):
    size = {"f32": 4, "bf16": 2}
    R = case["R"]
    if case["op"] == "norm":
        d, sx, sy = case["d"], size[case["x"]], size[case["y"]]
        if not case["train"]:
            return {"bytes": R * d * (sx + sy) + 8 * d, "flops": 8 * R * d}
        # x, dy, the residual's gradient in; y, dx out; weight and bias in, their gradients out
        return {"bytes": R * d * (3 * sx + 2 * sy) + 16 * d, "flops": 20 * R * d}
    if case["op"] == "gated":
        d, H = case["d"], case["H"]
        if not case["train"]:
            return {"bytes": 2 * (2 * R * d + 3 * d * H), "flops": 6 * R * d * H}
        return {"bytes": 2 * (4 * R * d + 6 * d * H), "flops": 18 * R * d * H}
    K, N = case["K"], case["N"]
    return {"bytes": N * ((K + 1) // 2) + 2 * N * -(-K // case["group"]) + R * (K * size[case["x"]] + N * size[case["y"]]) + 4 * N,
            "flops": 2 * R * K * N}


# ---------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    D = torch.float64
    if case["op"] == "norm":
        x, w, b = s.x.to(D), s.w.to(D), s.b.to(D)
        var, mu = torch.var_mean(x, dim=1, unbiased=False, keepdim=True)
        r = (var + EPS).rsqrt()
        z = (x - mu) * r
        out = [w * z + b]
        if case["train"]:
            v = s.dy.to(D)
            gw = v * w
            n = case["d"]
            out.append((gw * n - gw.sum(1, keepdim=True) - z * (gw * z).sum(1, keepdim=True)) * (r / n) + s.dres.to(D))
            out += [torch.sum(v * z, dim=0), torch.sum(v, dim=0)]
        return out
    if case["op"] == "gated":
        x, wg, wu, wd = s.x.to(D), s.wg.to(D), s.wu.to(D), s.wd.to(D)
        g, u = torch.mm(x, wg.T), torch.mm(x, wu.T)
        if case["act"] == "silu":
            p = torch.sigmoid(g)
            slope = p + g * p * (1 - p)
        else:
            p = torch.special.ndtr(g)
            slope = p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
        a = g * p * u
        out = [torch.mm(a, wd.T)]
        if case["train"]:
            v = s.dy.to(D)
            da = torch.mm(v, wd)
            dg, du = da * u * slope, da * (g * p)
            out += [torch.mm(dg, wg) + torch.mm(du, wu), torch.mm(dg.T, x), torch.mm(du.T, x), torch.mm(v.T, a)]
        return out
    K, N = case["K"], case["N"]
    level = torch.empty(N, s.q.shape[1] * 2, dtype=D, device="cuda")
    level[:, 0::2] = (s.q % 16).to(D)
    level[:, 1::2] = (s.q // 16).to(D)
    which = torch.arange(K, device="cuda") // case["group"]
    return [torch.addmm(s.bias.to(D), s.x.to(D), ((level[:, :K] - 8) * s.scale.to(D)[:, which]).T)]
