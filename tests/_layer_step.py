"""One training step  y = h + FF(LN(h))  with the loss sum(c * y), in fp64 on the CPU: its gradients by the formulas, with the roundings of
the library's path where asked for, and with a planted mistake where asked for."""
import torch

MISTAKES = ["no block", "no dU", "no dG", "norm backward skipped", "no residual", "sign", "f' without its second term", "dG and dU swapped",
            "norm without its mean term", "norm without its xh term", "zero", "twice"]


def bf16(t):
    return t.to(torch.bfloat16).double()


def problem(R, d, H, seed):
    """h, c (bf16 values), weight, bias, Wg, Wu, Wd (bf16 values)."""
    gen = torch.Generator().manual_seed(seed)
    rnd = lambda *n: torch.randn(*n, generator=gen, dtype=torch.float64)
    h, c = rnd(R, d).float().double(), bf16(rnd(R, d))
    w, b = (1 + 0.2 * rnd(d)).float().double(), (0.2 * rnd(d)).float().double()
    return h, c, w, b, bf16(rnd(H, d) * d ** -0.5), bf16(rnd(H, d) * d ** -0.5), bf16(rnd(d, H) * H ** -0.5)


def activation(g, act):
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s, g * s * (1 - s)
    P = torch.special.ndtr(g)
    return g * P, P, g * torch.exp(-g * g / 2) / (2 * torch.pi) ** 0.5


def gradients(h, c, w, b, Wg, Wu, Wd, act="silu", eps=1e-5, mistake=None, rounded=False):
    """dh, dw, db, dWg, dWu, dWd."""
    q = bf16 if rounded else (lambda t: t)
    mean = h.mean(1, keepdim=True)
    r = ((h - mean).square().mean(1, keepdim=True) + eps) ** -0.5
    xh = (h - mean) * r
    x = q(xh * w + b)
    g, u = x @ Wg.T, x @ Wu.T
    f, df1, df2 = activation(g, act)
    hidden = q(f * u)
    df = df1 if mistake == "f' without its second term" else df1 + df2
    da = c @ Wd
    dG, dU = q(da * u * df), q(da * f)
    if mistake == "dG and dU swapped":
        dG, dU = dU, dG
    dx = (0 if mistake == "no dG" else dG @ Wg) + (0 if mistake == "no dU" else dU @ Wu)
    dx = q(dx) * (0 if mistake == "no block" else 1)
    v = dx * w
    dh = v
    if mistake != "norm backward skipped":
        dh = r * (v - (0 if mistake == "norm without its mean term" else v.mean(1, keepdim=True))
                  - (0 if mistake == "norm without its xh term" else xh * (v * xh).mean(1, keepdim=True)))
    if mistake != "no residual":
        dh = dh + c
    out = [dh, (dx * xh).sum(0), dx.sum(0), dG.T @ x, dU.T @ x, c.T @ hidden]
    if mistake in ("sign", "zero", "twice"):
        out = [t * {"sign": -1, "zero": 0, "twice": 2}[mistake] for t in out]
    return out


def loss(h, c, w, b, Wg, Wu, Wd, act="silu", eps=1e-5):
    mean = h.mean(1, keepdim=True)
    x = (h - mean) * ((h - mean).square().mean(1, keepdim=True) + eps) ** -0.5 * w + b
    return (c * (h + (activation(x @ Wg.T, act)[0] * (x @ Wu.T)) @ Wd.T)).sum()


# A rounding to bf16 moves a tensor by at most b = 2^-8 of its norm.  On the way of dh: x; hence g and u, a product with a random matrix
# of 264 x 136 keeping a relative error within its largest singular value over the mean one, (1 + sqrt(264 / 136)) / sqrt(264 / 136)
# = 1.7; in da u f' and da f these errors meet, f' and f passing g's on with a factor of up to 1.5; dG and dU add b of their own, the
# products with Wg and Wu again a factor (1 + sqrt(136 / 264)) = 1.7, dx b:  ((1.7 + 1.7 * 1.5 + 1) 1.7 + 1) b = 9.9 b.  The weights'
# gradients have no more roundings than that behind them.
LIMIT = 10 * 2.0 ** -8


def off(got, want):
    """Distance of a gradient from the right one, relative to the latter's norm."""
    return float((got - want).norm() / want.norm())


def shares(got, want, c):
    """`off` of every gradient; dh without the residual's share c, which would hide the block's."""
    return [off(got[0] - c, want[0] - c)] + [off(g, w) for g, w in zip(got[1:], want[1:])]
