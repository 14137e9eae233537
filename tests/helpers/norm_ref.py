"""Group norm with an activation in 64 bits, and how far binary32 arithmetic may be from it.

The bounds are first-order: U = 2^-24 per rounding; an element goes through at most K additions of a sum."""
import math

import torch

U = 2.0 ** -24


def act64(z, act):
    """(act(z), act'(z))"""
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    if act == "gelu":
        cdf = torch.special.ndtr(z)
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return z, torch.ones_like(z)


def act_slack(z, y, dz, act):
    """How far act(z) and act'(z) may be for arguments off by dz: the largest slopes of the functions and of their
    derivatives (SiLU 1.1, 0.5; GELU 1.13, 0.8), and the evaluation: exp to 2 units and its argument's rounding, erf to
    2 units, a quotient to 2 units, a handful of products."""
    work = (16 + 4 * z.abs()) * U
    if act == "none":
        return dz, torch.zeros_like(z)
    if act == "relu":
        return dz, (z.abs() <= dz).double()                 # on the wrong side of the step
    if act == "silu":
        return 1.1 * dz + y.abs() * work, 0.5 * dz + (1 + z.abs()) * work
    return 1.13 * dz + (y.abs() + z.abs()) * work, 0.8 * dz + (1 + z.abs()) * work


def per_group(x, groups):
    n, c = x.shape[0], x.shape[-1]
    return x.reshape(n, -1, groups, c // groups)


def spread(g, shape):
    """[n, groups] over [n, s, c]"""
    n, s, c = shape
    return g[:, None, :, None].expand(n, s, g.shape[1], c // g.shape[1]).reshape(n, s, c)


def additions(s, cg):
    """K: the rows of a chunk that one thread adds (at most 512 here), the threads, the chunks and channels a warp joins."""
    return 64 + min(s, 512) + cg


def statistics(x, groups, eps):
    """mean, rstd and their bounds, [n, groups]."""
    x4 = per_group(x.double(), groups)
    mean = x4.mean((1, 3))
    var = (x4 - mean[:, None, :, None]).square().mean((1, 3))
    k = additions(x4.shape[1], x4.shape[3])
    dmean = k * U * x4.abs().mean((1, 3))
    rstd = (var + eps) ** -0.5
    drel = 0.5 * ((k + 8) * U * var + dmean ** 2 + 8 * U * dmean * var.sqrt()) / (var + eps) + 4 * U
    return mean, rstd, dmean, drel


def forward(x, groups, w, b, eps, act):
    """y, mean, rstd and the bounds of the three."""
    mean, rstd, dmean, drel = statistics(x, groups, eps)
    xd = x.double()
    d = xd - spread(mean, x.shape)
    r = spread(rstd, x.shape)
    slope = (r * w.double()).abs()
    z = d * r * w.double() + b.double()
    off = spread(dmean, x.shape) + U * d.abs()
    dz = slope * off + slope * d.abs() * (spread(drel, x.shape) + 4 * U) + 2 * U * (z.abs() + b.double().abs())
    y, _ = act64(z, act)
    dy, _ = act_slack(z, y, dz, act)
    return (y, mean, rstd), (dy, dmean + U * mean.abs(), drel * rstd)


def backward(dy, x, mean, rstd, groups, w, b, act):
    """dx, dweight, dbias for the given statistics, and their bounds."""
    n, s, c = x.shape
    cg = c // groups
    k = additions(s, cg) + n
    m, r = spread(mean.double(), x.shape), spread(rstd.double(), x.shape)
    d = x.double() - m
    xh = d * r
    w, b = w.double(), b.double()
    z = xh * w + b
    dz_arg = 8 * U * ((xh * w).abs() + b.abs()) + U * (r * w).abs() * (x.double().abs() + m.abs())
    y, slope = act64(z, act)
    _, off = act_slack(z, y, dz_arg, act)
    g = dy.double() * slope
    dg = dy.double().abs() * (off + 2 * U * slope.abs())
    dbias, dweight = g.sum((0, 1)), (g * xh).sum((0, 1))
    e_bias = dg.sum((0, 1)) + k * U * g.abs().sum((0, 1))
    e_weight = (dg * xh.abs()).sum((0, 1)) + (k + 6) * U * (g * xh).abs().sum((0, 1))

    def mean_of(t):
        return spread(per_group(t, groups).mean((1, 3)), x.shape)

    a, e_a = mean_of(g * w), mean_of(dg * w.abs() + (k + 6) * U * (g * w).abs())
    q, e_q = mean_of(g * w * xh), mean_of(dg * (w * xh).abs() + (k + 8) * U * (g * w * xh).abs())
    dx = r * (g * w - a - xh * q)
    e_x = r * (dg * w.abs() + e_a + xh.abs() * e_q + 10 * U * ((g * w).abs() + a.abs() + (xh * q).abs()))
    return (dx, dweight, dbias), (e_x, e_weight, e_bias)


def inside(got, want, bound):
    """Whether got lies between the rounded ends of the interval (rounding is monotone)."""
    lo, hi = want - bound * 1.000001 - 1e-45, want + bound * 1.000001 + 1e-45
    if got.dtype == torch.bfloat16:
        lo, hi = lo.float().to(torch.bfloat16), hi.float().to(torch.bfloat16)
    else:
        bound = 2 * U * want.abs()                          # the ends' own rounding
        lo, hi = lo - bound, hi + bound
    return bool(((lo.double() <= got.double()) & (got.double() <= hi.double())).all())
