"""Layer norm, projections with activation and residual, and gated feed-forward
blocks in float64, straight from the definitions, each result with a bound of
what a float32 or bfloat16 evaluation may be off by.

Bounds.  A half step of bfloat16 is R = 2^-8 of a value, of float32 2^-24.  A
float32 sum of n products is off by at most (n + 32) 2^-24 of the sum of their
magnitudes (every addition rounded once; the 32 hold the rounding of what is
summed, 2^-24 of a product that the three-part products leave out, and the joins
of partial sums).  bfloat16 calls round z, dz, h, dg and du once (R) where they
are operands of a next product, and keep g and u to 2^-7 or better for the backward.  Activations: |act'| <= 1.13, |act''| <= 0.8
(gelu; silu 1.10 and 0.5), values off by 1e-6 of z (the fast forms' 1.5e-7 and
their exponentials' roundings)."""
import math

import torch

R = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
D1, D2, ACT = 1.13, 0.8, 1e-6


def acc(n):
    return (n + 32) * 2.0 ** -24


def act(z, name):
    """Value and derivative."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp(min=0), (z > 0).to(z.dtype)
    if name == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    phi = 0.5 * torch.erfc(-z * math.sqrt(0.5))
    return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)


def slopes(name):
    """Bounds of the derivative, of its own derivative, and of the values'
    error."""
    return (1.0, 0.0, 0.0) if name in ("none", "relu") else (D1, D2, ACT)


def norm(x, w, b, eps, dt, dy=None, res=None):
    """{name: (value, bound)} of y, mean, rstd and, with dy, dx, dw, db.  A row's
    sums: at most 64 values a lane and 8 exchanges; the mean's error, the
    deviations' and half the variance's reach n: 3 (72 + 8) roundings of its
    magnitude."""
    C = x.shape[1]
    mean = x.mean(1, keepdim=True)
    d = x - mean
    r = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + eps)
    n = d * r
    size = x.abs().mean(1, keepdim=True)
    e = 240 * 2.0 ** -24
    nm = (x.abs() + size) * r
    y = n * w + b
    out = {"y": (y, e * (nm * w.abs() + b.abs()) + R[dt] * y.abs()),
           "mean": (mean[:, 0], 80 * 2.0 ** -24 * size[:, 0]),
           # the variance loses by the mean's error squared and the roundings
           "rstd": (r[:, 0], e * r[:, 0] * (1 + (size * r)[:, 0] * 1e-2))}
    if dy is None:
        return out
    g = dy * w
    gn = (g * n).mean(1, keepdim=True)
    dx = r * (g - g.mean(1, keepdim=True) - n * gn) + res
    gm = r * (g.abs() + g.abs().mean(1, keepdim=True) + nm * (g.abs() * nm).mean(1, keepdim=True))
    out["dx"] = (dx, 2 * e * gm + 2.0 ** -23 * res.abs() + R[dt] * dx.abs())
    rows = x.shape[0]
    out["dw"] = ((dy * n).sum(0), (acc(rows) + e) * (dy.abs() * nm).sum(0))
    out["db"] = (dy.sum(0), acc(rows) * dy.abs().sum(0))
    return out


def linear(x, w, b, res, name, dt, dy=None, gt=None):
    """y, z and, with dy, dx, dw, db (in gt, dt by default)."""
    T, K = x.shape
    N = w.shape[0]
    s1, s2, sa = slopes(name)
    z = x @ w.T + b
    ez = acc(K) * (x.abs() @ w.abs().T + b.abs())
    a, d = act(z, name)
    y = a + res
    out = {"z": (z, ez + R[dt] * z.abs()),
           "y": (y, s1 * ez + sa * z.abs() + 2.0 ** -23 * y.abs() + R[dt] * y.abs())}
    if dy is None:
        return out
    rg = R[gt or dt]
    dz = dy * d
    # z as it is kept, the derivative's own value, the product's rounding
    edz = dy.abs() * (s2 * (ez + R[dt] * z.abs()) + 2 * sa) + R[dt] * dz.abs()
    if name == "none":
        edz = torch.zeros_like(dz)
    dx, dw, db = dz @ w, dz.T @ x, dz.sum(0)
    out["dx"] = (dx, edz @ w.abs() + acc(N) * (dz.abs() @ w.abs()) + R[dt] * dx.abs())
    out["dw"] = (dw, edz.T @ x.abs() + acc(T) * (dz.abs().T @ x.abs()) + rg * dw.abs())
    out["db"] = (db, edz.sum(0) + acc(T) * dz.abs().sum(0) + rg * db.abs())
    return out


def ffn(x, w1, b1, w2, b2, res, name, dt, dy=None, gt=None):
    """y and, with dy, dx, dw1, db1, dw2, db2."""
    T, K = x.shape
    N, F = w2.shape
    s1, s2, sa = slopes(name)
    z = x @ w1.T + b1
    ez = acc(K) * (x.abs() @ w1.abs().T + b1.abs())
    g, u, eg, eu = z[:, :F], z[:, F:], ez[:, :F], ez[:, F:]
    a, d = act(g, name)
    h = a * u
    eh = (s1 * eg + sa * g.abs()) * u.abs() + a.abs() * eu + R[dt] * h.abs() + 2.0 ** -22 * h.abs()
    y = h @ w2.T + b2 + res
    out = {"y": (y, eh @ w2.abs().T + acc(F) * (h.abs() @ w2.abs().T + b2.abs()) +
                 2.0 ** -23 * y.abs() + R[dt] * y.abs())}
    if dy is None:
        return out
    rg = R[gt or dt]
    dh = dy @ w2
    edh = acc(N) * (dy.abs() @ w2.abs())
    keep = 2.0 ** -7 if dt == "bf16" else 0.0
    kg, ku = eg + keep * g.abs(), eu + keep * u.abs()  # g and u as they are kept
    dg, du = dh * u * d, dh * a
    edg = (edh * u.abs() * s1 + dh.abs() * s1 * ku + (dh * u).abs() * (s2 * kg + 2 * sa) +
           R[dt] * dg.abs() + 2.0 ** -22 * dg.abs())
    edu = (edh * a.abs() + dh.abs() * (s1 * kg + sa * g.abs()) + R[dt] * du.abs() +
           2.0 ** -23 * du.abs())
    dz, edz = torch.cat([dg, du], 1), torch.cat([edg, edu], 1)
    dx, dw1, dw2 = dz @ w1, dz.T @ x, dy.T @ h
    out["dx"] = (dx, edz @ w1.abs() + acc(2 * F) * (dz.abs() @ w1.abs()) + R[dt] * dx.abs())
    out["dw1"] = (dw1, edz.T @ x.abs() + acc(T) * (dz.abs().T @ x.abs()) + rg * dw1.abs())
    out["db1"] = (dz.sum(0), edz.sum(0) + acc(T) * dz.abs().sum(0) + rg * dz.sum(0).abs())
    out["dw2"] = (dw2, dy.abs().T @ eh + acc(T) * (dy.abs().T @ h.abs()) + rg * dw2.abs())
    out["db2"] = (dy.sum(0), acc(T) * dy.abs().sum(0) + rg * dy.sum(0).abs())
    return out
