"""Attention over packed sequences, norm and rotation, and counter-based
dropout in float64, straight from the definitions, head after head, and the
magnitudes that the tolerances refer to."""
import math

import numpy as np
import torch


def attention(q, k, v, spans, scale, causal, dout=None):
    """q [Tq][Hq][D], k and v [Tk][Hkv][D] in float64; spans: (q0, n, k0, m) a
    sequence.  Returns a dict: o, lse and, with dout, dq, dk, dv, each with the
    sum of its terms' magnitudes under its name + "_mag"."""
    Tq, Hq, D = q.shape
    Tk, Hkv = k.shape[:2]
    G = Hq // Hkv
    z = lambda like: torch.zeros(like.shape, dtype=torch.float64)
    r = {"o": z(q), "o_mag": z(q), "lse": torch.zeros((Tq, Hq), dtype=torch.float64)}
    for name, like in (("dq", q), ("dk", k), ("dv", v)):
        r[name], r[name + "_mag"] = z(like), z(like)
    for q0, n, k0, m in spans:
        for h in range(Hq):
            j = h // G
            Q, K, V = q[q0:q0 + n, h], k[k0:k0 + m, j], v[k0:k0 + m, j]
            x = scale * (Q @ K.T)
            if causal:
                i = torch.arange(n)[:, None]
                x = x.masked_fill(torch.arange(m)[None] > i + m - n, -math.inf)
            lse = torch.logsumexp(x, 1) if m else torch.full((n,), -math.inf, dtype=x.dtype)
            p = torch.where(lse[:, None] == -math.inf, torch.zeros_like(x),
                            torch.exp(x - lse[:, None]))
            O, Om = p @ V, p @ V.abs()
            r["o"][q0:q0 + n, h], r["o_mag"][q0:q0 + n, h] = O, Om
            r["lse"][q0:q0 + n, h] = lse
            if dout is None:
                continue
            g = dout[q0:q0 + n, h]
            ds = p * (g @ V.T - (g * O).sum(1, keepdim=True))
            # o and the product with v are off by their own rounding
            dsm = p * (g.abs() @ V.abs().T + (g.abs() * Om).sum(1, keepdim=True))
            r["dq"][q0:q0 + n, h] = scale * ds @ K
            r["dq_mag"][q0:q0 + n, h] = abs(scale) * dsm @ K.abs()
            r["dk"][k0:k0 + m, j] += scale * ds.T @ Q
            r["dk_mag"][k0:k0 + m, j] += abs(scale) * dsm.T @ Q.abs()
            r["dv"][k0:k0 + m, j] += p.T @ g
            r["dv_mag"][k0:k0 + m, j] += p.T @ g.abs()
    return r


def rotary(x, w, pos, freq, axis, eps, norm, dy=None):
    """x [T][H][D] in float64: the result and its magnitude, and with dy also
    dx, dw and theirs."""
    D = x.shape[2]
    a = torch.zeros((pos.shape[0], D // 2), dtype=torch.float64)
    for j in range(D // 2):
        if 0 <= int(axis[j]) < pos.shape[1]:
            a[:, j] = pos[:, int(axis[j])].double() * freq[j].double()
    c, s = torch.cos(a)[:, None], torch.sin(a)[:, None]
    r = 1 / torch.sqrt((x * x).mean(2, keepdim=True) + eps) if norm else torch.ones(1)
    n = x * r
    y = n * w if norm else x
    y1, y2 = y[..., :D // 2], y[..., D // 2:]
    out = torch.cat([y1 * c - y2 * s, y1 * s + y2 * c], 2)
    mag = torch.cat([y1.abs() + y2.abs()] * 2, 2)
    if dy is None:
        return out, mag
    d1, d2 = dy[..., :D // 2], dy[..., D // 2:]
    g = torch.cat([d1 * c + d2 * s, d2 * c - d1 * s], 2)
    gm = torch.cat([d1.abs() + d2.abs()] * 2, 2)
    if not norm:
        return out, mag, g, gm
    dw, dwm = (g * n).sum((0, 1)), (gm * n.abs()).sum((0, 1))
    g, gm = g * w, gm * w.abs()
    dx = r * (g - n * (g * n).mean(2, keepdim=True))
    dxm = r * (gm + n.abs() * (gm * n.abs()).mean(2, keepdim=True))
    return out, mag, dx, dxm, dw, dwm


def philox(n, seed, counter):
    """32 bits for each of n elements by Philox 4x32-10, in Python integers."""
    out = []
    for b in range((n + 3) // 4):
        x = [b & 0xFFFFFFFF, b >> 32, counter & 0xFFFFFFFF, counter >> 32 & 0xFFFFFFFF]
        k = [seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF]
        for _ in range(10):
            p, q = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57
            x = [q >> 32 ^ x[1] ^ k[0], q & 0xFFFFFFFF, p >> 32 ^ x[3] ^ k[1], p & 0xFFFFFFFF]
            k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
        out += x
    return np.array(out[:n], np.int64)
