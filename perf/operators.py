"""Attention over hexagonal pixels, as cases to be timed.

A camera event is a set of lit pixels: a sequence of tokens with a position
each (time, and the pixel's place on the hexagonal grid), of another length
for every event.  The operators are the parts of an attention layer over
packed sequences of that kind:

 - ``rotary``: root-mean-square norm of every query and key head, then the
   rotation by positions of several axes, forward and backward; ``append`` is
   its serving form, which also stores keys and values in their cache places;
 - ``attn``: softmax attention over packed sequences, grouped heads, causal or
   not, forward and backward;
 - ``step``: attention of one or a few new tokens of every sequence over its
   cache;
 - ``drop``: dropout from a counter-based generator with a residual added; the
   mask is never stored, the backward makes it again.

``run`` computes a case in elementary torch operations in 32 bits, or, where
``own`` is true, by the library's entry points.  ``exact`` evaluates the
definitions in 64 bits, gradients by automatic differentiation.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6
AXES = 3  # time, and the two coordinates of a pixel's centre


# ------------------------------------------------------------------- cases

def rotary(name, T, Hq, Hkv, D, dtype):
    return dict(name=name, kind="rotary", T=T, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype)


def append(name, S, cap, Hq, Hkv, D, dtype):
    return dict(name=name, kind="append", S=S, cap=cap, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype)


def attn(name, S, lo, hi, Hq, Hkv, D, dtype, causal, bwd):
    return dict(name=name, kind="attn", S=S, lo=lo, hi=hi, lens=1, Hq=Hq, Hkv=Hkv, D=D,
                dtype=dtype, causal=causal, bwd=bwd)


def step(name, S, n, lo, hi, Hq, Hkv, D, dtype):
    return dict(name=name, kind="step", S=S, n=n, lo=lo, hi=hi, lens=1, Hq=Hq, Hkv=Hkv, D=D,
                dtype=dtype)


def drop(name, rows, cols, p, dtype, bwd):
    return dict(name=name, kind="drop", rows=rows, cols=cols, p=p, dtype=dtype, bwd=bwd)


def listed():
    return [
        # one new token each of four event streams, into their caches: a
        # serving call, whose time is its launch
        append("append_bf16", 4, 512, 8, 2, 64, "bf16"),
        # a training batch: 32 planes of 40 x 40 pixels
        rotary("rotary_bf16", 51200, 16, 4, 64, "bf16"),
        # one time-resolved event's lit pixels in torch's default dtype, an
        # odd head size
        rotary("rotary_odd_f32", 3287, 6, 3, 40, "f32"),
        # a handful of small events through one layer in inference
        attn("attn_tiny_f32", 4, 5, 37, 4, 2, 32, "f32", False, False),
        # a training batch of camera images, lit pixels only: many short
        # sequences of very different lengths
        attn("attn_events_bf16", 512, 20, 400, 8, 8, 32, "bf16", False, True),
        # whole camera images (1027 pixels) in torch's default dtype, training
        attn("attn_camera_f32", 16, 1027, 1027, 8, 4, 64, "f32", False, True),
        # time-ordered pixels of long events, causal in time, training: the
        # largest case
        attn("attn_causal_bf16", 24, 500, 5000, 16, 4, 128, "bf16", True, True),
        # one long stream's prompt in inference
        attn("attn_prompt_bf16", 1, 16432, 16432, 16, 4, 128, "bf16", True, False),
        # a few long streams, one new token each
        step("step_long_bf16", 3, 1, 9000, 16432, 16, 4, 128, "bf16"),
        # many streams of very different lengths, two new tokens each
        step("step_many_bf16", 192, 2, 32, 4000, 8, 2, 64, "bf16"),
        # one image's pixels through a dropout in torch's default dtype
        drop("drop_image_f32", 1027, 97, 0.1, "f32", True),
        # the residual branch of a training batch
        drop("drop_batch_bf16", 51200, 1024, 0.1, "bf16", True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "append", "attn", "attn", "attn", "step", "step", "drop"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    D = rng.choice([32, 40, 64, 64, 80, 128, 128])
    Hkv = rng.choice([1, 2, 3, 4, 8])
    Hq = Hkv * rng.choice([1, 1, 2, 3, 4])
    most = max(_cost(c) for c in listed())
    if kind == "rotary":
        c = rotary("", _log(rng, 50, 51200), Hq, Hkv, D, dtype)
    elif kind == "append":
        c = append("", _log(rng, 1, 128), _log(rng, 64, 1024), Hq, Hkv, D, dtype)
    elif kind == "attn":
        hi = _log(rng, 24, 16432 if dtype == "bf16" else 4000)
        lo = max(1, hi if rng.random() < 0.25 else _log(rng, max(1, hi // 40), hi))
        c = attn("", _log(rng, 1, 512), lo, hi, Hq, Hkv, D, dtype, rng.random() < 0.5,
                 rng.random() < 0.6)
        c["lens"] = rng.randint(2, 10 ** 6)
        # float32 runs at an eighth of the rate of bf16 or less
        while c["S"] > 1 and _cost(c) > most * (0.05 if dtype == "f32" else 0.6):
            c["S"] = (c["S"] + 1) // 2
    elif kind == "step":
        hi = _log(rng, 32, 16432)
        c = step("", _log(rng, 1, 256), rng.choice([1, 1, 1, 2, 3, 7]),
                 max(8, _log(rng, max(1, hi // 40), hi)), hi, Hq, Hkv, D, dtype)
        c["lens"] = rng.randint(2, 10 ** 6)
        c["hi"] = max(c["lo"], c["hi"])
        while c["S"] > 1 and work(c)["bytes"] > 4e8:
            c["S"] = (c["S"] + 1) // 2
    else:
        c = drop("", _log(rng, 16, 51200), rng.randint(24, 1024), rng.choice([0.1, 0.25, 0.5]),
                 dtype, rng.random() < 0.6)
    while kind in ("attn", "step") and _cost(c) > most * (0.05 if dtype == "f32" else 0.6):
        c["hi"] = c["hi"] // 2
        c["lo"] = min(c["lo"], c["hi"])
    c.pop("name", None)
    return c


def _lengths(c):
    """Tokens of every sequence: fixed by the case, spread over the logarithm
    of its range."""
    if c["lo"] == c["hi"]:
        return [c["lo"]] * c["S"]
    rng = random.Random(c["lens"])
    return [min(c["hi"], max(c["lo"], _log(rng, c["lo"], c["hi"]))) for _ in range(c["S"])]


def _cost(c):
    """Seconds on a card of 5 TB/s and 1 PFLOP/s: only to compare cases."""
    w = work(c)
    return w["bytes"] / 5e12 + w["flops"] / 1e15


# ------------------------------------------------------------------ inputs

class _Gen:
    """Inputs drawn on the device from the seed alone, rounded to the dtype."""

    def __init__(self, case, seed):
        self.dev = torch.device("cuda", 0) if torch.cuda.is_available() else torch.device("cpu")
        self.g = torch.Generator(device=self.dev).manual_seed(seed)
        self.dt = DTYPES[case["dtype"]]

    def normal(self, *shape, std=1.0, mean=0.0):
        t = torch.randn(shape, generator=self.g, device=self.dev)
        return (t * std + mean).to(self.dt)

    def ints(self, lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=self.g, device=self.dev)


def _positions(g, T):
    """Time slice and pixel centre of T tokens of 40 x 40 hexagonal planes
    (odd columns half a pitch lower, columns sqrt(3)/2 of a pitch apart)."""
    t, r, c = g.ints(0, 4096, T), g.ints(0, 40, T), g.ints(0, 40, T)
    return torch.stack([t.float(), r.float() + 0.5 * (c % 2).float(),
                        c.float() * (math.sqrt(3) / 2)], dim=1).contiguous()


def _frequencies(dev, D):
    """Radians a unit for every pair of a head, and the pair's axis: each axis
    owns a run of pairs whose wavelengths grow geometrically."""
    pairs = D // 2
    freq, axis = [], []
    for a in range(AXES):
        n = pairs // AXES + (a < pairs % AXES)
        base = 10000.0 if a == 0 else 100.0
        freq += [base ** (-i / n) for i in range(n)]
        axis += [a] * n
    return (torch.tensor(freq, dtype=torch.float32, device=dev),
            torch.tensor(axis, dtype=torch.int32, device=dev))


def _starts(lens, dev):
    a = [0]
    for n in lens:
        a.append(a[-1] + n)
    return torch.tensor(a, dtype=torch.int32, device=dev)


def prepare(case, seed):
    c = case
    g = _Gen(c, seed)
    s = {"case": c}
    kind = c["kind"]
    if kind in ("rotary", "append"):
        T = c["T"] if kind == "rotary" else c["S"]
        Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
        # queries, keys and values as one projection leaves them
        s["qkv"] = g.normal(T, Hq + 2 * Hkv, D)
        s["pos"] = _positions(g, T)
        s["freq"], s["axis"] = _frequencies(g.dev, D)
        s["wq"], s["wk"] = g.normal(D, std=0.1, mean=1.0), g.normal(D, std=0.1, mean=1.0)
        if kind == "append":
            s["kc"] = g.normal(T * c["cap"], Hkv, D)
            s["vc"] = g.normal(T * c["cap"], Hkv, D)
            at = torch.arange(T, device=g.dev) * c["cap"]
            s["slot"] = (at + g.ints(0, c["cap"], T)).to(torch.int32)
        else:
            s["dqo"], s["dko"] = g.normal(T, Hq, D), g.normal(T, Hkv, D)
    elif kind == "attn":
        lens = _lengths(c)
        T = sum(lens)
        s["lens"], s["start"] = lens, _starts(lens, g.dev)
        s["qkv"] = g.normal(T, c["Hq"] + 2 * c["Hkv"], c["D"])
        if c["bwd"]:
            s["do"] = g.normal(T, c["Hq"], c["D"])
    elif kind == "step":
        lens = _lengths(c)
        cap = max(lens)
        s["lens"], s["cap"] = lens, cap
        s["q"] = g.normal(c["S"], c["n"], c["Hq"], c["D"])
        s["kc"] = g.normal(c["S"] * cap, c["Hkv"], c["D"])
        s["vc"] = g.normal(c["S"] * cap, c["Hkv"], c["D"])
        s["start"] = (torch.arange(c["S"], device=g.dev) * cap).to(torch.int32)
        s["len"] = torch.tensor(lens, dtype=torch.int32, device=g.dev)
    else:
        s["x"], s["res"] = g.normal(c["rows"], c["cols"]), g.normal(c["rows"], c["cols"])
        s["rng"] = torch.tensor([seed * 7919 + 17, 3], dtype=torch.int64, device=g.dev)
        if c["bwd"]:
            s["dy"] = g.normal(c["rows"], c["cols"])
    return s


def _split(qkv, c):
    Hq, Hkv = c["Hq"], c["Hkv"]
    return qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]


def _n_valid(c):
    """Allowed (query, key) pairs of one head, summed over the sequences."""
    if c["kind"] == "step":
        n = c["n"]
        return sum(max(0, L - n + 1 + i) for L in _lengths(c) for i in range(n))
    return sum(L * (L + 1) // 2 if c["causal"] else L * L for L in _lengths(c))


# ---------------------------------------------------------------- own calls

def _own(s):
    from paper_1903_01814_amd import hexconv as hx
    c = s["case"]
    kind = c["kind"]
    if kind == "append":
        q, k, v = _split(s["qkv"], c)
        qo = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        hx.hexrotary_fwd(q, k, s["pos"], s["freq"], s["axis"], s["wq"], s["wk"], qo, s["kc"],
                         eps=EPS, v=v, vo=s["vc"], slot=s["slot"])
        return [qo, s["kc"], s["vc"]]
    if kind == "rotary":
        q, k, _ = _split(s["qkv"], c)
        new = lambda t, dt=None: torch.empty(t.shape, dtype=dt or t.dtype, device=t.device)
        qo, ko = new(q), new(k)
        hx.hexrotary_fwd(q, k, s["pos"], s["freq"], s["axis"], s["wq"], s["wk"], qo, ko, eps=EPS)
        dq, dk = new(q), new(k)
        dwq, dwk = new(s["wq"], torch.float32), new(s["wk"], torch.float32)
        nbytes = hx.hexrotary_bwd_workspace(c["T"], c["Hq"], c["Hkv"], c["D"], hx._dtype_code(q))
        ws = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
        hx.hexrotary_bwd(q, k, s["pos"], s["freq"], s["axis"], s["wq"], s["wk"], s["dqo"],
                         s["dko"], dq, dk, dwq, dwk, ws, eps=EPS)
        return [qo, ko, dq, dk, dwq, dwk]
    if kind == "attn":
        q, k, v = _split(s["qkv"], c)
        o = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
        hx.hexattn_fwd(q, k, v, o, lse, s["start"], causal=c["causal"])
        if not c["bwd"]:
            return [o, lse]
        # one gradient of the projection's output, as the projection takes it
        dqkv = torch.empty_like(s["qkv"])
        dq, dk, dv = _split(dqkv, c)
        nbytes = hx.hexattn_bwd_workspace(q.shape[0], k.shape[0], c["S"], c["Hq"], c["Hkv"],
                                          c["D"], hx._dtype_code(q))
        ws = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
        hx.hexattn_bwd(q, k, v, o, lse, s["do"], dq, dk, dv, ws, s["start"], causal=c["causal"])
        return [o, dqkv]
    if kind == "step":
        o = torch.empty_like(s["q"])
        nbytes = hx.hexattn_step_workspace(c["S"], c["n"], c["Hq"], c["Hkv"], c["D"], s["cap"],
                                           hx._dtype_code(o))
        ws = torch.empty(nbytes, dtype=torch.uint8, device=o.device)
        hx.hexattn_step(s["q"], s["kc"], s["vc"], o, ws, s["start"], s["len"], s["cap"])
        return [o]
    y = torch.empty_like(s["x"])
    hx.hexdropout(s["x"], s["res"], y, c["p"], s["rng"])
    if not c["bwd"]:
        return [y]
    dx = torch.empty_like(s["x"])
    hx.hexdropout(s["dy"], None, dx, c["p"], s["rng"])
    return [y, dx]


# --------------------------------------------------------------- plain form

def _plain_rotate(x, w, cos, sin):
    """Norm and rotation of [T][heads][D] in 32 bits: the result, and what
    the backward needs."""
    x = x.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * r
    y = n * w.float()
    h = x.shape[-1] // 2
    a, b = y[..., :h], y[..., h:]
    return torch.cat([a * cos - b * sin, a * sin + b * cos], -1), n, r


def _plain_rotate_bwd(dy, n, r, w, cos, sin):
    dy = dy.float()
    h = dy.shape[-1] // 2
    a, b = dy[..., :h], dy[..., h:]
    g = torch.cat([a * cos + b * sin, b * cos - a * sin], -1)
    dw = (g * n).sum((0, 1))
    g = g * w.float()
    return r * (g - n * (g * n).mean(-1, keepdim=True)), dw


def _plain_rotary(s):
    c = s["case"]
    q, k, v = _split(s["qkv"], c)
    ang = s["pos"][:, s["axis"].long()] * s["freq"]
    cos, sin = ang.cos()[:, None], ang.sin()[:, None]
    qo, nq, rq = _plain_rotate(q, s["wq"], cos, sin)
    ko, nk, rk = _plain_rotate(k, s["wk"], cos, sin)
    if c["kind"] == "append":
        at = s["slot"].long()
        s["kc"][at] = ko.to(k.dtype)
        s["vc"][at] = v
        return [qo.to(q.dtype), s["kc"], s["vc"]]
    dq, dwq = _plain_rotate_bwd(s["dqo"], nq, rq, s["wq"], cos, sin)
    dk, dwk = _plain_rotate_bwd(s["dko"], nk, rk, s["wk"], cos, sin)
    t = q.dtype
    return [qo.to(t), ko.to(t), dq.to(t), dk.to(t), dwq, dwk]


SCORES = 1 << 28  # held at once


def _batches(lens, heads):
    """Sequences of like length together, by their numbers."""
    out = []
    for i in sorted(range(len(lens)), key=lambda i: -lens[i]):
        most = lens[out[-1][0]] if out else 0
        if out and 2 * lens[i] >= most and (len(out[-1]) + 1) * heads * most * most <= SCORES:
            out[-1].append(i)
        else:
            out.append([i])
    return out


def _padded(x, at):
    """Rows `at` [B][n] of [T][heads][D] in 32 bits: [B][heads][n][D]."""
    return x[at].float().transpose(1, 2).contiguous()


def _plain_attn_batch(q, k, v, nq, nk, scale, causal, do=None):
    """Attention of B sequences padded to one length: q [B][Hq][n][D], k and v
    [B][Hkv][m][D], nq and nk their lengths [B]; output, log of the sum of
    exponentials, and with `do` (zero in the padding) the gradients, in pieces
    of the queries.  Causal: a sequence's last query sees every key."""
    B, Hq, n, D = q.shape
    Hkv, m = k.shape[1:3]
    dev = q.device
    kt, vt = k.transpose(2, 3).contiguous(), v.transpose(2, 3).contiguous()
    o, lse = torch.empty_like(q), torch.empty((B, Hq, n), device=dev)
    if do is not None:
        dq, dk, dv = torch.empty_like(q), torch.zeros_like(k), torch.zeros_like(v)
    j = torch.arange(m, device=dev)
    last = nk.view(B, 1, 1) - 1
    piece = max(1, min(n, SCORES // max(1, B * Hq * m)))
    for a in range(0, n, piece):
        b = min(n, a + piece)
        group = lambda t: t[:, :, a:b].reshape(B, Hkv, -1, D)  # noqa: E731
        whole = lambda t: t.reshape(B, Hq, b - a, -1)  # noqa: E731
        qs = group(q)
        x = torch.matmul(qs, kt) * scale
        see = last.expand(B, b - a, 1)
        if causal:
            i = torch.arange(a, b, device=dev).view(1, -1, 1)
            see = torch.minimum(last, i + last + 1 - nq.view(B, 1, 1))
        x = whole(x).masked_fill_((j > see).unsqueeze(1), float("-inf")).view(B, Hkv, -1, m)
        top = x.amax(-1, keepdim=True)
        p = torch.exp(x - top)
        z = p.sum(-1, keepdim=True)
        p = p / z
        os = torch.matmul(p, v)
        o[:, :, a:b] = whole(os)
        lse[:, :, a:b] = whole(top + z.log())[..., 0]
        if do is not None:
            g = group(do)
            dv += torch.matmul(p.transpose(2, 3), g)
            ds = p * (torch.matmul(g, vt) - (g * os).sum(-1, keepdim=True)) * scale
            dq[:, :, a:b] = whole(torch.matmul(ds, k))
            dk += torch.matmul(ds.transpose(2, 3), qs)
    return (o, lse) if do is None else (o, lse, dq, dk, dv)


def _plain_attn(s):
    c = s["case"]
    q, k, v = _split(s["qkv"], c)
    T = q.shape[0]
    # one row more, which takes the padding's results
    o, lse = q.new_empty((T + 1,) + q.shape[1:]), torch.empty((T + 1, c["Hq"]), device=q.device)
    d = q.new_empty((T + 1,) + s["qkv"].shape[1:]) if c["bwd"] else None
    n_all = (s["start"][1:] - s["start"][:-1]).long()
    for which in _batches(s["lens"], c["Hq"]):
        L = max(s["lens"][i] for i in which)
        ids = torch.tensor(which, device=q.device)
        n, i = n_all[ids], torch.arange(L, device=q.device)
        at = s["start"].long()[ids][:, None] + i
        here = i < n[:, None]
        at, to = at.clamp(max=T - 1), torch.where(here, at, T)
        do = _padded(s["do"], at) * here[:, None, :, None] if c["bwd"] else None
        r = _plain_attn_batch(_padded(q, at), _padded(k, at), _padded(v, at), n, n,
                              1.0 / math.sqrt(c["D"]), c["causal"], do)
        o[to] = r[0].transpose(1, 2).to(o.dtype)
        lse[to] = r[1].transpose(1, 2)
        if c["bwd"]:
            d[to] = torch.cat(r[2:], 1).transpose(1, 2).to(o.dtype)
    return [o[:T], d[:T]] if c["bwd"] else [o[:T], lse[:T]]


def _plain_step(s):
    c = s["case"]
    q, o = s["q"], torch.empty_like(s["q"])
    for which in _batches(s["lens"], c["Hq"]):
        L = max(s["lens"][i] for i in which)
        ids = torch.tensor(which, device=q.device)
        at = s["start"].long()[ids][:, None] + torch.arange(L, device=q.device)
        r = _plain_attn_batch(q[ids].float().transpose(1, 2).contiguous(), _padded(s["kc"], at),
                              _padded(s["vc"], at), torch.full_like(ids, c["n"]),
                              s["len"].long()[ids], 1.0 / math.sqrt(c["D"]), True)
        o[ids] = r[0].transpose(1, 2).to(o.dtype)
    return [o]


def _philox(n, rng, call=0):
    """32 random bits for each of n elements, as int64: Philox 4x32 with ten
    rounds (Salmon et al., SC 2011), one block for four elements.  Key: the
    64-bit seed rng[0]; counter: the block's number, then rng[1] + call."""
    low = 0xFFFFFFFF
    k0, k1 = rng[0] & low, (rng[0] >> 32) & low
    at = rng[1] + call
    i = torch.arange((n + 3) // 4, dtype=torch.int64, device=rng.device)
    x = [i & low, i >> 32, (at & low).expand_as(i), ((at >> 32) & low).expand_as(i)]
    for _ in range(10):
        a, b = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57  # wrapping in 64 bits keeps the bits
        x = [((b >> 32) & low) ^ x[1] ^ k0, b & low, ((a >> 32) & low) ^ x[3] ^ k1, a & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack(x, 1).reshape(-1)[:n]


def _plain_drop(s):
    c = s["case"]
    x = s["x"]
    keep = (_philox(x.numel(), s["rng"]) >= int(c["p"] * 2.0 ** 32)).view(x.shape)
    f = 1.0 / (1.0 - c["p"])
    zero = torch.zeros((), device=x.device)
    y = (torch.where(keep, x.float() * f, zero) + s["res"].float()).to(x.dtype)
    if not c["bwd"]:
        return [y]
    return [y, torch.where(keep, s["dy"].float() * f, zero).to(x.dtype)]


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind in ("rotary", "append"):
        return _plain_rotary(state)
    if kind == "attn":
        return _plain_attn(state)
    return _plain_step(state) if kind == "step" else _plain_drop(state)


# -------------------------------------------------------------------- work

def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    kind = c["kind"]
    if kind in ("rotary", "append"):
        T = c["T"] if kind == "rotary" else c["S"]
        qk, kv, D = c["Hq"] + c["Hkv"], c["Hkv"], c["D"]
        x = T * qk * D
        once = T * AXES * 4 + D // 2 * 8 + 2 * D * e
        if kind == "append":
            # queries, keys and values read, written to their places
            return {"bytes": 2 * (x + T * kv * D) * e + T * 4 + once, "flops": 8 * x}
        # forward: x read, y written; backward: x and dy read, dx written
        return {"bytes": 5 * x * e + 2 * once + 2 * D * 4, "flops": 24 * x}
    if kind == "attn":
        T, D = sum(_lengths(c)), c["D"]
        q, kv = T * c["Hq"] * D, T * c["Hkv"] * D
        stat = T * c["Hq"] * 4
        b, f = (2 * q + 2 * kv) * e + stat, 4
        if c["bwd"]:
            b += (4 * q + 4 * kv) * e + stat  # q, k, v, o, do read; dq, dk, dv written
            f += 10
        return {"bytes": b + 4 * (c["S"] + 1), "flops": f * D * c["Hq"] * _n_valid(c)}
    if kind == "step":
        D = c["D"]
        b = 2 * sum(_lengths(c)) * c["Hkv"] * D * e + 2 * c["S"] * c["n"] * c["Hq"] * D * e
        return {"bytes": b + 8 * c["S"], "flops": 4 * D * c["Hq"] * _n_valid(c)}
    n = c["rows"] * c["cols"]
    # x and the residual read, y written; dy read, dx written
    return {"bytes": (5 if c["bwd"] else 3) * n * e + 16, "flops": (2 if c["bwd"] else 1) * 2 * n}


# ------------------------------------------------------------------- exact

def _exact_rotary(s):
    c = s["case"]
    q, k, v = (t.double() for t in _split(s["qkv"], c))
    q, k = q.clone().requires_grad_(True), k.clone().requires_grad_(True)
    wq, wk = (s[n].double().requires_grad_(True) for n in ("wq", "wk"))
    turn = s["freq"].double() * s["pos"].double().index_select(1, s["axis"].long())
    turn = torch.polar(torch.ones_like(turn), turn).unsqueeze(1)

    def f(x, w):
        y = x * w / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + EPS)
        z = torch.complex(*y.chunk(2, -1)) * turn
        return torch.cat([z.real, z.imag], -1)

    qo, ko = f(q, wq), f(k, wk)
    if c["kind"] == "append":
        kc, vc = s["kc"].double(), s["vc"].double()
        kc.index_copy_(0, s["slot"].long(), ko.detach())
        vc.index_copy_(0, s["slot"].long(), v)
        return [qo.detach(), kc, vc]
    dq, dk, dwq, dwk = torch.autograd.grad([qo, ko], [q, k, wq, wk],
                                           [s["dqo"].double(), s["dko"].double()])
    return [qo.detach(), ko.detach(), dq, dk, dwq, dwk]


def _exact_head(q, k, v, causal, do):
    """One head of one sequence: [n][D] queries over [m][D] keys, aligned at
    their ends; output, log sum, gradients."""
    n, m = q.shape[0], k.shape[0]
    if do is not None:
        q, k, v = (t.clone().requires_grad_(True) for t in (q, k, v))
    x = q @ k.T / math.sqrt(q.shape[1])
    if causal:
        x = x + torch.full((n, m), -math.inf, dtype=x.dtype, device=x.device).triu(m - n + 1)
    o = torch.softmax(x, 1) @ v
    if do is None:
        return o, torch.logsumexp(x, 1)
    return o.detach(), torch.autograd.grad(o, (q, k, v), do)


def _exact_attn(s):
    c = s["case"]
    q, k, v = _split(s["qkv"], c)
    G = c["Hq"] // c["Hkv"]
    o = torch.empty(q.shape, dtype=torch.float64, device=q.device)
    lse = torch.empty(q.shape[:2], dtype=torch.float64, device=q.device)
    d = torch.zeros(s["qkv"].shape, dtype=torch.float64, device=q.device) if c["bwd"] else None
    a = 0
    for n in s["lens"]:
        at = slice(a, a + n)
        for h in range(c["Hq"]):
            j = h // G
            one = (q[at, h].double(), k[at, j].double(), v[at, j].double(), c["causal"])
            if c["bwd"]:
                o[at, h], (gq, gk, gv) = _exact_head(*one, s["do"][at, h].double())
                d[at, h] += gq
                d[at, c["Hq"] + j] += gk
                d[at, c["Hq"] + c["Hkv"] + j] += gv
            else:
                o[at, h], lse[at, h] = _exact_head(*one, None)
        a += n
    return [o, d] if c["bwd"] else [o, lse]


def _exact_step(s):
    c = s["case"]
    G = c["Hq"] // c["Hkv"]
    o = torch.empty(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    for i, m in enumerate(s["lens"]):
        at = slice(i * s["cap"], i * s["cap"] + m)
        for h in range(c["Hq"]):
            o[i, :, h] = _exact_head(s["q"][i, :, h].double(), s["kc"][at, h // G].double(),
                                     s["vc"][at, h // G].double(), True, None)[0]
    return [o]


def _exact_drop(s):
    """Philox in 16-bit halves, so that no product passes 63 bits."""
    c = s["case"]
    x = s["x"]
    n = x.numel()
    seed, at = int(s["rng"][0]), int(s["rng"][1])
    key = [seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF]
    i = torch.arange((n + 3) // 4, dtype=torch.int64, device=x.device)

    def product(w, m):
        low = (w & 0xFFFF) * m
        high = (w >> 16) * m + (low >> 16)
        return high >> 16, (high & 0xFFFF) << 16 | low & 0xFFFF

    w = [i % 2 ** 32, i // 2 ** 32, torch.full_like(i, at & 0xFFFFFFFF),
         torch.full_like(i, at >> 32 & 0xFFFFFFFF)]
    for r in range(10):
        (ha, la), (hb, lb) = product(w[0], 0xD2511F53), product(w[2], 0xCD9E8D57)
        w = [hb ^ w[1] ^ (key[0] + r * 0x9E3779B9) % 2 ** 32, lb,
             ha ^ w[3] ^ (key[1] + r * 0xBB67AE85) % 2 ** 32, la]
    bits = torch.stack(w, 1).flatten()[:n].view(x.shape)
    kept = (bits >= math.floor(c["p"] * 2 ** 32)).double() / (1 - c["p"])
    y = s["res"].double() + s["x"].double() * kept
    return [y, s["dy"].double() * kept] if c["bwd"] else [y]


def exact(case, seed):
    kind = case["kind"]
    # head after head in 64 bits: about 5 TFLOP/s with the exponentials
    if kind == "attn" and work(case)["flops"] * (1 if not case["causal"] else 2) > 5e13:
        return None
    s = prepare(case, seed)
    if kind in ("rotary", "append"):
        return _exact_rotary(s)
    if kind == "attn":
        return _exact_attn(s)
    return _exact_step(s) if kind == "step" else _exact_drop(s)
