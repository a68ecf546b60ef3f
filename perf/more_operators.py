"""The token-wise half of a transformer block over pixel tokens, as cases to be
timed.

The lit pixels of camera events are packed tokens [tokens][features].  Beside
attention, a network over them has these operators, each acting on every token
by itself:

 - ``norm``: layer norm with weights, forward and backward; the backward adds
   the residual branch's gradient and sums the weights' gradients;
 - ``linear``: a projection with bias, activation and residual in its
   epilogue, forward and backward;
 - ``ffn``: a gated feed-forward block with residual, y = (act(x wg^T + bg)
   (x wu^T + bu)) w2^T + b2 + res, forward and backward.

``run`` computes a case in elementary torch operations in 32 bits, or, where
``own`` is true, by the library's entry points.  ``exact`` evaluates the
definitions in 64 bits, gradients by automatic differentiation.  Gradients of
weights and biases come in the weights' type, those of the norm in float32.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


# ------------------------------------------------------------------- cases

def norm(name, T, C, dtype, bwd):
    return dict(name=name, kind="norm", T=T, C=C, dtype=dtype, bwd=bwd)


def linear(name, T, K, N, dtype, act, bias, res, bwd):
    return dict(name=name, kind="linear", T=T, K=K, N=N, dtype=dtype, act=act, bias=bias, res=res,
                bwd=bwd)


def ffn(name, T, K, F, dtype, act, bias, res, bwd):
    return dict(name=name, kind="ffn", T=T, K=K, F=F, dtype=dtype, act=act, bias=bias, res=res,
                bwd=bwd)


def listed():
    return [
        # one new token each of four event streams: a serving call, whose time
        # is its launch
        norm("norm_step_bf16", 4, 2048, "bf16", False),
        # one time-resolved event's lit pixels in torch's default dtype, a
        # number of features that no vector divides
        norm("norm_odd_f32", 3287, 97, "f32", True),
        # a training batch: 32 planes of 40 x 40 pixels
        norm("norm_batch_bf16", 51200, 1024, "bf16", True),
        # the output projection of one new token of each of four streams: time
        # is the reading of the weights
        linear("linear_step_bf16", 4, 2048, 2048, "bf16", "none", False, True, False),
        # one camera image through a layer of odd sizes, training
        linear("linear_odd_f32", 1027, 97, 211, "f32", "gelu", True, False, True),
        # a batch of camera images in torch's default dtype, training
        linear("linear_image_f32", 16432, 512, 512, "f32", "none", True, True, True),
        # a training batch through a projection with activation and residual
        linear("linear_batch_bf16", 51200, 1024, 1024, "bf16", "gelu", True, True, True),
        # one long stream's prompt through the output projection, inference
        linear("linear_prompt_bf16", 16432, 2048, 2048, "bf16", "none", False, True, False),
        # one new token each of three streams
        ffn("ffn_step_bf16", 3, 2048, 5464, "bf16", "silu", False, True, False),
        # an event of odd sizes throughout, training
        ffn("ffn_odd_bf16", 3287, 200, 531, "bf16", "silu", True, True, True),
        # four camera images in torch's default dtype, training
        ffn("ffn_camera_f32", 4108, 256, 683, "f32", "gelu", True, True, True),
        # a batch of time-ordered pixels of long events, training: the largest
        # case
        ffn("ffn_batch_bf16", 16432, 2048, 5464, "bf16", "silu", False, True, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size over the logarithm of the range: any, or a multiple of 8 or 64,
    as sizes of features are."""
    step = rng.choice([1, 8, 8, 64])
    return max(lo, _log(rng, lo, hi) // step * step)


def draw(rng):
    kind = rng.choice(["norm", "norm", "linear", "linear", "linear", "ffn", "ffn", "ffn"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    bwd = rng.random() < 0.6
    # tokens: a step of a few streams, or up to a training batch
    T = _log(rng, 1, 64) if not bwd and rng.random() < 0.5 else _log(rng, 64, 51200)
    if kind == "norm":
        c = norm("", T, _size(rng, 24, 4096), dtype, bwd)
    elif kind == "linear":
        c = linear("", T, _size(rng, 24, 2048), _size(rng, 24, 2048), dtype,
                   rng.choice(["none", "gelu", "silu"]), rng.random() < 0.5, rng.random() < 0.5,
                   bwd)
    else:
        c = ffn("", T, _size(rng, 32, 2048), _size(rng, 64, 5464), dtype,
                rng.choice(["silu", "silu", "gelu"]), rng.random() < 0.5, rng.random() < 0.5, bwd)
    # float32 products run at an eighth of the rate of bf16
    most = max(_cost(x) for x in listed()) * (0.1 if dtype == "f32" else 0.9)
    while c["T"] > 1 and _cost(c) > most:
        c["T"] = (c["T"] + 1) // 2
    c.pop("name", None)
    return c


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


def prepare(case, seed):
    c = case
    g = _Gen(c, seed)
    s = {"case": c}
    T = c["T"]
    if c["kind"] == "norm":
        C = c["C"]
        s["x"] = g.normal(T, C, std=1.5, mean=0.3)
        s["w"], s["b"] = g.normal(C, std=0.1, mean=1.0), g.normal(C, std=0.1)
        if c["bwd"]:
            s["dy"], s["res"] = g.normal(T, C), g.normal(T, C)
        return s
    K = c["K"]
    N = c["N"] if c["kind"] == "linear" else K
    s["x"] = g.normal(T, K)
    if c["kind"] == "linear":
        s["w"] = g.normal(N, K, std=K ** -0.5)
        s["b"] = g.normal(N, std=0.2) if c["bias"] else None
    else:
        F = c["F"]
        # rows of the gate, then rows of the other projection
        s["w1"], s["w2"] = g.normal(2 * F, K, std=K ** -0.5), g.normal(N, F, std=F ** -0.5)
        s["b1"] = g.normal(2 * F, std=0.2) if c["bias"] else None
        s["b2"] = g.normal(N, std=0.2) if c["bias"] else None
    s["res"] = g.normal(T, N) if c["res"] else None
    if c["bwd"]:
        s["dy"] = g.normal(T, N)
    return s


# ---------------------------------------------------------------- own calls

def _own(s):
    from paper_1903_01814_amd import hexconv as hx
    c, x = s["case"], s["x"]
    T, dt = x.shape[0], hx._dtype_code(s["x"])
    new = lambda *shape, dtype=x.dtype: torch.empty(shape, dtype=dtype, device=x.device)  # noqa: E731
    like = lambda t: None if t is None else torch.empty_like(t)  # noqa: E731

    def space(nbytes):
        return new(nbytes, dtype=torch.uint8) if nbytes else None

    if c["kind"] == "norm":
        C = c["C"]
        y = torch.empty_like(x)
        if not c["bwd"]:
            hx.hexnorm_fwd(x, s["w"], s["b"], y, eps=EPS)
            return [y]
        mean, rstd = new(T, dtype=torch.float32), new(T, dtype=torch.float32)
        hx.hexnorm_fwd(x, s["w"], s["b"], y, mean, rstd, eps=EPS)
        dx = torch.empty_like(x)
        dw, db = new(C, dtype=torch.float32), new(C, dtype=torch.float32)
        hx.hexnorm_bwd(x, s["w"], mean, rstd, s["dy"], s["res"], dx, dw, db,
                       space(hx.hexnorm_bwd_workspace(T, C, dt)))
        return [y, dx, dw, db]
    act = {"none": hx.HEX_ACT_NONE, "gelu": hx.HEX_ACT_GELU, "silu": hx.HEX_ACT_SILU}[c["act"]]
    K = c["K"]
    if c["kind"] == "linear":
        N = c["N"]
        y = new(T, N)
        # the backward of an activation needs what it was applied to
        z = new(T, N) if c["bwd"] and act != hx.HEX_ACT_NONE else None
        hx.hexlinear_fwd(x, s["w"], s["b"], s["res"], y, z,
                         space(hx.hexlinear_fwd_workspace(T, N, K, K, dt)), act=act)
        if not c["bwd"]:
            return [y]
        dx, dw, db = torch.empty_like(x), torch.empty_like(s["w"]), like(s["b"])
        hx.hexlinear_bwd(x, s["w"], z, s["dy"], dx, dw, db,
                         space(hx.hexlinear_bwd_workspace(T, N, K, K, N, act, dt)), act=act)
        return [y, dx, dw] + ([db] if c["bias"] else [])
    F, N = c["F"], K
    Fp = hx.hexffn_width(F)
    y, h = new(T, N), new(T, Fp)
    gu = new(T, 2 * Fp) if c["bwd"] else None
    hx.hexffn_fwd(x, s["w1"], s["b1"], s["w2"], s["b2"], s["res"], y, gu, h,
                  space(hx.hexffn_fwd_workspace(T, K, F, N, K, dt)), act=act)
    if not c["bwd"]:
        return [y]
    dx, dw1, dw2 = torch.empty_like(x), torch.empty_like(s["w1"]), torch.empty_like(s["w2"])
    db1, db2 = like(s["b1"]), like(s["b2"])
    hx.hexffn_bwd(x, s["w1"], s["w2"], gu, h, s["dy"], dx, dw1, db1, dw2, db2,
                  space(hx.hexffn_bwd_workspace(T, K, F, N, K, N, dt)), act=act)
    return [y, dx, dw1, dw2] + ([db1, db2] if c["bias"] else [])


# --------------------------------------------------------------- plain form

def _act(z, act):
    """Activation and its derivative in 32 bits."""
    if act == "none":
        return z, None
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return z * s, s * (1.0 + z * (1.0 - s))
    phi = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z * phi, phi + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_norm(s):
    c, x = s["case"], s["x"].float()
    w = s["w"].float()
    d = x - x.mean(1, keepdim=True)
    r = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
    n = d * r
    t = s["x"].dtype
    y = (n * w + s["b"].float()).to(t)
    if not c["bwd"]:
        return [y]
    dy = s["dy"].float()
    g = dy * w
    dx = r * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True)) + s["res"].float()
    return [y, dx.to(t), (dy * n).sum(0), dy.sum(0)]


def _plain_linear(s):
    c, x, w = s["case"], s["x"].float(), s["w"].float()
    z = x @ w.T
    if c["bias"]:
        z = z + s["b"].float()
    y, d = _act(z, c["act"])
    if c["res"]:
        y = y + s["res"].float()
    t = s["x"].dtype
    if not c["bwd"]:
        return [y.to(t)]
    dz = s["dy"].float()
    if d is not None:
        dz = dz * d
    out = [y, dz @ w, dz.T @ x] + ([dz.sum(0)] if c["bias"] else [])
    return [o.to(t) for o in out]


def _plain_ffn(s):
    c, x, w1, w2 = s["case"], s["x"].float(), s["w1"].float(), s["w2"].float()
    F = c["F"]
    z = x @ w1.T
    if c["bias"]:
        z = z + s["b1"].float()
    u = z[:, F:]
    a, d = _act(z[:, :F], c["act"])
    h = a * u
    y = h @ w2.T
    if c["bias"]:
        y = y + s["b2"].float()
    if c["res"]:
        y = y + s["res"].float()
    t = s["x"].dtype
    if not c["bwd"]:
        return [y.to(t)]
    dy = s["dy"].float()
    dh = dy @ w2
    dz = torch.cat([dh * u * d, dh * a], 1)
    out = [y, dz @ w1, dz.T @ x, dy.T @ h]
    if c["bias"]:
        out += [dz.sum(0), dy.sum(0)]
    return [o.to(t) for o in out]


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_norm, "linear": _plain_linear, "ffn": _plain_ffn}[
        state["case"]["kind"]](state)


# -------------------------------------------------------------------- work

def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    T = c["T"]
    if c["kind"] == "norm":
        x = T * c["C"]
        # x read, y written; dy and the residual's gradient read, dx written
        b = (5 if c["bwd"] else 2) * x * e + 2 * c["C"] * e + (8 * c["C"] if c["bwd"] else 0)
        return {"bytes": b, "flops": (20 if c["bwd"] else 8) * x}
    K = c["K"]
    if c["kind"] == "linear":
        N, weights, bias = c["N"], c["N"] * K, c["N"] if c["bias"] else 0
    else:
        N, weights, bias = K, 3 * c["F"] * K, 2 * c["F"] + K if c["bias"] else 0
    b = T * K + weights + bias + T * N * (2 if c["res"] else 1)
    if c["bwd"]:
        b += T * N + T * K + weights + bias  # dy read; dx and the weights' gradients written
    return {"bytes": b * e, "flops": (6 if c["bwd"] else 2) * T * weights}


# ------------------------------------------------------------------- exact

def _grad_of(y, wanted, dy):
    grads = torch.autograd.grad(y, [t for t in wanted if t is not None], dy.double())
    return [y.detach()] + list(grads)


def exact(case, seed):
    c = case
    # products in 64 bits: about 30 TFLOP/s
    if work(c)["flops"] > 4e14:
        return None
    s = prepare(c, seed)
    v = {k: t.double() if torch.is_tensor(t) else None for k, t in s.items()}
    if c["bwd"]:
        for k in ("x", "w", "b", "w1", "b1", "w2", "b2"):
            if v.get(k) is not None:
                v[k].requires_grad_(True)
    lin = torch.nn.functional.linear
    act = {"none": lambda t: t, "silu": torch.nn.functional.silu,
           "gelu": torch.nn.functional.gelu}[c.get("act", "none")]
    if c["kind"] == "norm":
        y = torch.nn.functional.layer_norm(v["x"], (c["C"],), v["w"], v["b"], EPS)
        if not c["bwd"]:
            return [y]
        y, dx, dw, db = _grad_of(y, [v["x"], v["w"], v["b"]], s["dy"])
        return [y, dx + v["res"], dw, db]
    if c["kind"] == "linear":
        y = act(lin(v["x"], v["w"], v["b"]))
        wanted = [v["x"], v["w"], v["b"]]
    else:
        gate, up = lin(v["x"], v["w1"], v["b1"]).split(c["F"], 1)
        y = lin(act(gate) * up, v["w2"], v["b2"])
        wanted = [v["x"], v["w1"], v["w2"], v["b1"], v["b2"]]
    if c["res"]:
        y = y + v["res"]
    return _grad_of(y, wanted, s["dy"]) if c["bwd"] else [y]
