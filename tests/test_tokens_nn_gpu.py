"""The layer norm, projection and feed-forward layers and the block of both with
attention: gradients against float64 autograd, the block over a cache against its
whole-sequence forward, recomputed forwards, captured graphs, inputs of any
strides."""
import math

import pytest

from gpu_helpers import torch_mod

torch = pytest.importorskip("torch")
hnn = pytest.importorskip("paper_1903_01814_amd.nn")
pytestmark = pytest.mark.gpu

F = torch.nn.functional
# Norms of differences.  float32: a few hundred roundings that add up as their
# root, 1e-5 holds all.  bfloat16: a result's rounding is 1.7e-3 of its norm (2^-8 at
# most, 2^-8 / sqrt 3 where values lie evenly, less towards a step's upper end) and a
# gradient passes through up to five of them, 2e-2 with room for their growth.
TOL = {torch.float32: 1e-5, torch.bfloat16: 2e-2}
DTYPES = [torch.float32, torch.bfloat16]


def rel(got, want):
    return float((got.detach().double().cpu() - want.detach()).norm() /
                 want.detach().norm().clamp_min(1e-300))


def both(module):
    """The module's parameters in float64 on the host, by name."""
    return {n: p.detach().double().cpu().requires_grad_(True) for n, p in module.named_parameters()}


def ffn64(p, x, act, pre=""):
    n = F.layer_norm(x, x.shape[-1:], p[pre + "norm.weight"], p[pre + "norm.bias"], 1e-5)
    g, u = F.linear(n, p[pre + "weight1"], p.get(pre + "bias1")).chunk(2, -1)
    f = {"silu": F.silu, "gelu": F.gelu, "relu": F.relu, None: lambda t: t}[act]
    return x + F.linear(f(g) * u, p[pre + "weight2"], p.get(pre + "bias2"))


def check(module, got, want, x, x64, p64, gy, tol):
    assert rel(got, want) <= tol
    names = [n for n, _ in module.named_parameters()]
    grads = torch.autograd.grad(got, [x, *module.parameters()], gy)
    wants = torch.autograd.grad(want, [x64, *(p64[n] for n in names)], gy.double().cpu())
    for n, a, b in zip(["x"] + names, grads, wants):
        assert a.dtype == x.dtype
        assert rel(a, b) <= tol, (n, rel(a, b))


def shaken(module, seed=3):
    """Weights of a norm and biases away from their initial values."""
    torch.manual_seed(seed)
    with torch.no_grad():
        for p in module.parameters():
            if p.dim() == 1:
                p.add_(torch.randn_like(p) * 0.3)
    return module


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(5, 33), (2, 3, 64), (257, 104), (1, 7)])
def test_layer_norm(shape, dtype):
    torch_mod()
    m = shaken(hnn.HexLayerNorm(shape[-1], device="cuda", dtype=dtype))
    x = torch.randn(shape, device="cuda").to(dtype).requires_grad_(True)
    p, x64 = both(m), x.detach().double().cpu().requires_grad_(True)
    want = F.layer_norm(x64, shape[-1:], p["weight"], p["bias"], 1e-5)
    check(m, m(x), want, x, x64, p, torch.randn(shape, device="cuda").to(dtype), TOL[dtype])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", [None, "gelu", "silu"])
@pytest.mark.parametrize("shape,out", [((4, 40), 24), ((3, 50, 33), 41), ((300, 64), 128)])
def test_linear(shape, out, act, dtype):
    torch_mod()
    m = hnn.HexLinear(shape[-1], out, activation=act, device="cuda", dtype=dtype)
    x = torch.randn(shape, device="cuda").to(dtype).requires_grad_(True)
    r = torch.randn(shape[:-1] + (out,), device="cuda").to(dtype).requires_grad_(True)
    gy = torch.randn(r.shape, device="cuda").to(dtype)
    p, x64 = both(m), x.detach().double().cpu().requires_grad_(True)
    f = {"silu": F.silu, "gelu": F.gelu, None: lambda t: t}[act]
    want = f(F.linear(x64, p["weight"], p["bias"])) + r.detach().double().cpu()
    check(m, m(x, residual=r), want, x, x64, p, gy, TOL[dtype])
    assert torch.equal(torch.autograd.grad(m(x, residual=r), r, gy)[0], gy)
    # without a backward to follow: the same bits
    with torch.no_grad():
        assert torch.equal(m(x, residual=r), m(x.detach(), residual=r.detach()))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", [None, "gelu", "silu"])
@pytest.mark.parametrize("shape,hidden,bias", [((3, 40), 56, True), ((150, 64), 177, False),
                                               ((2, 60, 33), 41, True)])
def test_feed_forward(shape, hidden, bias, act, dtype):
    torch_mod()
    torch.manual_seed(1)
    m = shaken(hnn.HexFeedForward(shape[-1], hidden, act, bias, device="cuda", dtype=dtype))
    x = torch.randn(shape, device="cuda").to(dtype).requires_grad_(True)
    p, x64 = both(m), x.detach().double().cpu().requires_grad_(True)
    gy = torch.randn(shape, device="cuda").to(dtype)
    check(m, m(x), ffn64(p, x64, act), x, x64, p, gy, TOL[dtype])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("normed", [False, True])
def test_feed_forward_function(normed, residual, dtype):
    """Every subset of inputs that take a gradient."""
    torch_mod()
    g = torch.Generator().manual_seed(7)
    mk = lambda *s, k=1.0: (torch.randn(s, generator=g) * k).to(dtype).cuda()  # noqa: E731
    x, w1, w2, b1, b2, nw = mk(70, 32), mk(80, 32, k=0.2), mk(32, 40, k=0.2), mk(80), mk(32), mk(32)
    gy = mk(70, 32)
    ins = dict(x=x, w1=w1, w2=w2, b1=b1, b2=b2, nw=nw)

    def run(wanted):
        t = {k: v.clone().requires_grad_(k in wanted) for k, v in ins.items()}
        y = hnn.hex_feed_forward(t["x"], t["w1"], t["w2"], t["b1"], t["b2"], "gelu", residual,
                                 (t["nw"], None, 1e-5) if normed else None)
        return dict(zip(wanted, torch.autograd.grad(y, [t[k] for k in wanted], gy)))

    all_of = [k for k in ins if normed or k != "nw"]
    want = run(all_of)
    x64 = {k: v.double().cpu().requires_grad_(True) for k, v in ins.items()}
    n = F.layer_norm(x64["x"], (32,), x64["nw"], None, 1e-5) if normed else x64["x"]
    a, b = F.linear(n, x64["w1"], x64["b1"]).chunk(2, -1)
    y = F.linear(F.gelu(a) * b, x64["w2"], x64["b2"]) + (x64["x"] if residual else 0)
    for k, t in zip(all_of, torch.autograd.grad(y, [x64[k] for k in all_of], gy.double().cpu())):
        assert rel(want[k], t) <= TOL[dtype], k
    for wanted in (["x"], ["w1"], ["b1"], ["w2"], ["b2"], ["x", "w2"], ["w1", "b2"]):
        for k, t in run(wanted).items():
            if k[0] == "b" and "w" + k[1] not in wanted:  # summed in another order
                assert rel(t, want[k].double().cpu()) <= TOL[dtype], (wanted, k)
            else:
                assert torch.equal(t, want[k]), (wanted, k)


@pytest.mark.parametrize("dtype", DTYPES)
def test_inputs_as_they_come(dtype):
    """Transposed, sliced, shifted and expanded inputs and gradients."""
    torch_mod()
    torch.manual_seed(0)
    ff = hnn.HexFeedForward(24, 40, device="cuda", dtype=dtype)
    lin = hnn.HexLinear(24, 33, activation="silu", device="cuda", dtype=dtype)
    big = torch.randn(60, 100, device="cuda").to(dtype)
    views = [big.t()[:50, :24], big[:50, 1:25], big[3:53, 8:32], big[:1, :24].expand(50, 24),
             big.view(-1)[5:5 + 50 * 24].view(50, 24), big[::2][:, :24]]
    for v in views:
        for m in (ff, lin, ff.norm):
            got = []
            for x in (v, v.clone(memory_format=torch.contiguous_format)):
                x = x.detach().requires_grad_(True)
                y = m(x)
                got.append([y.detach(), torch.autograd.grad(y.sum(), x)[0],
                            *torch.autograd.grad(m(x)[:, ::2].sum(), list(m.parameters()))])
            for a, b in zip(*got):
                assert torch.equal(a, b)


def test_relu_layer():
    torch_mod()
    m = hnn.HexLinear(20, 30, activation="relu", device="cuda")
    x = torch.randn(40, 20, device="cuda", requires_grad=True)
    y = m(x)
    want = torch.relu(F.linear(x, m.weight, m.bias))
    assert rel(y, want.double().cpu()) <= 1e-6
    gy = torch.randn_like(y)
    for a, b in zip(torch.autograd.grad(y, [x, m.weight], gy),
                    torch.autograd.grad(want, [x, m.weight], gy)):
        assert rel(a, b.double().cpu()) <= 1e-6


def refuse(f, kind, match):
    with pytest.raises(kind, match=match):
        f()


def test_layers_refuse():
    torch_mod()
    refuse(lambda: hnn.HexLinear(8, 8, activation="tanh"), ValueError, "no activation")
    x, w = torch.randn(4, 8, device="cuda"), torch.randn(6, 8, device="cuda")
    refuse(lambda: hnn.hex_linear(x, w, residual=x), ValueError, "residual has shape")
    refuse(lambda: hnn.hex_linear(x, w.bfloat16()), TypeError, "dtype")
    refuse(lambda: hnn.hex_linear(x, w[:, :7]), ValueError, "shape")
    refuse(lambda: hnn.hex_linear(x.half(), w.half()), TypeError, "unsupported dtype")
    refuse(lambda: hnn.hex_feed_forward(x, torch.randn(12, 8, device="cuda"), w, residual=True),
           ValueError, "residual needs")
    refuse(lambda: hnn.hex_layer_norm(x, w[0, :4]), ValueError, "shape")


# ------------------------------------------------------------------- the block

def block(dtype=torch.float32, seed=0, dim=48, **kw):
    torch.manual_seed(seed)
    b = hnn.HexPixelBlock(dim, 4, 2, 16, hidden=72, device="cuda", dtype=dtype, **kw)
    return shaken(b)


def tokens(dtype, lens, dim=48, seed=1):
    g = torch.Generator().manual_seed(seed)
    T = sum(lens)
    start = [0]
    for n in lens:
        start.append(start[-1] + n)
    return (torch.randn(T, dim, generator=g).to(dtype).cuda(), torch.rand(T, 3, generator=g).cuda() * 9,
            torch.tensor(start, dtype=torch.int32, device="cuda"))


def attention64(p, x, pos, freq, axis, lens, heads, D, causal):
    """The attention layer with its norm in float64."""
    Hq, Hkv = heads
    n = F.layer_norm(x, x.shape[-1:], p["norm.weight"], p["norm.bias"], 1e-5)
    qkv = F.linear(n, p["qkv.weight"]).view(-1, Hq + 2 * Hkv, D)
    ang = pos[:, axis.long()] * freq
    c, s = ang.cos()[:, None], ang.sin()[:, None]

    def turn(t, w):
        y = t * torch.rsqrt((t * t).mean(-1, keepdim=True) + 1e-6) * w
        a, b = y.chunk(2, -1)
        return torch.cat([a * c - b * s, a * s + b * c], -1)

    q, k, v = turn(qkv[:, :Hq], p["q_norm"]), turn(qkv[:, Hq:Hq + Hkv], p["k_norm"]), qkv[:, Hq + Hkv:]
    out, at = [], 0
    for m in lens:
        rows = []
        for h in range(Hq):
            j = h * Hkv // Hq
            y = q[at:at + m, h] @ k[at:at + m, j].T / math.sqrt(D)
            if causal:
                y = y.masked_fill(torch.ones(m, m).triu(1).bool(), -math.inf)
            rows.append(torch.softmax(y, 1) @ v[at:at + m, j])
        out.append(torch.stack(rows, 1))
        at += m
    return x + F.linear(torch.cat(out).flatten(1), p["out.weight"])


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens", [[40, 1, 60], [3]])
def test_block_gradients(lens, dtype, causal):
    """The operators together, forward and backward, against float64."""
    torch_mod()
    b = block(dtype, causal=causal)
    x, pos, start = tokens(dtype, lens)
    x.requires_grad_(True)
    p = both(b)
    x64 = x.detach().double().cpu().requires_grad_(True)
    pa = {n[len("attention."):]: t for n, t in p.items() if n.startswith("attention.")}
    y = attention64(pa, x64, pos.double().cpu(), b.attention.freq.double().cpu(),
                    b.attention.axis.cpu(), lens, (4, 2), 16, causal)
    want = ffn64(p, y, "silu", "feed_forward.")
    gy = torch.randn(x.shape, device="cuda").to(dtype)
    check(b, b(x, pos, start), want, x, x64, p, gy, 2 * TOL[dtype])


# bfloat16: values up to 5, rounded at some ten places on either way
@pytest.mark.parametrize("dtype,lim", [(torch.float32, 3e-5), (torch.bfloat16, 0.1)])
def test_block_streams(dtype, lim):
    """Prompts and steps over a cache give what the whole sequences give."""
    torch_mod()
    b = block(dtype, causal=True).eval()
    lens, new = [7, 0, 12, 40], 5
    x, pos, start = tokens(dtype, [n + new for n in lens])
    whole = b(x, pos, start).detach()
    first = [int(s) for s in start[:-1]]
    cut = lambda t: torch.cat([t[a:a + n] for a, n in zip(first, lens)])  # noqa: E731
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    cache = b.new_cache(4, 50)
    got = b.prefill(cut(x), cut(pos), torch.tensor(at, dtype=torch.int32, device="cuda"), cache, 40)
    assert float((got.float() - cut(whole).float()).abs().max()) <= lim
    t = 0
    while t < new:
        n = min(2, new - t)
        pick = lambda v: torch.stack([v[a + m + t:a + m + t + n] for a, m in zip(first, lens)])  # noqa: E731
        y = b.step(pick(x), pick(pos), cache)
        assert y.shape == (4, n, 48)
        assert float((y.float() - pick(whole).float()).abs().max()) <= lim
        t += n


@pytest.mark.parametrize("dtype", DTYPES)
def test_checkpointed_block(dtype):
    torch_mod()
    from torch.utils.checkpoint import checkpoint
    b = block(dtype, dropout=0.3)
    x, pos, start = tokens(dtype, [30, 50])
    gy = torch.randn(x.shape, device="cuda").to(dtype)
    got = []
    for run in (b, lambda *a: checkpoint(b, *a, use_reentrant=False)):
        torch.manual_seed(5)
        xi = x.clone().requires_grad_(True)
        y = run(xi, pos, start)
        got.append([y.detach(), *torch.autograd.grad(y, [xi, *b.parameters()], gy)])
    for u, v in zip(*got):
        assert torch.equal(u, v)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens", [[2], [90, 60]])
def test_captured_block(dtype, lens):
    """Forward and gradients recorded once: every replay has the eager call's bits
    for new inputs, with eager work between."""
    torch_mod()
    b = block(dtype)
    x, pos, start = tokens(dtype, lens)
    x.requires_grad_(True)
    gy = torch.randn(x.shape, device="cuda").to(dtype)
    params = [x, *b.parameters()]

    def work():
        y = b(x, pos, start)
        return [y.detach(), *torch.autograd.grad(y, params, gy)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work()
    for i in range(4):
        with torch.no_grad():
            x.normal_()
        for t in out:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for u, v in zip(out, work()):
            assert torch.equal(u, v)


@pytest.mark.parametrize("dtype", DTYPES)
def test_block_without_tokens(dtype):
    torch_mod()
    b = block(dtype, dropout=0.5, causal=True)
    x, pos, start = tokens(dtype, [])
    x.requires_grad_(True)
    y = b(x, pos, start)
    assert y.shape == (0, 48)
    for g, p in zip(torch.autograd.grad(y, [x, *b.parameters()], torch.empty_like(y)),
                    [x, *b.parameters()]):
        assert g.shape == p.shape and not bool(g.any())
    b.eval()
    cache = b.new_cache(0, 4)
    assert b.step(x.view(0, 2, 48), pos.view(0, 2, 3), cache).shape == (0, 2, 48)


def test_layer_without_norm_is_as_it_was():
    """The attention layer's states have no new entries, and its results are those of
    its parts."""
    torch_mod()
    torch.manual_seed(2)
    layer = hnn.HexPixelAttention(48, 4, 2, 16, device="cuda")
    assert sorted(layer.state_dict()) == ["k_norm", "out.weight", "q_norm", "qkv.weight"]
    x, pos, start = tokens(torch.float32, [20, 9])
    o = hnn.HexPixelAttentionFunction.apply(layer.qkv(x).view(-1, 8, 16), layer.q_norm, layer.k_norm,
                                            pos, layer.freq, layer.axis, start, (4, 2), 1e-6, False)
    assert torch.equal(layer(x, pos, start), x + layer.out(o.flatten(1)))


def test_second_derivatives_refused():
    """The gradients' own gradients are not there: asked for, they raise."""
    d = dict(device="cuda")
    x = torch.randn(5, 8, requires_grad=True, **d)
    w = torch.randn(8, 8, requires_grad=True, **d)
    w1, w2 = (torch.randn(s, requires_grad=True, **d) for s in ((16, 8), (8, 8)))
    for y in (hnn.hex_layer_norm(x, w[0]), hnn.hex_linear(x, w),
              hnn.hex_feed_forward(x, w1, w2, norm=(None, None, 1e-5))):
        gx, = torch.autograd.grad(y.square().sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            gx.sum().backward()
