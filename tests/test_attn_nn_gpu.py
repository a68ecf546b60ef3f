"""The attention layer and its functions under autograd, and the example that
runs them together: gradients against float64 autograd, dropout's gradient
under the same mask, training on events of lit pixels, streams over a cache."""
import math
import os
import sys

import pytest

import attn_ref as ref
from gpu_helpers import torch_mod

torch = pytest.importorskip("torch")
hnn = pytest.importorskip("paper_1903_01814_amd.nn")
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))
pytestmark = pytest.mark.gpu


def rel(got, want):
    return float((got.detach().double().cpu() - want).norm() / want.norm().clamp_min(1e-300))


def layer64(qkv, wq, wk, pos, freq, axis, lens, heads, causal):
    """Norm, rotation and attention of one tensor in float64, differentiable."""
    Hq, Hkv = heads
    ang = pos.double()[:, axis.long()] * freq.double()
    c, s = ang.cos()[:, None], ang.sin()[:, None]

    def turn(x, w):
        y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w
        a, b = y.chunk(2, -1)
        return torch.cat([a * c - b * s, a * s + b * c], -1)

    q, k, v = turn(qkv[:, :Hq], wq), turn(qkv[:, Hq:Hq + Hkv], wk), qkv[:, Hq + Hkv:]
    out, at = [], 0
    for n in lens:
        rows = []
        for h in range(Hq):
            j = h * Hkv // Hq
            x = q[at:at + n, h] @ k[at:at + n, j].T / math.sqrt(q.shape[2])
            if causal:
                x = x.masked_fill(torch.ones(n, n).triu(1).bool(), -math.inf)
            rows.append(torch.softmax(x, 1) @ v[at:at + n, j])
        out.append(torch.stack(rows, 1))
        at += n
    return torch.cat(out)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dt,tol", [("f32", 1e-5), ("bf16", 2e-2)])
def test_pixel_attention_gradients(dt, tol, causal):
    """bf16: rotated heads, probabilities and results are each rounded to 2^-9
    of themselves, and a gradient passes through four of them."""
    torch_mod()
    g = torch.Generator().manual_seed(3)
    lens, heads, D = [40, 1, 77], (6, 2), 32
    T = sum(lens)
    dtype = torch.float32 if dt == "f32" else torch.bfloat16
    mk = lambda *s, m=0.0, k=1.0: (torch.randn(s, generator=g) * k + m).to(dtype)
    qkv, wq, wk, gy = mk(T, 10, D), mk(D, m=1.0, k=0.2), mk(D, m=1.0, k=0.2), mk(T, 6, D)
    pos = torch.rand((T, 3), generator=g) * 30
    freq, axis = hnn.hex_frequencies(D)
    ins = [t.double().requires_grad_(True) for t in (qkv, wq, wk)]
    want = layer64(*ins, pos, freq, axis, lens, heads, causal)
    grads = torch.autograd.grad(want, ins, gy.double())
    dev = [t.cuda().requires_grad_(True) for t in (qkv, wq, wk)]
    start = torch.tensor([0, 40, 41, T], dtype=torch.int32, device="cuda")
    rest = (pos.cuda(), freq.cuda(), axis.cuda())
    o = hnn.HexPixelAttentionFunction.apply(*dev, *rest, start, heads, 1e-6, causal)
    got = torch.autograd.grad(o, dev, gy.cuda())
    assert rel(o, want.detach()) <= tol
    for a, b in zip(got, grads):
        assert rel(a, b) <= tol
    # the same from the separate functions
    q, k, v = dev[0][:, :6], dev[0][:, 6:8], dev[0][:, 8:]
    qo, ko = hnn.hex_rotary(q, k, *rest, dev[1], dev[2])
    o2 = hnn.hex_attention(qo, ko, v, start, causal=causal)
    assert torch.equal(o2, o)
    for a, b in zip(torch.autograd.grad(o2, dev, gy.cuda()), got):
        assert torch.equal(a, b)


def test_attention_function_leaves_unused_tokens():
    """Tokens after the last sequence give zeros and take no gradient."""
    torch_mod()
    g = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn((30, 2, 16), generator=g).cuda().requires_grad_(True) for _ in range(3))
    start = torch.tensor([0, 20], dtype=torch.int32, device="cuda")
    o = hnn.hex_attention(q, k, v, start)
    assert not bool(o[20:].any())
    for d in torch.autograd.grad(o.sum(), (q, k, v)):
        assert not bool(d[20:].any()) and bool(torch.isfinite(d).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dropout_function(dtype):
    torch_mod()
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator().manual_seed(8)
    x, r, gy = (torch.randn((37, 21), generator=g).to(dt).cuda() for _ in range(3))
    x.requires_grad_(True), r.requires_grad_(True)
    rng = torch.tensor([99, 4], dtype=torch.int64, device="cuda")
    y = hnn.hex_dropout(x, 0.4, rng, residual=r, call=2)
    dx, dr = torch.autograd.grad(y, (x, r), gy)
    kept = torch.from_numpy(ref.philox(37 * 21, 99, 6) >= math.floor(0.4 * 2 ** 32)).view(37, 21)
    want = torch.where(kept, gy.double().cpu() / 0.6, torch.zeros((), dtype=torch.float64))
    lim = want.abs() * (2.0 ** -22 if dtype == "f32" else 2.0 ** -8)
    assert bool(((dx.double().cpu() - want).abs() <= lim).all())
    assert torch.equal(dr, gy)
    # another call, another mask; the same call, the same one
    other = hnn.hex_dropout(x, 0.4, rng, residual=r, call=3)
    assert not torch.equal(other, y)
    assert torch.equal(hnn.hex_dropout(x, 0.4, rng, residual=r, call=2), y)


def test_layer_draws_new_masks():
    torch_mod()
    torch.manual_seed(0)
    layer = hnn.HexPixelAttention(32, 2, dropout=0.5, device="cuda")
    x = torch.randn(50, 32, device="cuda")
    pos = torch.rand(50, 3, device="cuda")
    start = torch.tensor([0, 50], dtype=torch.int32, device="cuda")
    a, b = layer(x, pos, start), layer(x, pos, start)
    assert not torch.equal(a, b)
    layer.eval()
    assert torch.equal(layer(x, pos, start), layer(x, pos, start))


@pytest.mark.parametrize("dt,lim", [("f32", 1e-5), ("bf16", 0.06)])
def test_example_stream(dt, lim):
    """bf16: values of size up to 4, rounded at five places on either way."""
    torch_mod()
    import pixel_events
    dtype = torch.float32 if dt == "f32" else torch.bfloat16
    assert pixel_events.stream_error(dtype=dtype) <= lim


def test_example_trains():
    torch_mod()
    import pixel_events
    assert pixel_events.train() >= 0.9


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_layer_with_unused_tokens(dt):
    """Tokens after the last sequence pass through the layer as they are, and
    change no gradient: the same layer on the others alone has the same bits."""
    torch_mod()
    torch.manual_seed(3)
    layer = hnn.HexPixelAttention(64, 4, 2, 16, device="cuda", dtype=dt)
    start = torch.tensor([0, 30, 64], dtype=torch.int32, device="cuda")
    x0 = torch.randn(128, 64, device="cuda").to(dt)
    pos = torch.rand(128, 3, device="cuda") * 9
    filler = torch.full((1 << 22,), float("nan"), device="cuda")  # what fresh memory may hold
    del filler
    got = []
    for n in (128, 64):
        x = x0[:n].clone().requires_grad_()
        layer.zero_grad()
        y = layer(x, pos[:n].contiguous(), start)
        (y[:64].float() ** 2).sum().backward()
        got.append([y[:64], x.grad[:64]] + [p.grad.clone() for p in layer.parameters()])
        if n > 64:
            assert torch.equal(y[64:], x0[64:])
            assert not x.grad[64:].any()
    for a, b in zip(*got):
        assert torch.isfinite(a).all()
        err, size = (a - b).abs().max(), b.abs().max()
        assert err <= (1e-5 if dt == torch.float32 else 2e-2) * size


def test_prefill_cuts_at_capacity():
    """A prompt longer than its stream's room does not reach the next one's."""
    torch_mod()
    torch.manual_seed(4)
    layer = hnn.HexPixelAttention(32, 2, 1, 16, causal=True, device="cuda").eval()
    cache = layer.new_cache(3, 8)
    cache.k.zero_()
    cache.v.zero_()
    start = torch.tensor([0, 11, 13, 15], dtype=torch.int32, device="cuda")
    x, pos = torch.randn(15, 32, device="cuda"), torch.rand(15, 3, device="cuda")
    layer.prefill(x, pos, start, cache, 8)  # the first has 11
    assert cache.length.tolist() == [8, 2, 2]
    alone = layer.new_cache(2, 8)
    alone.k.zero_()
    alone.v.zero_()
    layer.prefill(x[11:].contiguous(), pos[11:].contiguous(), start[1:] - 11, alone, 2)
    used = lambda t: t.view(-1, 8, 16)[:, :2]  # noqa: E731
    assert torch.allclose(used(cache.k)[1:], used(alone.k), atol=1e-5)
    assert torch.allclose(used(cache.v)[1:], used(alone.v), atol=1e-5)
    assert not cache.k.view(3, 8, 16)[1:, 2:].any()


def test_cache_refuses_overflow():
    cache = hnn.HexCache(2, 5, 1, 8)
    cache.reserve(3)
    with pytest.raises(ValueError, match="capacity"):
        cache.reserve(3)
