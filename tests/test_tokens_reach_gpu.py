"""Projections and gated blocks, forward and backward, at the sizes that meet every
kernel of the matrix product with every epilogue (tokens_sizes.py): biases, residuals,
activations, kept values, every gradient, in float32 from bfloat16 operands too.

Every element is held to tokens_ref's bound of the worst case, and every 64 x 64 part
of a result to a norm of independent roundings, which a lost step of the contraction
passes by far.  bfloat16: a rounding is 1.7e-3 of a norm, a result with gradients has up
to two and what z's or g's and u's rounding does to the derivative, 2.6e-3 together;
3.5e-3 leaves parts of 512 elements their spread.  float32: a sum of n products, rounded
every eight or more, is off by 2^-24 sqrt(n) / 4 of its norm, operands and epilogue by a
few 2^-24."""
import pytest

import tokens_ref as ref
import tokens_sizes as sizes
from gpu_helpers import torch_mod, tdtype
from paper_1903_01814_amd import hexconv as hx

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ACTS = {"silu": hx.HEX_ACT_SILU, "gelu": hx.HEX_ACT_GELU, "none": hx.HEX_ACT_NONE}
CYCLE = ["silu", "gelu", "none"]


def cases(bf16, f32):
    """(size, type, activation, type of the weights' gradients): all activations and both
    types in turn."""
    out = []
    for dt, listed in (("bf16", bf16), ("f32", f32)):
        for i, s in enumerate(listed):
            out.append((s, dt, CYCLE[i % 3], "f32" if i % 2 else dt))
    return out


def part_norms(t):
    """Norms of the 64 x 64 parts of a matrix, and their numbers of elements."""
    pad = lambda v: torch.nn.functional.pad(  # noqa: E731
        v, (0, -v.shape[1] % 64, 0, -v.shape[0] % 64))
    fold = lambda v: v.view(v.shape[0] // 64, 64, v.shape[1] // 64, 64).sum((1, 3))  # noqa: E731
    return fold(pad(t * t)).sqrt(), fold(pad(torch.ones_like(t)))


def near(got, want, n, dt, what):
    value, bound = want
    assert got.shape == value.shape, what
    err = got.double() - value
    bad = ~(err.abs() <= bound)  # a NaN is bad
    assert not bool(bad.any()), "%s: %d of %d off, worst %.3g of its bound" % (
        what, int(bad.sum()), got.numel(), float((err.abs() / bound).nan_to_num(9e9).max()))
    if got.dim() < 2:
        return
    lim = 3.5e-3 if dt == "bf16" else 1e-6 + 2.0 ** -26 * n ** 0.5
    size, count = part_norms(value)
    rel = (part_norms(err)[0] / size)[count >= 512]
    assert rel.numel() == 0 or float(rel.max()) <= lim, "%s: %.3g of a part's norm" % (
        what, float(rel.max()))


def maker(seed, dt):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s, k=1.0: (torch.randn(s, generator=g, device="cuda") * k).to(tdtype(dt))


def nan(*shape, dt):
    return torch.full(shape, float("nan"), dtype=tdtype(dt), device="cuda")


def space(nbytes):
    """A workspace of just that size that holds NaN, as fresh memory may."""
    if not nbytes:
        return None
    return torch.full(((nbytes + 3) // 4,), float("nan"), device="cuda").view(torch.uint8)[:nbytes]


@pytest.mark.parametrize("size,dt,act,gt", cases(sizes.LINEAR_BF16, sizes.LINEAR_F32))
def test_linear(size, dt, act, gt):
    torch_mod()
    T, N, K = size
    mk = maker(T + N + K, dt)
    x, w, b, r, dy = mk(T, K), mk(N, K, k=K ** -0.5), mk(N, k=0.3), mk(T, N), mk(T, N)
    want = ref.linear(x.double(), w.double(), b.double(), r.double(), act, dt, dy.double(), gt)
    got = {"y": nan(T, N, dt=dt), "z": nan(T, N, dt=dt), "dx": nan(T, K, dt=dt),
           "dw": nan(N, K, dt=gt), "db": nan(N, dt=gt)}
    code = hx._dtype_code(x)
    hx.hexlinear_fwd(x, w, b, r, got["y"], got["z"],
                     space(hx.hexlinear_fwd_workspace(T, N, K, K, code)), act=ACTS[act])
    hx.hexlinear_bwd(x, w, got["z"], dy, got["dx"], got["dw"], got["db"],
                     space(hx.hexlinear_bwd_workspace(T, N, K, K, N, ACTS[act], code)),
                     act=ACTS[act])
    torch.cuda.synchronize()
    terms = {"y": K, "z": K, "dx": N, "dw": T, "db": T}
    for name in got:
        near(got[name], want[name], terms[name], dt, name)


@pytest.mark.parametrize("size,dt,act,gt", cases(sizes.FFN_BF16, sizes.FFN_F32))
def test_ffn(size, dt, act, gt):
    torch_mod()
    T, K, F, N = size
    mk = maker(T + K + F + N, dt)
    x, w1, b1 = mk(T, K), mk(2 * F, K, k=K ** -0.5), mk(2 * F, k=0.3)
    w2, b2, r, dy = mk(N, F, k=F ** -0.5), mk(N, k=0.3), mk(T, N), mk(T, N)
    want = ref.ffn(x.double(), w1.double(), b1.double(), w2.double(), b2.double(), r.double(), act,
                   dt, dy.double(), gt)
    code, Fp = hx._dtype_code(x), hx.hexffn_width(F)
    y, gu, h = nan(T, N, dt=dt), nan(T, 2 * Fp, dt=dt), nan(T, Fp, dt=dt)
    hx.hexffn_fwd(x, w1, b1, w2, b2, r, y, gu, h,
                  space(hx.hexffn_fwd_workspace(T, K, F, N, K, code)), act=ACTS[act])
    got = {"dx": nan(T, K, dt=dt), "dw1": nan(2 * F, K, dt=gt), "db1": nan(2 * F, dt=gt),
           "dw2": nan(N, F, dt=gt), "db2": nan(N, dt=gt)}
    hx.hexffn_bwd(x, w1, w2, gu, h, dy, *got.values(),
                  space(hx.hexffn_bwd_workspace(T, K, F, N, K, N, code)), act=ACTS[act])
    torch.cuda.synchronize()
    assert not h[:, F:].any() and not gu[:, F:Fp].any() and not gu[:, Fp + F:].any()
    got["y"] = y
    terms = {"y": F + K, "dx": 2 * F + N, "dw1": T + N, "db1": T, "dw2": T + K, "db2": T}
    for name in got:
        near(got[name], want[name], terms[name], dt, name)
