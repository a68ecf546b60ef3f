"""relu in projections and gated blocks against float64, forward and backward.  A value
that a float32 sum could turn either way about 0, |z| within its error bound, may have
either derivative: its gradient's bound is as large as that makes it."""
import pytest

import tokens_ref as ref
from gpu_helpers import torch_mod, tdtype
from paper_1903_01814_amd import hexconv as hx

torch = pytest.importorskip("torch")
hnn = pytest.importorskip("paper_1903_01814_amd.nn")
pytestmark = pytest.mark.gpu

RELU = hx.HEX_ACT_RELU


def either_way(z, ez, grad):
    """What a derivative of the other side adds to a gradient's error."""
    return grad.abs() * (z.abs() <= ez)


def linear_bounds(x, w, b, r, dy, dt):
    want = ref.linear(x, w, b, r, "relu", dt, dy)
    z = x @ w.T + b
    more = either_way(z, ref.acc(x.shape[1]) * (x.abs() @ w.abs().T + b.abs()), dy)
    for name, add in (("dx", more @ w.abs()), ("dw", more.T @ x.abs()), ("db", more.sum(0))):
        want[name] = (want[name][0], want[name][1] + add)
    return want


def ffn_bounds(x, w1, b1, w2, b2, r, dy, dt):
    want = ref.ffn(x, w1, b1, w2, b2, r, "relu", dt, dy)
    F = w2.shape[1]
    z = x @ w1.T + b1
    ez = ref.acc(x.shape[1]) * (x.abs() @ w1.abs().T + b1.abs())
    dg = either_way(z[:, :F], ez[:, :F], (dy @ w2) * z[:, F:])
    more = torch.cat([dg, torch.zeros_like(dg)], 1)
    for name, add in (("dx", more @ w1.abs()), ("dw1", more.T @ x.abs()), ("db1", more.sum(0))):
        want[name] = (want[name][0], want[name][1] + add)
    return want


def near(got, want):
    for name, t in got.items():
        value, bound = want[name]
        err = (t.double().cpu() - value).abs()
        assert bool((err <= bound).all()), "%s: worst %.3g of its bound" % (
            name, float((err / bound.clamp_min(1e-300)).nan_to_num(9e9).max()))


def maker(seed, dt):
    g = torch.Generator().manual_seed(seed)

    def mk(*s, k=1.0):
        t = (torch.randn(s, generator=g) * k).to(tdtype(dt))
        return t.double(), t.cuda()
    return mk


def nan(*shape, dt):
    return torch.full(shape, float("nan"), dtype=tdtype(dt), device="cuda")


def space(nbytes):
    return torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda") if nbytes else None


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,K", [(1, 24, 16), (19, 41, 63), (90, 48, 56), (700, 264, 520)])
def test_linear(T, N, K, dt):
    torch_mod()
    mk = maker(T, dt)
    ins = [mk(T, K), mk(N, K, k=K ** -0.5), mk(N, k=0.3), mk(T, N), mk(T, N)]
    want = linear_bounds(*(a for a, _ in ins), dt)
    x, w, b, r, dy = (a for _, a in ins)
    got = {"y": nan(T, N, dt=dt), "z": nan(T, N, dt=dt), "dx": nan(T, K, dt=dt),
           "dw": nan(N, K, dt=dt), "db": nan(N, dt=dt)}
    code = hx._dtype_code(x)
    hx.hexlinear_fwd(x, w, b, r, got["y"], got["z"],
                     space(hx.hexlinear_fwd_workspace(T, N, K, K, code)), act=RELU)
    hx.hexlinear_bwd(x, w, got["z"], dy, got["dx"], got["dw"], got["db"],
                     space(hx.hexlinear_bwd_workspace(T, N, K, K, N, RELU, code)), act=RELU)
    near(got, want)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,K,F,N", [(1, 16, 24, 16), (20, 41, 53, 33), (90, 48, 56, 48),
                                     (131, 200, 331, 200), (700, 264, 520, 264)])
def test_ffn(T, K, F, N, dt):
    torch_mod()
    mk = maker(T + F, dt)
    ins = [mk(T, K), mk(2 * F, K, k=K ** -0.5), mk(2 * F, k=0.3), mk(N, F, k=F ** -0.5),
           mk(N, k=0.3), mk(T, N), mk(T, N)]
    want = ffn_bounds(*(a for a, _ in ins), dt)
    x, w1, b1, w2, b2, r, dy = (a for _, a in ins)
    code, Fp = hx._dtype_code(x), hx.hexffn_width(F)
    y, gu, h = nan(T, N, dt=dt), nan(T, 2 * Fp, dt=dt), nan(T, Fp, dt=dt)
    hx.hexffn_fwd(x, w1, b1, w2, b2, r, y, gu, h,
                  space(hx.hexffn_fwd_workspace(T, K, F, N, K, code)), act=RELU)
    got = {"dx": nan(T, K, dt=dt), "dw1": nan(2 * F, K, dt=dt), "db1": nan(2 * F, dt=dt),
           "dw2": nan(N, F, dt=dt), "db2": nan(N, dt=dt)}
    hx.hexffn_bwd(x, w1, w2, gu, h, dy, *got.values(),
                  space(hx.hexffn_bwd_workspace(T, K, F, N, K, N, code)), act=RELU)
    near(dict(got, y=y), want)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T", [3, 80])
def test_gates_at_zero_and_below(T, dt):
    """Gates of exactly 0 and -0, and of values that bfloat16 keeps least of: relu'(0) is
    0, and the smallest positive gate passes its gradient."""
    torch_mod()
    F = 8
    gates = torch.tensor([0.0, -0.0, 2.0 ** -100, -2.0 ** -100, 2.0 ** -15, -2.0 ** -15, 1.0, -1.0])
    x = torch.ones(T, 1, dtype=tdtype(dt), device="cuda")
    w1 = torch.cat([gates, torch.ones(F)])[:, None].to(tdtype(dt)).cuda()
    for roll in range(8):  # each at the first place of the eight, too
        w = torch.cat([w1[:F].roll(roll, 0), w1[F:]])
        w2 = torch.eye(F, dtype=tdtype(dt), device="cuda")
        code = hx._dtype_code(x)
        y, gu, h = nan(T, F, dt=dt), nan(T, 2 * F, dt=dt), nan(T, F, dt=dt)
        hx.hexffn_fwd(x, w, None, w2, None, None, y, gu, h,
                      space(hx.hexffn_fwd_workspace(T, 1, F, F, 1, code)), act=RELU)
        dy, db1 = torch.ones(T, F, dtype=tdtype(dt), device="cuda"), nan(2 * F, dt="f32")
        hx.hexffn_bwd(x, w, w2, gu, h, dy, None, None, db1, None, None,
                      space(hx.hexffn_bwd_workspace(T, 1, F, F, 1, F, code)), act=RELU)
        want = gates.roll(roll)
        assert torch.equal(y.float().cpu(), want.clamp(min=0).expand(T, F))
        assert torch.equal(db1[:F].cpu(), (want > 0).float() * T)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_layer(dt):
    """The layers take relu: against torch's gradients of the same layer in float64."""
    torch_mod()
    torch.manual_seed(4)
    m = hnn.HexFeedForward(40, 56, "relu", bias=True, norm=False, device="cuda", dtype=tdtype(dt))
    x = torch.randn(70, 40, device="cuda").to(tdtype(dt)).requires_grad_(True)
    gy = torch.randn(70, 40, device="cuda").to(tdtype(dt))
    y = m(x)
    grads = torch.autograd.grad(y, [x, m.weight1, m.bias1, m.weight2, m.bias2], gy)
    c = lambda t: t.detach().double().cpu()  # noqa: E731
    want = ffn_bounds(c(x), c(m.weight1), c(m.bias1), c(m.weight2), c(m.bias2), c(x), c(gy), dt)
    # the residual's gradient is added to dx after its rounding, and the sum rounded again
    value, bound = want["dx"]
    value = value + c(gy)
    want["dx"] = (value, bound + ref.R[dt] * value.abs())
    got = dict(zip(("dx", "dw1", "db1", "dw2", "db2"), grads), y=y.detach())
    near(got, want)
