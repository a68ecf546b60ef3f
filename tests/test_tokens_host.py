"""Refusals of the token-wise entry points, on the host: bad sizes, strides,
types and pointers are rejected before anything is enqueued (fake addresses are
never touched), empty calls return without work."""
import pytest

import tokens_ref as ref
from paper_1903_01814_amd import hexconv as hx

torch = pytest.importorskip("torch")

P = [0x10000 * i for i in range(1, 20)]
BAD, UNS, OK = hx.HEX_ERR_INVALID_ARG, hx.HEX_ERR_UNSUPPORTED, hx.HEX_OK
BIG = 1 << 40


def norm(x=P[0], w=P[1], b=P[2], y=P[3], mean=P[4], rstd=P[5], T=5, C=48, ldx=48, ldy=48, eps=1e-5,
         dt=0):
    return hx.load().hexnorm_fwd(x, w, b, y, mean, rstd, T, C, ldx, ldy, eps, dt, None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), BAD), (dict(C=0), BAD), (dict(C=16385, ldx=20000, ldy=20000), UNS),
    (dict(dt=2), BAD), (dict(eps=-1.0), BAD), (dict(eps=float("nan")), BAD), (dict(ldx=47), BAD),
    (dict(ldy=47), BAD), (dict(ldx=1 << 22), UNS), (dict(x=None), BAD), (dict(y=None), BAD),
    (dict(x=P[0] + 4), BAD), (dict(w=P[1] + 8), BAD), (dict(b=P[2] + 2), BAD),
    (dict(mean=None), BAD), (dict(rstd=None), BAD), (dict(mean=P[4] + 2), BAD),
    (dict(rstd=P[5] + 1), BAD), (dict(T=(1 << 31) - 1), UNS),
    (dict(T=1 << 24, C=2048, ldx=2048, ldy=2048), UNS)])
def test_norm_refuses(kw, status):
    assert norm(**kw) == status


def norm_bwd(x=P[0], w=P[1], mean=P[2], rstd=P[3], dy=P[4], res=P[5], dx=P[6], dw=P[7], db=P[8],
             ws=P[9], nb=BIG, T=5, C=48, ldx=48, ldg=48, ldr=48, ldd=48, dt=0):
    return hx.load().hexnorm_bwd(x, w, mean, rstd, dy, res, dx, dw, db, ws, nb, T, C, ldx, ldg, ldr,
                                 ldd, dt, None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), BAD), (dict(mean=None), BAD), (dict(rstd=None), BAD), (dict(dy=None), BAD),
    (dict(dx=None), BAD), (dict(ws=None), BAD), (dict(nb=2 * 48 * 4 - 1), BAD), (dict(ldr=47), BAD),
    (dict(ldd=40), BAD), (dict(ldg=1), BAD), (dict(dw=P[7] + 4), BAD), (dict(res=P[5] + 4), BAD),
    (dict(mean=P[2] + 2), BAD), (dict(C=20000, ldx=20000, ldg=20000, ldd=20000), UNS)])
def test_norm_backward_refuses(kw, status):
    assert hx.hexnorm_bwd_workspace(5, 48, 0) >= 2 * 48 * 4
    assert norm_bwd(**kw) == status


def lin(x=P[0], w=P[1], b=P[2], res=P[3], y=P[4], z=P[5], ws=P[6], nb=BIG, M=90, N=48, K=72, ldx=72,
        ldr=48, ldy=48, act=0, dt=0):
    return hx.load().hexlinear_fwd(x, w, b, res, y, z, ws, nb, M, N, K, ldx, ldr, ldy, act, dt, None)


SIZES = [(dict(M=-1), BAD), (dict(N=0), BAD), (dict(K=0), BAD), (dict(dt=2), BAD),
         (dict(act=4), BAD), (dict(act=-1), BAD), (dict(ldx=71), BAD), (dict(ldx=1 << 22), UNS),
         (dict(N=(1 << 20) + 1, ldr=1 << 21, ldy=1 << 21), UNS),
         (dict(K=(1 << 20) + 1, ldx=1 << 21), UNS), (dict(M=(1 << 31) - 1), UNS),
         (dict(M=1 << 27), UNS), (dict(x=P[0] + 8), BAD), (dict(w=P[1] + 4), BAD)]


@pytest.mark.parametrize("kw,status", SIZES + [
    (dict(x=None), BAD), (dict(w=None), BAD), (dict(y=None), BAD), (dict(ws=None), BAD),
    (dict(nb=100), BAD), (dict(ldy=47), BAD), (dict(ldr=47), BAD), (dict(b=P[2] + 4), BAD),
    (dict(z=P[5] + 2), BAD), (dict(ws=P[6] + 4), BAD)])
def test_linear_refuses(kw, status):
    assert hx.hexlinear_fwd_workspace(90, 48, 72, 72, 0) > 100
    assert lin(**kw) == status


def lin_bwd(x=P[0], w=P[1], z=P[2], dy=P[3], dx=P[4], dw=P[5], db=P[6], ws=P[7], nb=BIG, M=90, N=48,
            K=72, ldx=72, ldg=48, ldd=72, act=2, dwt=0, dt=0):
    return hx.load().hexlinear_bwd(x, w, z, dy, dx, dw, db, ws, nb, M, N, K, ldx, ldg, ldd, act, dwt,
                                   dt, None)


@pytest.mark.parametrize("kw,status", SIZES[:8] + SIZES[11:] + [
    (dict(z=None), BAD), (dict(dy=None), BAD), (dict(w=None), BAD), (dict(x=None), BAD),
    (dict(ws=None), BAD), (dict(nb=1000), BAD), (dict(ldg=47), BAD), (dict(ldd=71), BAD),
    (dict(dwt=1), BAD), (dict(dwt=2), BAD), (dict(dx=P[4] + 4), BAD), (dict(dw=P[5] + 4), BAD)])
def test_linear_backward_refuses(kw, status):
    assert hx.hexlinear_bwd_workspace(90, 48, 72, 72, 48, 2, 0) > 1000
    assert lin_bwd(**kw) == status


def ffn(x=P[0], w1=P[1], b1=P[2], w2=P[3], b2=P[4], res=P[5], y=P[6], gu=P[7], h=P[8], ws=P[9],
        nb=BIG, M=90, K=72, F=40, N=48, ldx=72, ldr=48, ldy=48, act=3, dt=0):
    return hx.load().hexffn_fwd(x, w1, b1, w2, b2, res, y, gu, h, ws, nb, M, K, F, N, ldx, ldr, ldy,
                                act, dt, None)


def ffn_bwd(x=P[0], w1=P[1], w2=P[2], gu=P[3], h=P[4], dy=P[5], dx=P[6], dw1=P[7], db1=P[8],
            dw2=P[9], db2=P[10], ws=P[11], nb=BIG, M=90, K=72, F=40, N=48, ldx=72, ldg=48, ldd=72,
            act=3, dwt=0, dt=0):
    return hx.load().hexffn_bwd(x, w1, w2, gu, h, dy, dx, dw1, db1, dw2, db2, ws, nb, M, K, F, N, ldx,
                                ldg, ldd, act, dwt, dt, None)


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), BAD), (dict(K=0), BAD), (dict(F=0), BAD), (dict(N=0), BAD), (dict(dt=5), BAD),
    (dict(act=4), BAD), (dict(ldx=71), BAD), (dict(ldx=1 << 22), UNS), (dict(F=1 << 20), UNS),
    (dict(F=1 << 19, K=1 << 12, ldx=1 << 12), UNS), (dict(M=1 << 27), UNS), (dict(x=None), BAD),
    (dict(w1=None), BAD), (dict(w2=None), BAD), (dict(y=None), BAD), (dict(h=None), BAD),
    (dict(ws=None), BAD), (dict(nb=1000), BAD), (dict(gu=P[7] + 8), BAD), (dict(b1=P[2] + 4), BAD),
    (dict(ldy=40), BAD), (dict(ldr=40), BAD)])
def test_ffn_refuses(kw, status):
    assert hx.hexffn_fwd_workspace(90, 72, 40, 48, 72, 0) > 1000
    assert ffn(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), BAD), (dict(w1=None), BAD), (dict(w2=None), BAD), (dict(gu=None), BAD),
    (dict(h=None), BAD), (dict(dy=None), BAD), (dict(ws=None), BAD), (dict(nb=1000), BAD),
    (dict(ldg=47), BAD), (dict(ldd=71), BAD), (dict(dwt=1), BAD), (dict(dw1=P[7] + 4), BAD),
    (dict(F=0), BAD), (dict(M=-2), BAD)])
def test_ffn_backward_refuses(kw, status):
    assert hx.hexffn_bwd_workspace(90, 72, 40, 48, 72, 48, 0) > 1000
    assert ffn_bwd(**kw) == status


def test_empty_calls():
    assert norm(T=0, x=None, y=None) == OK
    assert lin(M=0, x=None, w=None, y=None, ws=None, nb=0) == OK
    assert ffn(M=0, x=None, w1=None, w2=None, y=None, h=None, ws=None, nb=0) == OK
    # no gradient wanted
    assert lin_bwd(dx=None, dw=None, db=None, dy=None, ws=None, nb=0) == OK
    assert ffn_bwd(dx=None, dw1=None, db1=None, dw2=None, db2=None, dy=None, ws=None, nb=0) == OK


def test_workspaces():
    assert hx.hexnorm_bwd_workspace(0, 48, 0) == 0 == hx.hexnorm_bwd_workspace(9, 0, 0)
    assert hx.hexlinear_fwd_workspace(9, 48, 0, 72, 0) == 0
    assert hx.hexlinear_fwd_workspace(9, 48, 72, 71, 0) == 0
    assert hx.hexlinear_bwd_workspace(9, 48, 72, 72, 48, 9, 0) == 0
    assert hx.hexffn_fwd_workspace(9, 72, -1, 48, 72, 0) == 0
    assert hx.hexffn_bwd_workspace(0, 72, 40, 48, 72, 48, 0) == 0
    assert hx.hexffn_width(41) == 48 and hx.hexffn_width(48) == 48
    with pytest.raises(hx.HexError):
        hx.hexffn_width(0)


@pytest.mark.parametrize("n", [1 << 20, 1 << 30, (1 << 31) - 1])
def test_workspaces_of_the_largest_arguments(n):
    """Products past 32 bits neither wrap to a size nor end the process."""
    for dt in (0, 1):
        assert hx.hexlinear_fwd_workspace(n, n, n, n, dt) == 0
        assert hx.hexlinear_bwd_workspace(n, 1 << 20, 1 << 20, 1 << 20, 1 << 20, 1, dt) == 0
        hx.hexlinear_fwd_workspace(n, 8, 8, 8, dt)
        hx.hexlinear_bwd_workspace(n, 8, 8, 8, 8, 1, dt)
        hx.hexlinear_fwd_workspace(8, 1 << 13, 1 << 20, 1 << 20, dt)
        hx.hexffn_bwd_workspace(8, 1 << 13, 1 << 17, 1 << 13, 1 << 13, 1 << 13, dt)
        assert hx.hexffn_fwd_workspace(n, n, n, n, n, dt) == 0
        hx.hexnorm_bwd_workspace(n, 16384, dt)


def test_binding_refuses():
    """Host tensors, wrong types, rows that are not dense, mixed gradients."""
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="device tensor"):
        hx.hexnorm_fwd(x, None, None, x)
    with pytest.raises(ValueError, match="device tensor"):
        hx.hexlinear_fwd(x, x, None, None, x)
    with pytest.raises(TypeError, match="unsupported dtype"):
        hx.hexlinear_fwd(x.double(), x, None, None, x)
    with pytest.raises(TypeError, match="gradients of weights"):
        hx.hexlinear_bwd(x, x, None, x, None, x.bfloat16(), None, None)
    with pytest.raises(TypeError, match="gradients of weights"):
        hx.hexffn_bwd(x, x, x, x, x, x, None, x, None, x.bfloat16(), None, None)


def test_reference():
    """The float64 forms against autograd's gradients and differences."""
    g = torch.Generator().manual_seed(0)
    mk = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    x, w1, b1, w2, b2, res, dy = mk(5, 6), mk(14, 6), mk(14), mk(4, 7), mk(4), mk(5, 4), mk(5, 4)
    for name in ("none", "gelu", "silu"):
        ins = [t.clone().requires_grad_(True) for t in (x, w1, b1, w2, b2)]
        z = ins[0] @ ins[1].T + ins[2]
        f = {"none": lambda t: t, "gelu": torch.nn.functional.gelu,
             "silu": torch.nn.functional.silu}[name]
        y = (f(z[:, :7]) * z[:, 7:]) @ ins[3].T + ins[4] + res
        want = torch.autograd.grad(y, ins, dy)
        got = ref.ffn(x, w1, b1, w2, b2, res, name, "f32", dy)
        for n, t in zip(("dx", "dw1", "db1", "dw2", "db2"), want):
            assert torch.allclose(got[n][0], t, atol=1e-12), n
        lin = ref.linear(x, w2.new_ones(4, 6), b2, res, name, "f32", dy)
        step = 1e-6 * mk(5, 6)
        up = ref.linear(x + step, w2.new_ones(4, 6), b2, res, name, "f32")["y"][0]
        down = ref.linear(x - step, w2.new_ones(4, 6), b2, res, name, "f32")["y"][0]
        assert abs(float(((up - down) / 2 * dy).sum() - (lin["dx"][0] * step).sum())) < 1e-13
    ins = [x.clone().requires_grad_(True), mk(6).requires_grad_(True), mk(6).requires_grad_(True)]
    y = torch.nn.functional.layer_norm(ins[0], (6,), ins[1], ins[2], 1e-3)
    gy, add = mk(5, 6), mk(5, 6)
    want = torch.autograd.grad(y, ins, gy)
    got = ref.norm(x, ins[1].detach(), ins[2].detach(), 1e-3, "f32", gy, add)
    assert torch.allclose(got["y"][0], y.detach()) and torch.allclose(got["dx"][0], want[0] + add)
    assert torch.allclose(got["dw"][0], want[1]) and torch.allclose(got["db"][0], want[2])


def test_ffn_width_whole_lines():
    """Rows of h begin on cache lines past 256 columns."""
    assert [hx.hexffn_width(f) for f in (1, 8, 250, 256, 257, 320, 683)] == [8, 8, 256, 256, 320,
                                                                             320, 704]
