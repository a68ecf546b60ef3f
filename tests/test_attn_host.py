"""Refusals of the attention entry points, on the host: bad sizes, strides,
types and pointers are rejected before anything is enqueued (fake addresses
are never touched), empty calls return without work."""
import pytest

import attn_ref
from paper_1903_01814_amd import hexconv as hx

torch = pytest.importorskip("torch")

P = [0x10000 * i for i in range(1, 20)]
BAD, UNS, OK = hx.HEX_ERR_INVALID_ARG, hx.HEX_ERR_UNSUPPORTED, hx.HEX_OK


def fwd(q=P[0], k=P[1], v=P[2], o=P[3], lse=P[4], qs=P[5], ks=P[6], kl=None, S=2, Tq=9, Tk=9, Hq=4,
        Hkv=2, D=32, ldq=128, ldk=64, ldv=64, ldo=128, scale=1.0, flags=0, dt=0):
    return hx.load().hexattn_fwd(q, k, v, o, lse, qs, ks, kl, S, Tq, Tk, Hq, Hkv, D, ldq, ldk, ldv,
                                 ldo, scale, flags, dt, None)


def bwd(q=P[0], k=P[1], v=P[2], o=P[3], lse=P[4], do=P[5], dq=P[6], dk=P[7], dv=P[8], ws=P[9],
        nb=1 << 20, qs=P[10], ks=P[11], S=2, Tq=9, Tk=9, Hq=4, Hkv=2, D=32, ldq=128, ldk=64,
        ldv=64, ldo=128, lddo=128, lddq=128, lddk=64, lddv=64, scale=1.0, flags=0, dt=0):
    return hx.load().hexattn_bwd(q, k, v, o, lse, do, dq, dk, dv, ws, nb, qs, ks, S, Tq, Tk, Hq,
                                 Hkv, D, ldq, ldk, ldv, ldo, lddo, lddq, lddk, lddv, scale, flags,
                                 dt, None)


HEADS = [(dict(Hq=0), BAD), (dict(Hkv=0), BAD), (dict(Hq=3), BAD), (dict(D=0), BAD),
         (dict(D=20), UNS), (dict(D=136, Hq=1, Hkv=1, ldq=136, ldk=136, ldv=136, ldo=136), UNS),
         (dict(dt=2), BAD), (dict(S=-1), BAD), (dict(Tq=-1), BAD), (dict(Tk=-1), BAD),
         (dict(ldq=127), BAD), (dict(ldq=130), BAD), (dict(ldk=60), BAD), (dict(ldv=66), BAD),
         (dict(ldk=68, dt=1), BAD), (dict(ldo=100), BAD), (dict(scale=float("inf")), BAD),
         (dict(scale=float("nan")), BAD), (dict(scale=-1.0), BAD), (dict(flags=2), BAD),
         (dict(q=P[0] + 8), BAD),
         (dict(k=P[1] + 4), BAD), (dict(v=None), BAD), (dict(qs=None), BAD), (dict(ks=None), BAD),
         (dict(Tq=1 << 30), UNS), (dict(S=1 << 30), UNS)]


@pytest.mark.parametrize("kw,status", HEADS + [(dict(o=None), BAD), (dict(q=None), BAD),
                                               (dict(lse=P[4] + 4), BAD)])
def test_forward_refuses(kw, status):
    assert fwd(**kw) == status


@pytest.mark.parametrize("kw,status", HEADS + [
    (dict(ws=None), BAD), (dict(nb=9 * 4 * 4 - 1), BAD), (dict(lse=None), BAD), (dict(do=None), BAD),
    (dict(dq=None), BAD), (dict(dk=None), BAD), (dict(dv=P[8] + 2), BAD), (dict(o=None), BAD),
    (dict(lddo=64), BAD), (dict(lddq=64), BAD), (dict(lddk=32), BAD), (dict(lddv=65), BAD)])
def test_backward_refuses(kw, status):
    assert bwd(**kw) == status


def test_empty_calls():
    assert fwd(S=0) == OK and fwd(Tq=0) == OK
    assert fwd(S=0, q=None, k=None, v=None, o=None, lse=None, qs=None, ks=None) == OK
    assert bwd(S=0) == OK
    assert bwd(Tq=0, Tk=0, q=None, k=None) == OK
    assert step(S=0, q=None, o=None) == OK
    assert hx.load().hexdropout(None, None, None, 0, 0.5, None, 0, 0, None) == OK
    assert rot(T=0, q=None, k=None) == OK


def step(q=P[0], k=P[1], v=P[2], o=P[3], ws=P[4], nb=1 << 40, ks=P[5], kl=P[6], S=2, n=1, Hq=4,
         Hkv=2, D=32, Tk=900, max_len=400, ldk=64, ldv=64, scale=1.0, dt=0):
    return hx.load().hexattn_step(q, k, v, o, ws, nb, ks, kl, S, n, Hq, Hkv, D, Tk, max_len, ldk,
                                  ldv, scale, dt, None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=0), BAD), (dict(S=-1), BAD), (dict(Tk=-1), BAD), (dict(max_len=-1), BAD),
    (dict(Hq=3), BAD), (dict(D=12), UNS), (dict(D=256, ldk=512, ldv=512), UNS), (dict(dt=7), BAD),
    (dict(ldk=62), BAD), (dict(ldv=32), BAD), (dict(ldk=68, dt=1), BAD), (dict(q=None), BAD),
    (dict(o=None), BAD), (dict(k=None), BAD), (dict(ks=None), BAD), (dict(kl=None), BAD),
    (dict(ws=None), BAD), (dict(nb=16), BAD), (dict(q=P[0] + 2), BAD), (dict(ws=P[4] + 4), BAD),
    (dict(scale=float("nan")), BAD), (dict(scale=-0.5), BAD), (dict(S=1 << 30), UNS),
    (dict(max_len=(1 << 30) + 1), UNS)])
def test_step_refuses(kw, status):
    # without a GPU the plan is made for 256 compute units, with one for its own
    assert hx.hexattn_step_workspace(2, 1, 4, 2, 32, 400, 0) > 16
    assert step(**kw) == status


def rot(q=P[0], k=P[1], v=None, pos=P[2], freq=P[3], axis=P[4], wq=P[5], wk=P[6], qo=P[7], ko=P[8],
        vo=None, slot=None, T=5, Hq=4, Hkv=2, D=32, A=3, ldq=128, ldk=64, ldv=64, ldqo=128, ldko=64,
        ldvo=64, n=5, eps=1e-6, flags=1, dt=0):
    return hx.load().hexrotary_fwd(q, k, v, pos, freq, axis, wq, wk, qo, ko, vo, slot, T, Hq, Hkv,
                                   D, A, ldq, ldk, ldv, ldqo, ldko, ldvo, n, eps, flags, dt, None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), BAD), (dict(A=0), BAD), (dict(A=9), UNS), (dict(eps=-1.0), BAD),
    (dict(eps=float("nan")), BAD), (dict(flags=2), BAD), (dict(v=P[9]), BAD), (dict(vo=P[9]), BAD),
    (dict(v=P[9], vo=P[10], ldv=60), BAD), (dict(v=P[9], vo=P[10], ldvo=32), BAD),
    (dict(n=-1), BAD), (dict(Hkv=3), BAD), (dict(D=44), UNS), (dict(ldq=64), BAD),
    (dict(ldk=66), BAD), (dict(ldqo=64), BAD), (dict(ldko=60), BAD), (dict(q=None), BAD),
    (dict(pos=None), BAD), (dict(freq=None), BAD), (dict(axis=None), BAD), (dict(qo=None), BAD),
    (dict(ko=P[8] + 4), BAD), (dict(wq=P[5] + 8), BAD), (dict(dt=-1), BAD)])
def test_rotary_refuses(kw, status):
    assert rot(**kw) == status


def rot_bwd(q=P[0], k=P[1], pos=P[2], freq=P[3], axis=P[4], wq=P[5], wk=P[6], gq=P[7], gk=P[8],
            dq=P[9], dk=P[10], dwq=P[11], dwk=P[12], ws=P[13], nb=1 << 20, T=5, Hq=4, Hkv=2, D=32,
            A=3, ldq=128, ldk=64, ldgq=128, ldgk=64, lddq=128, lddk=64, eps=1e-6, flags=1, dt=0):
    return hx.load().hexrotary_bwd(q, k, pos, freq, axis, wq, wk, gq, gk, dq, dk, dwq, dwk, ws, nb,
                                   T, Hq, Hkv, D, A, ldq, ldk, ldgq, ldgk, lddq, lddk, eps, flags,
                                   dt, None)


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), BAD), (dict(ws=None), BAD), (dict(nb=255), BAD), (dict(flags=0), BAD),
    (dict(gq=None), BAD), (dict(dk=None), BAD), (dict(dwq=P[11] + 4), BAD), (dict(lddq=64), BAD),
    (dict(ldgk=32), BAD), (dict(A=9), UNS), (dict(T=-2), BAD), (dict(D=4), UNS)])
def test_rotary_backward_refuses(kw, status):
    assert hx.hexrotary_bwd_workspace(5, 4, 2, 32, 0) == 256
    assert rot_bwd(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(p=1.0), BAD), (dict(p=-0.1), BAD), (dict(p=float("nan")), BAD), (dict(n=-1), BAD),
    (dict(x=None), BAD), (dict(y=None), BAD), (dict(rng=None), BAD), (dict(rng=P[3] + 4), BAD),
    (dict(res=P[1] + 4), BAD), (dict(dt=2), BAD), (dict(n=1 << 40), UNS)])
def test_dropout_refuses(kw, status):
    def f(x=P[0], res=P[1], y=P[2], n=64, p=0.1, rng=P[3], dt=0):
        return hx.load().hexdropout(x, res, y, n, p, rng, 0, dt, None)
    assert f(**kw) == status


def test_workspace_of_bad_arguments():
    assert hx.hexattn_bwd_workspace(9, 9, 2, 3, 2, 32, 0) == 0
    assert hx.hexattn_bwd_workspace(9, 9, 2, 4, 2, 32, 0) >= 9 * 4 * 4
    assert hx.hexattn_step_workspace(0, 1, 4, 2, 32, 100, 0) == 0
    assert hx.hexrotary_bwd_workspace(0, 4, 2, 32, 0) == 0


@pytest.mark.parametrize("n", [1 << 20, 1 << 30, (1 << 31) - 1])
@pytest.mark.parametrize("S,max_len", [(1, 100), (1 << 20, 100), (3, (1 << 31) - 1)])
def test_workspaces_of_the_largest_arguments(S, max_len, n):
    """Products past 32 bits neither wrap to a size nor end the process."""
    hx.hexattn_step_workspace(S, n, 4, 1, 64, max_len, 1)
    assert hx.hexattn_step_workspace(S, 1 << 30, 4, 1, 64, max_len, 1) == 0
    hx.hexattn_bwd_workspace(n, n, S, 4, 1, 64, 1)
    assert hx.hexattn_bwd_workspace(n, 1 << 30, S, 65535, 1, 128, 1) == 0
    assert hx.hexrotary_bwd_workspace(n, 65535, 65535, 128, 1) <= 1024 * 2 * 128 * 4


def test_binding_refuses():
    """Host tensors, wrong types and heads that are not dense."""
    q = torch.zeros(4, 2, 32)
    s = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor"):
        hx.hexattn_fwd(q, q, q, q, None, s)
    with pytest.raises(ValueError, match="device tensor"):
        hx.hexdropout(q, None, q, 0.5, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(TypeError, match="int64"):
        hx.hexdropout(q, None, q, 0.5, s)
    with pytest.raises(TypeError, match="unsupported dtype"):
        hx.hexattn_fwd(q.double(), q, q, q, None, s)
    with pytest.raises(ValueError, match="k_len needs k_start"):
        hx.hexattn_fwd(q, q, q, q, None, s, k_len=s)


def test_reference_rows_without_keys():
    """The float64 reference itself: a row that sees no key is zero, and a
    single key is returned as it is."""
    g = torch.Generator().manual_seed(0)
    q, k = torch.randn(5, 1, 8, generator=g).double(), torch.randn(3, 1, 8, generator=g).double()
    r = attn_ref.attention(q, k, k, [(0, 5, 0, 3)], 1.0, True, q)
    assert bool((r["o"][:2] == 0).all()) and bool((r["lse"][:2] == -float("inf")).all())
    assert torch.allclose(r["o"][2], k[0]) and not bool(r["dq"][:2].any())
