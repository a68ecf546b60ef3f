"""Limits that the attention entry points state, on the host: sizes of
workspaces, alignment of offsets."""
import pytest

from paper_1903_01814_amd import hexconv as hx

torch = pytest.importorskip("torch")


def plan_bytes(Tq, Tk, S, Hq):
    """What the gradient's workspace holds beside its partial sums: 4 bytes a
    row of Tq Hq, 4 a sequence, 48 for each key tile of 128 and each of up to
    3 * 1024 + 1 shares (three times), lines of 256 bytes."""
    return 4 * Tq * Hq + 4 * S + 48 * (Tk // 128 + S + 3 * 3073) + 2048


@pytest.mark.parametrize("D", [32, 64, 96, 128])
@pytest.mark.parametrize("dt", [hx.HEX_F32, hx.HEX_BF16])
@pytest.mark.parametrize("Hkv", [1, 4, 64, 511, 700, 767, 768, 1023, 1535, 2048, 4000, 20000])
@pytest.mark.parametrize("Tq,Tk,S", [(4096, 4096, 1), (100000, 100000, 24), (3, 100, 1),
                                     (1 << 16, 1 << 16, 60)])
def test_gradient_workspace_is_bounded(Tq, Tk, S, Hkv, D, dt):
    """Partial sums take up to 0.9 GB whatever the number of key heads, 0.45 GB
    up to 64 of them."""
    nb = hx.hexattn_bwd_workspace(Tq, Tk, S, Hkv, Hkv, D, dt)
    if max(Tq, Tk) * Hkv > (1 << 31) - 4096:
        assert nb == 0
        return
    assert 4 * Tq * Hkv <= nb <= (0.45e9 if Hkv <= 64 else 0.9e9) + plan_bytes(Tq, Tk, S, Hkv)


@pytest.mark.parametrize("G", [1, 4])
@pytest.mark.parametrize("D", [32, 128])
@pytest.mark.parametrize("dt", [hx.HEX_F32, hx.HEX_BF16])
@pytest.mark.parametrize("Tq,Tk,S,Hkv", [(9, 9, 2, 2), (150, 150, 30, 8), (100, 50000, 10, 4),
                                         (64, 1 << 20, 1, 16)])
def test_nothing_to_divide_needs_no_partial_sums(Tq, Tk, S, Hkv, D, dt, G):
    """Up to 19 tiles of 32 rows in all: every key tile is one piece."""
    assert Tq * G // 32 + 1 <= 20
    assert hx.hexattn_bwd_workspace(Tq, Tk, S, Hkv * G, Hkv, D, dt) <= plan_bytes(Tq, Tk, S,
                                                                                  Hkv * G)


P = [0x10000 * i for i in range(1, 14)]


@pytest.mark.parametrize("off", [1, 2, 3])
@pytest.mark.parametrize("which", ["q_start", "k_start", "k_len"])
def test_offsets_need_their_alignment(which, off):
    """4 bytes, as the rotation's arrays; fake addresses, refused before
    anything is enqueued."""
    at = {"q_start": P[10], "k_start": P[11], "k_len": P[12]}
    at[which] += off
    lib = hx.load()
    fwd = lib.hexattn_fwd(*P[:5], at["q_start"], at["k_start"], at["k_len"], 2, 9, 9, 4, 2, 32, 128,
                          64, 64, 128, 1.0, 0, 0, None)
    assert fwd == hx.HEX_ERR_INVALID_ARG
    if which != "k_len":
        bwd = lib.hexattn_bwd(*P[:10], 1 << 24, at["q_start"], at["k_start"], 2, 9, 9, 4, 2, 32,
                              128, 64, 64, 128, 128, 128, 64, 64, 1.0, 0, 0, None)
        assert bwd == hx.HEX_ERR_INVALID_ARG
    if which != "q_start":
        step = lib.hexattn_step(*P[:5], 1 << 30, at["k_start"], at["k_len"], 2, 1, 4, 2, 32, 900,
                                400, 64, 64, 1.0, 0, None)
        assert step == hx.HEX_ERR_INVALID_ARG


def test_no_tokens_into_a_cache():
    """No tokens, whose values have no address, and caches that do."""
    rc = hx.load().hexrotary_fwd(None, None, None, P[2], P[3], P[4], P[5], P[6], None, P[8], P[9],
                                 P[10], 0, 4, 2, 32, 3, 128, 64, 64, 128, 64, 64, 5, 1e-6, 1, 0,
                                 None)
    assert rc == hx.HEX_OK
