"""A token whose inputs or gradients are not finite reaches no other token's results,
through every kind of tile."""
import pytest

from gpu_helpers import torch_mod, tdtype
from paper_1903_01814_amd import hexconv as hx

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def space(nbytes):
    return torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda") if nbytes else None


def run(x, w, w1, w2, dy, dyk):
    """y, z and dx of a projection with silu, y and dx of a gated block, y and dx of a
    norm."""
    (T, K), N, F, code = x.shape, w.shape[0], w2.shape[1], hx._dtype_code(x)
    new = lambda n: torch.empty(T, n, dtype=x.dtype, device="cuda")  # noqa: E731
    y, z, dx = new(N), new(N), new(K)
    act = hx.HEX_ACT_SILU
    hx.hexlinear_fwd(x, w, None, None, y, z, space(hx.hexlinear_fwd_workspace(T, N, K, K, code)),
                     act=act)
    hx.hexlinear_bwd(x, w, z, dy, dx, None, None,
                     space(hx.hexlinear_bwd_workspace(T, N, K, K, N, act, code)), act=act)
    Fp = hx.hexffn_width(F)
    fy, gu, h, fdx = new(K), new(2 * Fp), new(Fp), new(K)
    hx.hexffn_fwd(x, w1, None, w2, None, None, fy, gu, h,
                  space(hx.hexffn_fwd_workspace(T, K, F, K, K, code)))
    hx.hexffn_bwd(x, w1, w2, gu, h, dyk, fdx, None, None, None, None,
                  space(hx.hexffn_bwd_workspace(T, K, F, K, K, K, code)))
    ny, ndx = new(K), new(K)
    mean, rstd = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    hx.hexnorm_fwd(x, None, None, ny, mean, rstd)
    hx.hexnorm_bwd(x, None, mean, rstd, dyk, None, ndx, None, None, None)
    return [y, z, dx, fy, fdx, ny, ndx]


@pytest.mark.parametrize("T,N,K,F", [(1, 24, 16, 24), (20, 40, 33, 41), (33, 72, 64, 72),
                                     (700, 264, 200, 331), (9000, 1040, 520, 1368),
                                     (8300, 1000, 1032, 1500)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_tokens_apart(T, N, K, F, dt):
    torch_mod()
    g = torch.Generator(device="cuda").manual_seed(T)
    mk = lambda *s, k=1.0: (torch.randn(s, generator=g, device="cuda") * k).to(tdtype(dt))  # noqa: E731
    x, w, w1, w2 = mk(T, K), mk(N, K, k=K ** -0.5), mk(2 * F, K, k=K ** -0.5), mk(K, F, k=F ** -0.5)
    dy, dyk = mk(T, N), mk(T, K)
    want = run(x, w, w1, w2, dy, dyk)
    assert all(bool(torch.isfinite(t).all()) for t in want)
    # one token's inputs, another's gradients, the last one's both
    hit = sorted({T // 2, T // 3, T - 1})
    x[T // 2, K // 2], x[T - 1, 0] = NAN, INF
    for t in (dy, dyk):
        t[T // 3, 0], t[T - 1, -1] = -INF, NAN
    got = run(x, w, w1, w2, dy, dyk)
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[hit] = False
    for i, (a, b) in enumerate(zip(got, want)):
        assert torch.equal(a[keep], b[keep]), i
        assert not bool(torch.isfinite(a[T - 1]).all()), i
