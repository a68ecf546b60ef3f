"""The token-wise operators at sizes past what 32 bits count."""
import pytest

from gpu_helpers import torch_mod
from paper_1903_01814_amd import hexconv as hx

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def ones(*shape):
    return torch.ones(shape, dtype=BF16, device="cuda")


def zeros_only(t):
    return not any(bool(part.any()) for part in t.view(-1).split(1 << 28))


def test_no_tokens_of_large_weights():
    """Gradients of 2^32 elements and more are zeros where there is no token, and what
    lies behind them stays."""
    torch_mod()
    x, dy = ones(0, 1 << 13), ones(0, (1 << 20) - 3)
    n = dy.shape[1] * x.shape[1]
    room, db = ones(n + 8), ones(dy.shape[1])
    hx.hexlinear_bwd(x, None, None, dy, None, room[:n].view(dy.shape[1], x.shape[1]), db, None)
    assert zeros_only(room[:n]) and zeros_only(db) and bool(room[n:].all())
    del room

    F, N = 1 << 19, (1 << 13) + 1
    x, dy, h = ones(0, 8), ones(0, N), ones(0, hx.hexffn_width(F))
    dw2 = ones(N, F)  # in w2's place too, of which only the shape is read
    hx.hexffn_bwd(x, None, dw2, None, h, dy, None, None, None, dw2, None, None)
    assert zeros_only(dw2)


@pytest.mark.parametrize("dt", [torch.float32, BF16])
@pytest.mark.parametrize("n", [1, 3, 4, 5, 8, 11, 2047, 2048, 2049])
def test_no_tokens_of_odd_weights(n, dt):
    """Every end of a gradient that no token reaches, and nothing behind it."""
    torch_mod()
    x, dy = (torch.empty(0, c, dtype=dt, device="cuda") for c in (1, n))
    room, db = (torch.ones(n + 16, dtype=dt, device="cuda") for _ in range(2))
    hx.hexlinear_bwd(x, None, None, dy, None, room[:n].view(n, 1), db[:n], None)
    for t in (room, db):
        assert not bool(t[:n].any()) and bool(t[n:].all())
