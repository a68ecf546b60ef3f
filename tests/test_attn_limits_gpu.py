"""Gradients with a workspace of exactly the size asked for: nothing behind it
is written, with partial sums and without."""
import pytest

import attn_ref as ref
from gpu_helpers import torch_mod
from paper_1903_01814_amd import hexconv as hx
from test_attn_gpu import TOL, ints, nan, near, normal

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,H,D", [
    (1300, 1600, 8),   # one share of a head: tiles of many rows, none divided
    (300, 40, 32),     # few rows: none divided
    (2600, 6, 64),     # divided
])
def test_gradient_keeps_to_its_workspace(T, H, D, dt):
    """The first, one middle and the last head against float64."""
    torch_mod()
    g = torch.Generator().manual_seed(T)
    start = [0, T // 13, T]
    q, k, v, do = (normal(g, T, H, D, dt=dt)[1] for _ in range(4))
    nb = hx.hexattn_bwd_workspace(T, T, 2, H, H, D, hx._dtype_code(q))
    ws = torch.full((nb + (1 << 20),), 99, dtype=torch.uint8, device="cuda")
    o, lse = nan(T, H, D, dt=dt), nan(T, H)
    grads = [nan(T, H, D, dt=dt) for _ in range(3)]
    hx.hexattn_fwd(q, k, v, o, lse, ints(start), causal=True)
    hx.hexattn_bwd(q, k, v, o, lse, do, *grads, ws[:nb], ints(start), causal=True)
    torch.cuda.synchronize()
    assert bool((ws[nb:] == 99).all())
    at = [0, H // 2, H - 1]
    spans = [(a, b - a, a, b - a) for a, b in zip(start, start[1:])]
    want = ref.attention(*(t[:, at].double().cpu() for t in (q, k, v)), spans, D ** -0.5, True,
                         do[:, at].double().cpu())
    near(o[:, at], want["o"], want["o_mag"], TOL[dt], "o")
    for t, n in zip(grads, ("dq", "dk", "dv")):
        near(t[:, at], want[n], want[n + "_mag"], TOL[dt], n)
