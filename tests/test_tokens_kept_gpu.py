"""How gated blocks in bfloat16 keep g and u for their backward: eight neighbours as
float16 where all of them have its exponents, as bfloat16 else; the last bit of the
first says which (1: float16)."""
import pytest

from gpu_helpers import torch_mod
from paper_1903_01814_amd import hexconv as hx

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def kept(gu):
    """(values, whether float16) of [..][8 n] in groups of eight."""
    g = gu.reshape(-1, 8).contiguous()
    half = (g.view(torch.int16)[:, :1] & 1).bool()
    return torch.where(half, g.view(torch.float16).double(), g.double()), half[:, 0]


# few tokens, and tiles
@pytest.mark.parametrize("T", [7, 90])
@pytest.mark.parametrize("scale", [1.0, 2.0 ** -12, 2.0 ** 11, 2.0 ** 14])
def test_kept_values(T, scale):
    """Half a step of 11 bits, for the first of eight a step of them (10 bits); of 8
    bits, for the first half a step of 7.  g and u are sums of three products, off by 3
    roundings of float32 of their magnitudes."""
    torch_mod()
    F, K = 512, 3
    g = torch.Generator(device="cuda").manual_seed(T)
    x = (torch.randn(T, K, generator=g, device="cuda") * scale).bfloat16()
    w1 = torch.randn(2 * F, K, generator=g, device="cuda").bfloat16()
    w2 = torch.randn(K, F, generator=g, device="cuda").bfloat16()
    Fp = hx.hexffn_width(F)
    y, gu, h = (torch.empty(T, n, dtype=torch.bfloat16, device="cuda") for n in (K, 2 * Fp, Fp))
    nb = hx.hexffn_fwd_workspace(T, K, F, K, K, 1)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda") if nb else None
    hx.hexffn_fwd(x, w1, None, w2, None, None, y, gu, h, ws)
    want = x.double().cpu() @ w1.double().cpu().t()
    size = (x.double().cpu().abs() @ w1.double().cpu().abs().t()).reshape(-1, 8)
    assert Fp == F
    got, half = kept(gu.cpu())
    want = want.reshape(-1, 8)
    least, most = want.abs().min(1).values, want.abs().max(1).values
    inside, outside = (least > 2.0 ** -13.9) & (most < 2.0 ** 14.9), (least < 2.0 ** -14.1) | (
        most > 2.0 ** 15.1)
    assert bool(half[inside].all()) and not bool(half[outside].any())
    # (deviations of 1.7 times the scale)
    assert int((inside if 2.0 ** -12 < scale < 2.0 ** 14 else outside).sum()) > 100
    step = torch.full((1, 8), 2.0 ** -11)
    step[0, 0] = 2.0 ** -10
    step = torch.where(half[:, None], step, 8 * step)
    off = (got - want).abs() / (step * want.abs() + 3 * 2.0 ** -24 * size)
    assert float(off[half].max() if bool(half.any()) else 0) <= 1.001
    assert float(off[~half].max() if bool((~half).any()) else 0) <= 1.001
