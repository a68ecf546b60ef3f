"""Packed attention where the first sequence starts past the first token, as
with a part start[a:b + 1] of a batch's offsets: results follow the float64
reference (tolerances as in test_attn_gpu.py), and outputs of tokens before the
first sequence and after the last stay as they were, whatever the inputs hold
there.  Which rows the blocks take is replayed on the CPU in
test_attn_span.py."""
import pytest

import attn_ref as ref
from gpu_helpers import tdtype, torch_mod
from paper_1903_01814_amd import hexconv as hx
from test_attn_gpu import TOL, ints, near, near_lse, normal

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("heads", [(2, 2, 32), (4, 1, 64), (6, 2, 128), (8, 1, 40)])
@pytest.mark.parametrize("qs,ks", [
    ([300, 600], None), ([128, 400], None), ([200, 200, 205, 300], None), ([1, 2], None),
    ([1500, 2000], None), ([513, 600], [40, 340]), ([0, 70], [257, 300]), ([640, 641], [0, 500])])
def test_late_first_sequence(qs, ks, heads, dt, causal):
    torch_mod()
    Hq, Hkv, D = heads
    g = torch.Generator().manual_seed(qs[0] + sum(heads))
    ko = qs if ks is None else ks
    Tq = qs[-1] + 70
    Tk = Tq if ks is None else ks[-1] + 35
    q64, q = normal(g, Tq, Hq, D, dt=dt)
    k64, k = normal(g, Tk, Hkv, D, dt=dt)
    v64, v = normal(g, Tk, Hkv, D, dt=dt)
    do64, do = normal(g, Tq, Hq, D, dt=dt)
    for t, s in ((q, qs), (do, qs), (k, ko), (v, ko)):
        t[:s[0]], t[s[-1]:] = float("nan"), float("nan")
    spans = [(qs[i], qs[i + 1] - qs[i], ko[i], ko[i + 1] - ko[i]) for i in range(len(qs) - 1)]
    want = ref.attention(q64, k64, v64, spans, D ** -0.5, causal, do64)
    sevens = lambda t: torch.full_like(t, 7.0)  # noqa: E731
    o, dq, dk, dv = sevens(q), sevens(q), sevens(k), sevens(v)
    lse = torch.full((Tq, Hq), 7.0, device="cuda")
    qd, kd = ints(qs), None if ks is None else ints(ks)
    ws = torch.empty(hx.hexattn_bwd_workspace(Tq, Tk, len(spans), Hq, Hkv, D, hx._dtype_code(q)),
                     dtype=torch.uint8, device="cuda")
    hx.hexattn_fwd(q, k, v, o, lse, qd, kd, causal=causal)
    hx.hexattn_bwd(q, k, v, o, lse, do, dq, dk, dv, ws, qd, kd, causal=causal)
    torch.cuda.synchronize()
    at = slice(qs[0], qs[-1])
    near_lse(lse[at], want["lse"][at], dt, "lse")
    for name, t, s in (("o", o, qs), ("lse", lse, qs), ("dq", dq, qs), ("dk", dk, ko),
                       ("dv", dv, ko)):
        at = slice(s[0], s[-1])
        if name != "lse":
            near(t[at], want[name][at], want[name + "_mag"][at], TOL[dt], name)
        assert bool((t[:s[0]] == 7).all()) and bool((t[s[-1]:] == 7).all()), name


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("G", [1, 4])
@pytest.mark.parametrize("cache", [False, True])
def test_part_of_a_batch(cache, G, dt):
    """A slice of the offsets, over a cache as well: the part's rows, and
    nothing else."""
    torch_mod()
    g = torch.Generator().manual_seed(31)
    T, D, start, lens = 900, 64, [0, 250, 251, 600, 900], [250, 1, 300, 300]
    (q64, q), (k64, k), (v64, v) = (normal(g, T, h, D, dt=dt) for h in (G, 1, 1))
    if not cache:
        lens = [start[i + 1] - start[i] for i in range(4)]
    spans = [(start[i], start[i + 1] - start[i], start[i], lens[i]) for i in (1, 2)]
    want = ref.attention(q64, k64, v64, spans, D ** -0.5, True)
    o = torch.full_like(q, 7.0)
    s = ints(start)
    hx.hexattn_fwd(q, k, v, o, None, s[1:4].contiguous(), s[1:3 if cache else 4].contiguous(),
                   ints(lens[1:3]) if cache else None, causal=True)
    near(o[250:600], want["o"][250:600], want["o_mag"][250:600], TOL[dt], "o")
    assert bool((o[:250] == 7).all()) and bool((o[600:] == 7).all())
