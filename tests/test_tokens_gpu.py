"""Layer norm, projections and gated feed-forward blocks against float64, at the
sizes where they can go wrong: one token, numbers of tokens and features around
the tiles' and vectors', strided rows, every activation, each output left out,
infinities and NaN in other rows, other streams, captured graphs.

Bounds are derived in tokens_ref."""
import pytest

import tokens_ref as ref
from gpu_helpers import tdtype, torch_mod
from paper_1903_01814_amd import hexconv as hx

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ACTS = {"none": hx.HEX_ACT_NONE, "relu": hx.HEX_ACT_RELU, "gelu": hx.HEX_ACT_GELU,
        "silu": hx.HEX_ACT_SILU}
DTYPES = ["f32", "bf16"]


def normal(g, *shape, dt="f32", std=1.0, mean=0.0):
    """float64 values exact in dt, and the device tensor of them."""
    t = (torch.randn(shape, generator=g) * std + mean).to(tdtype(dt))
    return t.double(), t.cuda()


def nan(*shape, dt="f32"):
    return torch.full(shape, float("nan"), dtype=tdtype(dt), device="cuda")


def strided(t, pad):
    """The same values with rows `pad` elements further apart, and the whole
    tensor around them (NaN)."""
    if pad == 0:
        return t, t
    whole = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype,
                       device=t.device)
    whole[:, :t.shape[1]] = t
    return whole[:, :t.shape[1]], whole


def space(nbytes):
    """A workspace that holds NaN, as fresh memory may."""
    if not nbytes:
        return None
    return torch.full(((nbytes + 3) // 4,), float("nan"), device="cuda").view(torch.uint8)[:nbytes]


def near(got, want, what):
    value, bound = want
    got = got.double().cpu()
    assert got.shape == value.shape, what
    assert torch.isfinite(got).all(), "%s: %d not finite" % (
        what, int((~torch.isfinite(got)).sum()))
    err = (got - value).abs()
    bad = err > bound
    assert not bad.any(), "%s: %d of %d off, worst %.3g of its bound" % (
        what, int(bad.sum()), got.numel(), float((err / bound.clamp_min(1e-300)).max()))


def zero(like):
    return torch.zeros(like, dtype=torch.float64)


# -------------------------------------------------------------------- norm

def run_norm(T, C, dt, pad=0, weights=True, res=True, seed=0, x=None, eps=1e-5):
    g = torch.Generator().manual_seed(seed + T * 31 + C)
    x64, xd = normal(g, T, C, dt=dt, std=1.5, mean=0.3) if x is None else x
    w64, w = normal(g, C, dt=dt, std=0.2, mean=1.0)
    b64, b = normal(g, C, dt=dt, std=0.3)
    dy64, dy = normal(g, T, C, dt=dt)
    r64, r = normal(g, T, C, dt=dt)
    if not weights:
        w64, b64, w, b = torch.ones(C).double(), zero((C,)), None, None
    if not res:
        r64, r = zero((T, C)), None
    want = ref.norm(x64, w64, b64, eps, dt, dy64, r64)
    (xs, _), (dys, _) = strided(xd, pad), strided(dy, 2 * pad)
    rs = None if r is None else strided(r, 3 * pad)[0]
    (y, ywhole), (dx, dxwhole) = strided(nan(T, C, dt=dt), pad), strided(nan(T, C, dt=dt), pad)
    mean, rstd = nan(T), nan(T)
    hx.hexnorm_fwd(xs, w, b, y, mean, rstd, eps=eps)
    dw, db = nan(C), nan(C)
    ws = space(hx.hexnorm_bwd_workspace(T, C, hx._dtype_code(xd)))
    hx.hexnorm_bwd(xs, w, mean, rstd, dys, rs, dx, dw, db, ws)
    torch.cuda.synchronize()
    got = {"y": y, "mean": mean, "rstd": rstd, "dx": dx, "dw": dw, "db": db}
    for name in got:
        near(got[name], want[name], name)
    if pad:
        assert torch.isnan(ywhole[:, C:]).all() and torch.isnan(dxwhole[:, C:]).all()
    return got


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("C", [1, 3, 8, 9, 63, 64, 65, 97, 128, 200, 256, 257, 500, 512, 1000, 1024,
                               1025, 2048, 2055, 4096, 5000, 8192, 16384])
@pytest.mark.parametrize("T", [1, 5, 130])
def test_norm_sizes(T, C, dt):
    torch_mod()
    run_norm(T, C, dt)


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("T,C,pad", [(33, 97, 1), (70, 64, 8), (9, 1024, 3), (257, 40, 24),
                                     (4500, 24, 0), (2100, 320, 0), (1300, 2048, 0)])
def test_norm_rows(T, C, pad, dt):
    """Strides of any number, and more rows than blocks."""
    torch_mod()
    run_norm(T, C, dt, pad=pad)


@pytest.mark.parametrize("dt", DTYPES)
def test_norm_without(dt):
    """No weights, no residual, no statistics, no weights' gradients."""
    torch_mod()
    got = run_norm(50, 72, dt, weights=False, res=False)
    g = torch.Generator().manual_seed(50 * 31 + 72)
    _, x = normal(g, 50, 72, dt=dt, std=1.5, mean=0.3)
    y = nan(50, 72, dt=dt)
    hx.hexnorm_fwd(x, None, None, y)
    assert torch.equal(y, got["y"])
    dy = torch.ones_like(x)
    both = []
    for dw, db in ((None, None), (nan(72), None), (None, nan(72)), (nan(72), nan(72))):
        dx = nan(50, 72, dt=dt)
        ws = space(hx.hexnorm_bwd_workspace(50, 72, hx._dtype_code(x)))
        hx.hexnorm_bwd(x, None, got["mean"], got["rstd"], dy, None, dx, dw, db,
                       None if dw is None and db is None else ws)
        both.append((dx, dw, db))
    for dx, dw, db in both:
        assert torch.equal(dx, both[3][0])
        assert dw is None or torch.equal(dw, both[3][1])
        assert db is None or torch.equal(db, both[3][2])


@pytest.mark.parametrize("dt", DTYPES)
def test_norm_of_constant_rows(dt):
    """Rows without variance: n is 0 and 1 / sqrt(eps) the factor; a large mean
    with a small spread keeps the spread's digits."""
    torch_mod()
    x = torch.full((3, 48), 7.0, dtype=tdtype(dt))
    run_norm(3, 48, dt, x=(x.double(), x.cuda()))
    x = (torch.randn(4, 96, generator=torch.Generator().manual_seed(1)) + 1000.0).to(tdtype(dt))
    run_norm(4, 96, dt, x=(x.double(), x.cuda()))


def test_norm_keeps_rows_apart():
    """What is not finite in a row stays there."""
    torch_mod()
    x = torch.randn(40, 130, device="cuda")
    w, b = torch.rand(130, device="cuda"), torch.rand(130, device="cuda")
    want, y = nan(40, 130), nan(40, 130)
    hx.hexnorm_fwd(x, w, b, want)
    x[3, 5], x[17, 0] = float("nan"), float("inf")
    hx.hexnorm_fwd(x, w, b, y)
    keep = [i for i in range(40) if i not in (3, 17)]
    assert torch.equal(y[keep], want[keep])
    assert torch.isnan(y[3]).all() and torch.isnan(y[17]).any()


# ------------------------------------------------------------------ linear

def run_linear(T, N, K, dt, act="none", bias=True, res=True, pad=0, gt=None, seed=0):
    g = torch.Generator().manual_seed(seed + T * 31 + N * 7 + K)
    x64, x = normal(g, T, K, dt=dt)
    w64, w = normal(g, N, K, dt=dt, std=K ** -0.5)
    b64, b = normal(g, N, dt=dt, std=0.3)
    r64, r = normal(g, T, N, dt=dt)
    dy64, dy = normal(g, T, N, dt=dt)
    if not bias:
        b64, b = zero((N,)), None
    if not res:
        r64, r = zero((T, N)), None
    want = ref.linear(x64, w64, b64, r64, act, dt, dy64, gt)
    (xs, _), (dys, _) = strided(x, pad), strided(dy, 2 * pad)
    rs = None if r is None else strided(r, 3 * pad)[0]
    (y, ywhole), (dx, dxwhole) = strided(nan(T, N, dt=dt), pad), strided(nan(T, K, dt=dt), pad)
    code = hx._dtype_code(x)
    z = nan(T, N, dt=dt)
    ldx, ldy = xs.stride(0) if T > 1 else K, dys.stride(0) if T > 1 else N
    hx.hexlinear_fwd(xs, w, b, rs, y, z, space(hx.hexlinear_fwd_workspace(T, N, K, ldx, code)),
                     act=ACTS[act])
    y2 = nan(T, N, dt=dt)
    hx.hexlinear_fwd(xs, w, b, rs, y2, None,
                     space(hx.hexlinear_fwd_workspace(T, N, K, ldx, code)), act=ACTS[act])
    dw, db = nan(N, K, dt=gt or dt), nan(N, dt=gt or dt)
    ws = space(hx.hexlinear_bwd_workspace(T, N, K, ldx, ldy, ACTS[act], code))
    hx.hexlinear_bwd(xs, w, z, dys, dx, dw, db, ws, act=ACTS[act])
    torch.cuda.synchronize()
    got = {"y": y, "z": z, "dx": dx, "dw": dw, "db": db}
    for name in got:
        near(got[name], want[name], name)
    assert torch.equal(y, y2)
    if pad:
        assert torch.isnan(ywhole[:, N:]).all() and torch.isnan(dxwhole[:, K:]).all()
    return dict(got, x=xs, w=w, b=b, res=rs, dy=dys)


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("N,K", [(1, 1), (8, 8), (16, 72), (40, 97), (97, 40), (64, 64), (65, 200),
                                 (128, 129), (200, 64), (256, 320), (300, 33)])
@pytest.mark.parametrize("T", [1, 4, 17, 64, 65, 130])
def test_linear_sizes(T, N, K, dt):
    torch_mod()
    run_linear(T, N, K, dt, act="gelu" if (N + K) % 2 else "none")


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("N,K", [(24, 4096), (24, 4100), (4200, 264), (4199, 1033)])
@pytest.mark.parametrize("T", [1, 8, 9, 16, 32, 33])
def test_linear_few_tokens_of_long_rows(T, N, K, dt):
    """Every number of waves that share the contraction, and both block heights."""
    torch_mod()
    run_linear(T, N, K, dt, act="silu")


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("act", sorted(ACTS))
@pytest.mark.parametrize("T,N,K,pad", [(3, 48, 56, 0), (77, 40, 64, 8), (77, 41, 63, 5)])
def test_linear_activations(T, N, K, pad, act, dt):
    """Strided rows; a relu's inputs are away from its border: rows that it
    could turn either way have a bound of its size."""
    torch_mod()
    run_linear(T, N, K, dt, act=act, pad=pad, res=T > 3, bias=act != "silu")


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("T,N,K", [(1000, 64, 200), (700, 520, 264), (2600, 40, 24), (900, 264, 512)])
def test_linear_many_tokens(T, N, K, dt):
    """Several tiles a block's size, divided sums."""
    torch_mod()
    run_linear(T, N, K, dt, act="silu")


@pytest.mark.parametrize("T", [5, 90])
def test_linear_float32_gradients(T):
    torch_mod()
    run_linear(T, 72, 48, "bf16", act="gelu", gt="f32")


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("N,K", [(72, 48), (41, 35)])
def test_linear_parts(N, K, dt):
    """Each gradient alone has the bits it has beside the others (a bias's that it has
    beside its weights', else sums in another order)."""
    torch_mod()
    a = run_linear(90, N, K, dt, act="silu")
    size = float(a["dy"].float().abs().sum(0).max())
    code, act = hx._dtype_code(a["x"]), hx.HEX_ACT_SILU
    for want in (("dx",), ("dw",), ("db",), ("dw", "db"), ()):
        out = {n: torch.full_like(a[n], float("nan")) if n in want else None
               for n in ("dx", "dw", "db")}
        hx.hexlinear_bwd(a["x"], a["w"] if "dx" in want else None, a["z"], a["dy"], out["dx"],
                         out["dw"], out["db"],
                         space(hx.hexlinear_bwd_workspace(90, N, K, K, N, act, code)), act=act)
        for n in want:
            assert same(out[n], a[n], size if want == ("db",) else 0, dt), n


def same(got, want, size, dt):
    """Equal, or where size is given within 122 roundings of sums of that size and
    the result's own."""
    if not size:
        return torch.equal(got, want)
    lim = 2 * (ref.acc(90) * 1.13 * size + ref.R[dt] * want.double().abs())
    return bool(((got.double() - want.double()).abs() <= lim).all())


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("T", [3, 20, 150])
@pytest.mark.parametrize("N,K", [(64, 128), (50, 70)])
def test_linear_keeps_tokens_apart(T, N, K, dt):
    torch_mod()
    a = run_linear(T, N, K, dt, act="gelu")
    x = a["x"].clone()
    x[T // 2, K // 2] = float("nan")
    x[T - 1, 0] = float("inf")
    y = nan(T, N, dt=dt)
    hx.hexlinear_fwd(x, a["w"], a["b"], a["res"], y, None,
                     space(hx.hexlinear_fwd_workspace(T, N, K, K, hx._dtype_code(x))),
                     act=hx.HEX_ACT_GELU)
    keep = [i for i in range(T) if i not in (T // 2, T - 1)]
    assert torch.equal(y[keep], a["y"][keep])
    assert torch.isnan(y[T // 2]).all() and not torch.isfinite(y[T - 1]).all()


# -------------------------------------------------------------------- ffn

def run_ffn(T, K, F, N, dt, act="silu", bias=True, res=True, pad=0, gt=None, seed=0):
    g = torch.Generator().manual_seed(seed + T * 31 + F * 7 + K)
    x64, x = normal(g, T, K, dt=dt)
    w164, w1 = normal(g, 2 * F, K, dt=dt, std=K ** -0.5)
    w264, w2 = normal(g, N, F, dt=dt, std=F ** -0.5)
    b164, b1 = normal(g, 2 * F, dt=dt, std=0.3)
    b264, b2 = normal(g, N, dt=dt, std=0.3)
    r64, r = normal(g, T, N, dt=dt)
    dy64, dy = normal(g, T, N, dt=dt)
    if not bias:
        b164, b1, b264, b2 = zero((2 * F,)), None, zero((N,)), None
    if not res:
        r64, r = zero((T, N)), None
    want = ref.ffn(x64, w164, b164, w264, b264, r64, act, dt, dy64, gt)
    (xs, _), (dys, _) = strided(x, pad), strided(dy, 2 * pad)
    rs = None if r is None else strided(r, 3 * pad)[0]
    (y, ywhole), (dx, dxwhole) = strided(nan(T, N, dt=dt), pad), strided(nan(T, K, dt=dt), pad)
    code, Fp = hx._dtype_code(x), hx.hexffn_width(F)
    ldx, ldy = xs.stride(0) if T > 1 else K, dys.stride(0) if T > 1 else N
    gu, h = nan(T, 2 * Fp, dt=dt), nan(T, Fp, dt=dt)
    nb = hx.hexffn_fwd_workspace(T, K, F, N, ldx, code)
    hx.hexffn_fwd(xs, w1, b1, w2, b2, rs, y, gu, h, space(nb), act=ACTS[act])
    y2, h2 = nan(T, N, dt=dt), nan(T, Fp, dt=dt)
    hx.hexffn_fwd(xs, w1, b1, w2, b2, rs, y2, None, h2, space(nb), act=ACTS[act])
    gt_ = gt or dt
    got = {"dw1": nan(2 * F, K, dt=gt_), "db1": nan(2 * F, dt=gt_), "dw2": nan(N, F, dt=gt_),
           "db2": nan(N, dt=gt_)}
    hx.hexffn_bwd(xs, w1, w2, gu, h, dys, dx, *got.values(),
                  space(hx.hexffn_bwd_workspace(T, K, F, N, ldx, ldy, code)), act=ACTS[act])
    torch.cuda.synchronize()
    got.update(y=y, dx=dx)
    for name in got:
        near(got[name], want[name], name)
    assert torch.equal(y, y2) and torch.equal(h, h2)
    assert not h[:, F:].any() and not gu[:, F:Fp].any() and not gu[:, Fp + F:].any()
    if pad:
        assert torch.isnan(ywhole[:, N:]).all() and torch.isnan(dxwhole[:, K:]).all()
    return dict(got, x=xs, w1=w1, b1=b1, w2=w2, b2=b2, res=rs, dy=dys, gu=gu, h=h)


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("K,F,N", [(1, 1, 1), (8, 8, 8), (64, 72, 64), (40, 97, 40), (97, 40, 33),
                                   (128, 136, 64), (200, 331, 200), (33, 264, 72)])
@pytest.mark.parametrize("T", [1, 3, 16, 40, 64, 65, 131])
def test_ffn_sizes(T, K, F, N, dt):
    torch_mod()
    run_ffn(T, K, F, N, dt)


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
@pytest.mark.parametrize("T,K,F,pad", [(3, 48, 56, 0), (77, 40, 64, 8), (77, 41, 63, 5)])
def test_ffn_activations(T, K, F, pad, act, dt):
    torch_mod()
    run_ffn(T, K, F, K, dt, act=act, pad=pad, res=T > 3, bias=act != "silu")


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("T,K,F", [(700, 64, 200), (1300, 136, 344), (600, 264, 520)])
def test_ffn_many_tokens(T, K, F, dt):
    torch_mod()
    run_ffn(T, K, F, K, dt)


def test_ffn_float32_gradients():
    torch_mod()
    run_ffn(90, 48, 72, 48, "bf16", gt="f32")


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("K,F", [(48, 72), (35, 41)])
def test_ffn_parts(K, F, dt):
    torch_mod()
    a = run_ffn(90, K, F, K, dt)
    code = hx._dtype_code(a["x"])
    names = ("dx", "dw1", "db1", "dw2", "db2")
    # |dg| and |du| are below |dh| max(|u| 1.13, |act g|)
    dh = (a["dy"].double().abs() @ a["w2"].double().abs())
    z = a["x"].double().abs() @ a["w1"].double().abs().t() + a["b1"].double().abs()
    size = float((dh * 1.13 * torch.maximum(z[:, :F], z[:, F:])).sum(0).max())
    for want in (("dx",), ("dw1",), ("db1",), ("dw2",), ("db2",), ("dw1", "db2"), ()):
        out = {n: torch.full_like(a[n], float("nan")) if n in want else None for n in names}
        hx.hexffn_bwd(a["x"], a["w1"], a["w2"], a["gu"], a["h"], a["dy"], *out.values(),
                      space(hx.hexffn_bwd_workspace(90, K, F, K, K, K, code)))
        for n in want:
            alone = n.startswith("db") and n.replace("b", "w") not in want
            assert same(out[n], a[n], size if alone else 0, dt), n


# ------------------------------------------------------- as programs use them

@pytest.mark.parametrize("dt", DTYPES)
def test_no_tokens(dt):
    """Nothing is written but zeros to the weights' gradients."""
    torch_mod()
    ty = tdtype(dt)
    x, w = torch.empty(0, 40, dtype=ty, device="cuda"), torch.ones(24, 40, dtype=ty, device="cuda")
    y = torch.empty(0, 24, dtype=ty, device="cuda")
    hx.hexlinear_fwd(x, w, None, None, y)
    dw, db = nan(24, 40, dt=dt), nan(24, dt=dt)
    hx.hexlinear_bwd(x, w, None, y, x, dw, db, None)
    assert not dw.any() and not db.any()
    w1, w2 = torch.ones(30, 40, dtype=ty, device="cuda"), torch.ones(40, 15, dtype=ty, device="cuda")
    gu, h = (torch.empty(0, n, dtype=ty, device="cuda") for n in (32, 16))
    hx.hexffn_fwd(x, w1, None, w2, None, None, x, gu, h)
    grads = [nan(30, 40), nan(30), nan(40, 15), nan(40)]
    hx.hexffn_bwd(x, w1, w2, gu, h, x, x, *grads, None)
    assert not any(bool(t.any()) for t in grads)
    hx.hexnorm_fwd(x, None, None, x)
    dw, db = nan(40), nan(40)
    m = torch.empty(0, device="cuda")
    hx.hexnorm_bwd(x, None, m, m, x, None, x, dw, db, None)
    assert not dw.any() and not db.any()


def chain(p, ws, out):
    """Norm, projection and feed-forward block, forward and backward, into
    given tensors."""
    T, K = p["x"].shape
    F, N = p["w2"].shape[1], p["w2"].shape[0]
    hx.hexnorm_fwd(p["x"], p["nw"], p["nb"], out["n"], out["mean"], out["rstd"])
    hx.hexlinear_fwd(out["n"], p["w"], p["b"], p["x"], out["y"], out["z"], ws, act=hx.HEX_ACT_GELU)
    hx.hexffn_fwd(out["y"], p["w1"], None, p["w2"], None, out["y"], out["o"], out["gu"], out["h"],
                  ws)
    hx.hexffn_bwd(out["y"], p["w1"], p["w2"], out["gu"], out["h"], p["do"], out["dy"], out["dw1"],
                  None, out["dw2"], None, ws)
    hx.hexlinear_bwd(out["n"], p["w"], out["z"], out["dy"], out["dn"], out["dw"], out["db"], ws,
                     act=hx.HEX_ACT_GELU)
    hx.hexnorm_bwd(p["x"], p["nw"], out["mean"], out["rstd"], out["dn"], p["do"], out["dx"],
                   out["dnw"], out["dnb"], ws)


def chain_state(T, K, F, dt, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ty = tdtype(dt)
    mk = lambda *s, k=1.0: (torch.randn(s, generator=g, device="cuda") * k).to(ty)  # noqa: E731
    p = dict(x=mk(T, K), nw=mk(K), nb=mk(K), w=mk(K, K, k=K ** -0.5), b=mk(K),
             w1=mk(2 * F, K, k=K ** -0.5), w2=mk(K, F, k=F ** -0.5), do=mk(T, K))
    code, Fp = hx._dtype_code(p["x"]), hx.hexffn_width(F)
    need = max(hx.hexlinear_fwd_workspace(T, K, K, K, code),
               hx.hexffn_fwd_workspace(T, K, F, K, K, code),
               hx.hexffn_bwd_workspace(T, K, F, K, K, K, code),
               hx.hexlinear_bwd_workspace(T, K, K, K, K, hx.HEX_ACT_GELU, code),
               hx.hexnorm_bwd_workspace(T, K, code))
    shapes = dict(n=(T, K), y=(T, K), z=(T, K), o=(T, K), gu=(T, 2 * Fp), h=(T, Fp), dy=(T, K),
                  dn=(T, K), dx=(T, K), dw1=(2 * F, K), dw2=(K, F), dw=(K, K), db=(K,))
    out = {n: nan(*s, dt=dt) for n, s in shapes.items()}
    for n, s in dict(mean=(T,), rstd=(T,), dnw=(K,), dnb=(K,)).items():
        out[n] = nan(*s)
    return p, need, out


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("T,K,F", [(2, 64, 96), (130, 72, 100), (300, 97, 65)])
def test_chain_repeats_and_replays(T, K, F, dt):
    """The operators one after another: the same bits again, on another stream,
    and in every replay of a graph, with eager calls of other inputs and dirty
    workspaces between."""
    torch_mod()
    p, need, out = chain_state(T, K, F, dt, 3)
    ws = space(need)
    chain(p, ws, out)
    torch.cuda.synchronize()
    want = {n: t.clone() for n, t in out.items()}
    assert all(bool(torch.isfinite(t).all()) for t in want.values())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for t in out.values():
        t.fill_(float("nan"))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        chain(p, space(need), out)
    side.synchronize()
    for n in want:
        assert torch.equal(out[n], want[n]), n
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain(p, ws, out)
    q, _, other = chain_state(T, K, F, dt, 4)
    for i in range(4):
        for t in out.values():
            t.fill_(float("nan"))
        ws.view(torch.uint8).fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for n in want:
            assert torch.equal(out[n], want[n]), (i, n)
        chain(q, space(need), other)
    # new inputs in the graph's own tensors
    for n in p:
        p[n].copy_(q[n])
    graph.replay()
    torch.cuda.synchronize()
    for n in want:
        assert torch.equal(out[n], other[n]), n


# ------------------------------------------------- sizes of whole training batches

def big64(a, b, chunk=2048):
    """a b^T in float64 on the device, and the sum of its terms' magnitudes."""
    out, mag = (torch.empty(a.shape[0], b.shape[0], dtype=torch.float64, device="cuda")
                for _ in range(2))
    bt, ba = b.double().t().contiguous(), b.double().abs().t().contiguous()
    for i in range(0, a.shape[0], chunk):
        x = a[i:i + chunk].double()
        out[i:i + chunk], mag[i:i + chunk] = x @ bt, x.abs() @ ba
    return out, mag


def near_big(got, want, mag, n, dt, what):
    err = (got.double() - want).abs()
    bound = ref.acc(n) * mag + ref.R[dt] * want.abs()
    bad = err > bound
    assert not bool(bad.any()), "%s: %d off, worst %.3g of its bound" % (
        what, int(bad.sum()), float((err / bound).max()))


@pytest.mark.parametrize("T,N,K,dt", [
    (8500, 2300, 1000, "bf16"),   # large tiles, a rest of rows, part of a tile of k
    (4100, 2050, 2030, "bf16"),   # odd features, laid out before
    (20000, 1032, 1016, "bf16"),  # the contraction of dw shared by all units
    (2100, 1000, 2088, "f32"),
    (9000, 520, 300, "f32"),
])
def test_linear_large(T, N, K, dt):
    """Every row and column of products whose blocks go through large tiles and
    share the contraction in runs."""
    torch_mod()
    g = torch.Generator(device="cuda").manual_seed(T)
    ty = tdtype(dt)
    mk = lambda *s, k=1.0: (torch.randn(s, generator=g, device="cuda") * k).to(ty)  # noqa: E731
    x, w, r, dy = mk(T, K), mk(N, K, k=K ** -0.5), mk(T, N), mk(T, N)
    y, dx, dw, db = nan(T, N, dt=dt), nan(T, K, dt=dt), nan(N, K, dt=dt), nan(N, dt=dt)
    code = hx._dtype_code(x)
    hx.hexlinear_fwd(x, w, None, r, y, None, space(hx.hexlinear_fwd_workspace(T, N, K, K, code)))
    hx.hexlinear_bwd(x, w, None, dy, dx, dw, db,
                     space(hx.hexlinear_bwd_workspace(T, N, K, K, N, 0, code)))
    z, mag = big64(x, w)
    near_big(y, z + r.double(), mag + r.double().abs(), K, dt, "y")
    near_big(dx, *big64(dy, w.t().contiguous()), N, dt, "dx")
    near_big(dw, *big64(dy.t().contiguous(), x.t().contiguous()), T, dt, "dw")
    near_big(db, dy.double().sum(0), dy.double().abs().sum(0), T, dt, "db")
    del z, mag


@pytest.mark.parametrize("T,K,F", [(8300, 1000, 1500), (5000, 520, 2731)])
def test_ffn_large(T, K, F):
    """The gated product and its gradient over large tiles, bfloat16: every h within
    its bound; the other results by the norm of their errors, which are independent
    roundings."""
    torch_mod()
    g = torch.Generator(device="cuda").manual_seed(F)
    mk = lambda *s, k=1.0: (torch.randn(s, generator=g, device="cuda") * k).bfloat16()  # noqa: E731
    x, w1, w2, dy = mk(T, K), mk(2 * F, K, k=K ** -0.5), mk(K, F, k=F ** -0.5), mk(T, K)
    Fp, code = hx.hexffn_width(F), hx._dtype_code(x)
    y, h, gu = nan(T, K, dt="bf16"), nan(T, Fp, dt="bf16"), nan(T, 2 * Fp, dt="bf16")
    hx.hexffn_fwd(x, w1, None, w2, None, x, y, gu, h, space(hx.hexffn_fwd_workspace(T, K, F, K, K, code)))
    dx, dw1, dw2 = nan(T, K, dt="bf16"), nan(2 * F, K, dt="bf16"), nan(K, F, dt="bf16")
    hx.hexffn_bwd(x, w1, w2, gu, h, dy, dx, dw1, None, dw2, None,
                  space(hx.hexffn_bwd_workspace(T, K, F, K, K, K, code)))
    z, mag = big64(x, w1)
    a, s = ref.act(z[:, :F], "silu")
    h64 = a * z[:, F:]
    eg = ref.acc(K) * mag + 1e-6 * z.abs()
    lim = (1.2 * (eg[:, :F] * z[:, F:].abs() + a.abs() * eg[:, F:]) + ref.R["bf16"] * h64.abs() +
           2.0 ** -22 * h64.abs())
    assert bool(((h[:, :F].double() - h64).abs() <= lim).all())
    assert not bool(h[:, F:].any())
    rel = lambda p, q: float((p.double() - q).norm() / q.norm())  # noqa: E731
    # a rounding is 2^-8 / sqrt 3 of a value at the low end of a step, half that at the
    # high end: 1.7e-3 of a norm; two of them 2.4e-3, kept g and u 2.5e-4 more
    y64 = h64 @ w2.double().t().contiguous() + x.double()
    assert rel(y, y64) <= 2.5e-3
    dh = dy.double() @ w2.double()
    dz = torch.cat([dh * z[:, F:] * s, dh * a], 1)
    assert rel(dx, dz @ w1.double()) <= 2.6e-3
    assert rel(dw1, dz.t().contiguous() @ x.double()) <= 2.6e-3
    assert rel(dw2, dy.double().t().contiguous() @ h64) <= 2.6e-3


@pytest.mark.parametrize("scale", [1e-7, 1e4, 1e9])
@pytest.mark.parametrize("T", [5, 200])
def test_ffn_magnitudes(T, scale):
    """g and u far outside float16's exponents: kept as bfloat16, to 2^-7."""
    torch_mod()
    g = torch.Generator().manual_seed(3)
    x64, x = normal(g, T, 40, dt="bf16", std=scale)
    w164, w1 = normal(g, 2 * 72, 40, dt="bf16", std=0.15)
    w264, w2 = normal(g, 40, 72, dt="bf16", std=0.1)
    dy64, dy = normal(g, T, 40, dt="bf16")
    z = lambda *s: torch.zeros(s, dtype=torch.float64)  # noqa: E731
    want = ref.ffn(x64, w164, z(144), w264, z(40), z(T, 40), "silu", "bf16", dy64)
    code = hx._dtype_code(x)
    y, gu, h = nan(T, 40, dt="bf16"), nan(T, 144, dt="bf16"), nan(T, 72, dt="bf16")
    hx.hexffn_fwd(x, w1, None, w2, None, None, y, gu, h,
                  space(hx.hexffn_fwd_workspace(T, 40, 72, 40, 40, code)))
    got = {"dx": nan(T, 40, dt="bf16"), "dw1": nan(144, 40, dt="bf16"), "dw2": nan(40, 72, dt="bf16")}
    hx.hexffn_bwd(x, w1, w2, gu, h, dy, got["dx"], got["dw1"], None, got["dw2"], None,
                  space(hx.hexffn_bwd_workspace(T, 40, 72, 40, 40, 40, code)))
    got["y"] = y
    for n in got:
        near(got[n], want[n], n)


@pytest.mark.parametrize("T", [6, 90])
def test_ffn_keeps_tokens_apart(T):
    """Infinities and NaN of a token reach no other, forward and in dx."""
    torch_mod()
    for dt in DTYPES:
        a = run_ffn(T, 40, 64, 40, dt, bias=False, res=False)
        x = a["x"].clone()
        x[1, 3], x[T - 2, 0] = float("nan"), float("inf")
        code = hx._dtype_code(x)
        y, gu, h = torch.empty_like(a["y"]), torch.empty_like(a["gu"]), torch.empty_like(a["h"])
        hx.hexffn_fwd(x, a["w1"], None, a["w2"], None, None, y, gu, h,
                      space(hx.hexffn_fwd_workspace(T, 40, 64, 40, 40, code)))
        dx = torch.empty_like(a["dx"])
        hx.hexffn_bwd(x, a["w1"], a["w2"], gu, h, a["dy"], dx, None, None, None, None,
                      space(hx.hexffn_bwd_workspace(T, 40, 64, 40, 40, 40, code)))
        keep = [i for i in range(T) if i not in (1, T - 2)]
        assert torch.equal(y[keep], a["y"][keep]) and torch.equal(dx[keep], a["dx"][keep])
        assert torch.isnan(y[1]).all() and torch.isnan(dx[1]).all()
        assert not torch.isfinite(y[T - 2]).all()


# ------------------------------------------------- offsets that pass 32 bits

FAR = (1 << 22) - 8  # the longest stride; 520 rows of it are 2^31 elements and more


def far(t):
    """t's rows a stride of FAR apart (what lies between them is not written)."""
    v = torch.empty((t.shape[0], FAR), dtype=t.dtype, device="cuda")[:, :t.shape[1]]
    return v.copy_(t)


@pytest.mark.parametrize("dt", DTYPES)
def test_norm_far_rows(dt):
    torch_mod()
    T, C = 520, 72
    g = torch.Generator().manual_seed(5)
    (x64, x), (dy64, dy) = (normal(g, T, C, dt=dt) for _ in range(2))
    (w64, w), (b64, b) = (normal(g, C, dt=dt) for _ in range(2))
    want = ref.norm(x64, w64, b64, 1e-5, dt, dy64, zero((T, C)))
    x, dy, y, dx = far(x), far(dy), far(nan(T, C, dt=dt)), far(nan(T, C, dt=dt))
    mean, rstd, dw, db = nan(T), nan(T), nan(C), nan(C)
    hx.hexnorm_fwd(x, w, b, y, mean, rstd)
    hx.hexnorm_bwd(x, w, mean, rstd, dy, None, dx, dw, db,
                   space(hx.hexnorm_bwd_workspace(T, C, hx._dtype_code(x))))
    for name, got in (("y", y), ("dx", dx), ("dw", dw), ("db", db)):
        near(got, want[name], name)


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("N,K", [(48, 64), (41, 63)])
def test_linear_far_rows(N, K, dt):
    torch_mod()
    T = 520
    g = torch.Generator().manual_seed(6)
    x64, x = normal(g, T, K, dt=dt)
    w64, w = normal(g, N, K, dt=dt, std=K ** -0.5)
    r64, r = normal(g, T, N, dt=dt)
    dy64, dy = normal(g, T, N, dt=dt)
    want = ref.linear(x64, w64, zero((N,)), r64, "none", dt, dy64)
    x, r, dy, y, dx = far(x), far(r), far(dy), far(nan(T, N, dt=dt)), far(nan(T, K, dt=dt))
    code, dw, db = hx._dtype_code(x), nan(N, K, dt=dt), nan(N, dt=dt)
    hx.hexlinear_fwd(x, w, None, r, y, None, space(hx.hexlinear_fwd_workspace(T, N, K, FAR, code)))
    hx.hexlinear_bwd(x, w, None, dy, dx, dw, db,
                     space(hx.hexlinear_bwd_workspace(T, N, K, FAR, FAR, 0, code)))
    for name, got in (("y", y), ("dx", dx), ("dw", dw), ("db", db)):
        near(got, want[name], name)


def test_linear_far_rows_of_large_tiles():
    """Offsets within a tile of 256 rows come near 2^32 bytes there."""
    torch_mod()
    T, N, K = 2048, 8192, 512
    g = torch.Generator(device="cuda").manual_seed(7)
    x, w = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((T, K), (N, K)))
    xf, y = far(x), nan(T, N, dt="bf16")
    hx.hexlinear_fwd(xf, w, None, None, y, None, space(hx.hexlinear_fwd_workspace(T, N, K, FAR, 1)))
    value, mag = big64(x, w)
    near_big(y, value, mag, K, "bf16", "y")


def test_linear_output_past_32_bits():
    """More than 2^31 elements of y and of dy; rows at both ends are compared."""
    torch_mod()
    T, N, K = 1050000, 2048, 8
    g = torch.Generator(device="cuda").manual_seed(8)
    x, w = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((T, K), (N, K)))
    y = torch.empty((T, N), dtype=torch.bfloat16, device="cuda")
    hx.hexlinear_fwd(x, w, None, None, y, None, space(hx.hexlinear_fwd_workspace(T, N, K, K, 1)))
    dx = nan(T, K, dt="bf16")
    hx.hexlinear_bwd(x, w, None, y, dx, None, None,
                     space(hx.hexlinear_bwd_workspace(T, N, K, K, N, 0, 1)))
    for rows in (slice(0, 300), slice(T - 700, T)):
        value, mag = big64(x[rows], w)
        near_big(y[rows], value, mag, K, "bf16", "y")
        value, mag = big64(y[rows], w.t())
        near_big(dx[rows], value, mag, N, "bf16", "dx")
