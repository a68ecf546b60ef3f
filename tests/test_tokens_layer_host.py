"""The token-wise layers' host side on the CPU, with the library's functions
replaced by plain ones."""
import pytest

torch = pytest.importorskip("torch")
hnn = pytest.importorskip("paper_1903_01814_amd.nn")

F = torch.nn.functional


@pytest.fixture
def plain(monkeypatch):
    """Layer norm, projections, gated blocks and dropout by torch, each call's name
    written down."""
    calls = []

    def norm(x, weight, bias=None, eps=1e-5):
        calls.append("norm")
        return F.layer_norm(x, x.shape[-1:], weight, bias, eps)

    def linear(x, weight, bias=None, residual=None, activation=None):
        calls.append("linear")
        y = F.linear(x, weight, bias)
        return y if residual is None else y + residual

    def ffn(x, w1, w2, b1=None, b2=None, activation="silu", residual=False, norm=None):
        calls.append("ffn")
        n = x if norm is None else F.layer_norm(x, x.shape[-1:], *norm)
        g, u = F.linear(n, w1, b1).chunk(2, -1)
        y = F.linear(F.silu(g) * u, w2, b2)
        return y + x if residual else y

    def dropout(x, p, rng, residual=None, call=0):
        calls.append("dropout")
        return F.dropout(x, p) + residual

    for name, f in (("hex_layer_norm", norm), ("hex_linear", linear), ("hex_feed_forward", ffn),
                    ("hex_dropout", dropout)):
        monkeypatch.setattr(hnn, name, f)
    return calls


def served(block, x):
    """What prefill and step give behind an attention that passes x on."""
    block.attention.prefill = lambda x, *a: x
    block.attention.step = lambda x, *a: x
    return block.prefill(x, None, None, None, 9), block.step(x, None, None)


def test_serving_drops_nothing(plain):
    """prefill and step of a block in training give what they give in evaluation; its
    forward's feed-forward layer drops."""
    torch.manual_seed(0)
    block = hnn.HexPixelBlock(16, 2, hidden=24, causal=True, dropout=0.5)
    x = torch.randn(6, 16)
    want = block.eval().feed_forward(x)
    for y in served(block.train(), x):
        assert torch.equal(y, want)
    assert "dropout" not in plain
    assert not torch.equal(block.feed_forward(x), want) and "dropout" in plain


def test_serving_calls_the_layer(plain):
    """Hooks of the feed-forward layer run while serving, and another module may stand
    in its place."""
    torch.manual_seed(0)
    block = hnn.HexPixelBlock(16, 2, hidden=24, causal=True, dropout=0.5)
    x, seen = torch.randn(6, 16), []
    block.feed_forward.register_forward_hook(lambda m, a, y: seen.append(a[0] is x))
    served(block, x)
    assert seen == [True, True]
    block.feed_forward = torch.nn.Linear(16, 3)
    for y in served(block, x):
        assert torch.equal(y, block.feed_forward(x))


class Passing:
    """Attention that passes the queries on."""

    @staticmethod
    def apply(qkv, wq, wk, pos, freq, axis, start, heads, eps, causal):
        return qkv[:, :heads[0]]


def tiny_block(monkeypatch, dropout=0.0):
    monkeypatch.setattr(hnn, "HexPixelAttentionFunction", Passing)
    torch.manual_seed(0)
    return hnn.HexPixelBlock(16, 2, hidden=24, dropout=dropout), torch.randn(6, 16)


def test_block_without_hooks_is_fused(plain, monkeypatch):
    """Norm and projection, projection with its residual, norm and gated block: four
    calls of the library."""
    block, x = tiny_block(monkeypatch)
    block(x, None, None)
    assert plain == ["norm", "linear", "linear", "ffn"]


PARTS = ["attention.norm", "attention.qkv", "attention.out", "feed_forward.norm"]


@pytest.mark.parametrize("training", [False, True])
@pytest.mark.parametrize("name", PARTS)
def test_hooks_of_parts_run(plain, monkeypatch, name, training):
    """Hooks see each part's own result (a projection's without the residual), and
    what they return is taken."""
    block, x = tiny_block(monkeypatch)
    block.train(training)
    part, seen = block.get_submodule(name), []
    want = block(x, None, None)
    before = part.register_forward_pre_hook(lambda m, a: seen.append("pre"))
    after = part.register_forward_hook(lambda m, a, y: seen.append(y))
    y = block(x, None, None)
    # the residual added, or the norm made, apart
    assert float((y - want).detach().abs().max()) <= 1e-5
    assert seen[0] == "pre" and len(seen) == 2
    before.remove(), after.remove()
    zero = part.register_forward_hook(lambda m, a, y: torch.zeros_like(y))
    y = block(x, None, None)
    zero.remove()
    if name == "attention.out":  # only the residual is left
        assert torch.equal(y, block.feed_forward(x))
    if name == "feed_forward.norm":
        a = block.attention(x, None, None)
        assert torch.equal(y, a)  # a gated block without biases of zeros
    assert not torch.equal(y, want)
    assert torch.equal(block(x, None, None), want)


@pytest.mark.parametrize("name", PARTS)
def test_gradient_and_global_hooks_of_parts_run(plain, monkeypatch, name):
    block, x = tiny_block(monkeypatch)
    part, seen = block.get_submodule(name), []
    h = part.register_full_backward_hook(lambda m, i, o: seen.append(m))
    block(x.requires_grad_(True), None, None).sum().backward()
    h.remove()
    assert seen == [part]
    h = torch.nn.modules.module.register_module_forward_pre_hook(lambda m, a: seen.append(m))
    block(x, None, None)
    h.remove()
    assert seen.count(part) == 2


class Adapter(torch.nn.Module):
    """A module around another of one argument, as adapters are."""

    def __init__(self, base):
        super().__init__()
        self.base, self.times = base, 3.0

    def forward(self, x):
        return self.times * self.base(x)


@pytest.mark.parametrize("dropout", [0.0, 0.5])
@pytest.mark.parametrize("name", PARTS)
def test_parts_may_be_replaced(plain, monkeypatch, name, dropout):
    """A module in a part's place is the one that is called, without attributes of
    its own but forward."""
    block, x = tiny_block(monkeypatch, dropout)
    where, last = name.rsplit(".", 1)
    outer = block.get_submodule(where)
    block.eval()
    part = getattr(outer, last)
    want = block(x, None, None)
    setattr(outer, last, Adapter(part))
    y = block(x, None, None)
    assert float((y - want).detach().abs().max()) > 1e-3
    getattr(outer, last).times = 1.0
    assert float((block(x, None, None) - want).detach().abs().max()) <= 1e-5
    block.train()(x, None, None).sum().backward()
    assert part.weight.grad is not None


def test_patched_forward_runs(plain, monkeypatch):
    """A forward put on a part's instance is the one that runs."""
    block, x = tiny_block(monkeypatch)
    for name in PARTS:
        part, seen = block.get_submodule(name), []
        old = part.forward
        part.forward = lambda x, old=old, seen=seen: seen.append(1) or old(x)
        block(x, None, None)
        del part.forward
        assert seen == [1], name


def test_projections_are_linear_layers():
    """What looks for torch's linear layers finds the projections of either layer,
    with the same states and the same initial weights."""
    torch.manual_seed(3)
    a = hnn.HexPixelAttention(16, 2)
    torch.manual_seed(3)
    b = hnn.HexPixelAttention(16, 2, norm=True)
    for n in ("qkv", "out"):
        assert isinstance(getattr(b, n), torch.nn.Linear)
        assert torch.equal(getattr(a, n).weight, getattr(b, n).weight)
    assert set(b.state_dict()) == set(a.state_dict()) | {"norm.weight", "norm.bias"}
