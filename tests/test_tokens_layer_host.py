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
