"""HexPixelAttention's host side on the CPU, with the library's calls replaced
by plain ones where a test needs their results."""
import pytest

import attn_ref as ref

torch = pytest.importorskip("torch")
hnn = pytest.importorskip("paper_1903_01814_amd.nn")
cases = pytest.importorskip("attn_layer_cases")


@pytest.fixture
def plain_library(monkeypatch):
    """Rotation, attention and steps on host tensors, by the float64 reference
    and the entry points' definitions."""
    def rotary(q, k, pos, freq, axis, wq, wk, qo, ko, eps=1e-6, norm=True, v=None, vo=None,
               slot=None):
        turn = lambda x, w: ref.rotary(x.double(), w.double(), pos, freq, axis, eps,  # noqa: E731
                                       norm)[0].float()
        qo.copy_(turn(q, wq))
        for x, to in ((turn(k, wk), ko), (v, vo)):
            for t in range(0 if to is None else x.shape[0]):
                at = t if slot is None else int(slot[t])
                if 0 <= at < to.shape[0]:
                    to[at] = x[t]

    def attention(q, k, v, o, lse, q_start, k_start=None, k_len=None, scale=None, causal=False):
        T, Tk = q.shape[0], k.shape[0]
        cut = lambda a, n: [min(max(i, 0), n) for i in a.tolist()]  # noqa: E731
        qs, ks = cut(q_start, T), cut(q_start if k_start is None else k_start, Tk)
        spans = []
        for s in range(len(qs) - 1):
            m = ks[s + 1] - ks[s] if k_len is None else int(k_len[s])
            spans.append((qs[s], max(0, qs[s + 1] - qs[s]), ks[s], min(max(m, 0), Tk - ks[s])))
        r = ref.attention(q.double(), k.double(), v.double(), spans, q.shape[2] ** -0.5, causal)
        for q0, n, _, _ in spans:
            o[q0:q0 + n] = r["o"][q0:q0 + n].float()
            if lse is not None:
                lse[q0:q0 + n] = r["lse"][q0:q0 + n].float()

    def step(q, k, v, o, ws, k_start, k_len, max_len):
        S, n = q.shape[:2]
        starts = torch.arange(0, S * n + 1, n)
        attention(q.flatten(0, 1), k, v, o.flatten(0, 1), None, starts, k_start,
                  k_len.clamp(max=max_len), causal=True)

    monkeypatch.setattr(hnn.hx, "hexrotary_fwd", rotary)
    monkeypatch.setattr(hnn.hx, "hexattn_fwd", attention)
    monkeypatch.setattr(hnn.hx, "hexattn_step", step)
    monkeypatch.setattr(hnn.hx, "hexattn_step_workspace", lambda *a: 0)


def plain_layer(monkeypatch, **kw):
    """A training layer whose attention passes the queries on and whose dropout
    draws its mask on the CPU from the words it is given; the words of every
    call."""
    words = []

    class Attention:
        @staticmethod
        def apply(qkv, wq, wk, pos, freq, axis, start, heads, eps, causal):
            return qkv[:, :heads[0]]

    def dropout(x, p, rng, residual=None, call=0):
        words.append(rng.tolist())
        g = torch.Generator().manual_seed(hash(tuple(words[-1])) & 0xFFFFFFFF)
        return residual + x * (torch.rand(x.shape, generator=g) >= p) / (1 - p)

    monkeypatch.setattr(hnn, "HexPixelAttentionFunction", Attention)
    monkeypatch.setattr(hnn, "hex_dropout", dropout)
    torch.manual_seed(1)
    return hnn.HexPixelAttention(32, 2, **kw), words


def test_recomputed_forward_has_the_same_mask(monkeypatch):
    """Activation checkpointing runs the forward again for the backward: it has
    to get the output's mask, and other calls other masks."""
    from torch.utils.checkpoint import checkpoint
    layer, words = plain_layer(monkeypatch, dropout=0.5)
    x = torch.randn(20, 32)
    for reentrant in (False, True):
        del words[:]
        grads = []
        for run in (layer, lambda *a: checkpoint(layer, *a, use_reentrant=reentrant)):
            torch.manual_seed(7)
            xi = x.clone().requires_grad_(True)
            y = run(xi, None, None)
            grads.append((y.detach(), *torch.autograd.grad(y.square().sum(), xi))
                         if not reentrant else (y.detach(),))
            if reentrant:
                y.square().sum().backward()
                grads[-1] += (xi.grad,)
        assert len(words) == 3 and words[0] == words[1] == words[2]
        for a, b in zip(*grads):
            assert torch.equal(a, b)
        layer(x, None, None)
        assert words[3] != words[2]


def test_mask_words_are_no_state_of_the_layer(monkeypatch):
    """Two layers, and two calls of one, draw different words; nothing of them
    is in the layer's state, where wrappers would give every rank the same."""
    layer, words = plain_layer(monkeypatch, dropout=0.1)
    x = torch.randn(4, 32)
    before = {k: v.clone() for k, v in layer.state_dict().items()}
    layer(x, None, None), layer(x, None, None)
    assert words[0] != words[1]
    after = layer.state_dict()
    assert before.keys() == after.keys()
    assert all(torch.equal(before[k], after[k]) for k in before)
    assert "rng" not in dict(layer.named_buffers())


def test_state_with_mask_words_loads(monkeypatch):
    """States saved when the layer still held the words."""
    layer, _ = plain_layer(monkeypatch, dropout=0.1)
    net = torch.nn.Sequential(layer)
    state = net.state_dict()
    state["0.rng"] = torch.tensor([3, 4])
    net.load_state_dict(state)


@pytest.mark.parametrize("move", [
    lambda n: n.to(torch.bfloat16), lambda n: n.bfloat16(), lambda n: n.double().float(),
    lambda n: n.half().to(torch.float32), lambda n: n.to("meta").to_empty(device="cpu")])
def test_frequencies_keep_their_bits(move):
    """A layer of another type still turns by float32 frequencies, the ones that
    it was built with."""
    net = torch.nn.Sequential(hnn.HexPixelAttention(64, 2, bases=(5000.0, 70.0)))
    freq, axis = hnn.hex_frequencies(32, (5000.0, 70.0))
    net = move(net)
    assert net[0].freq.dtype is torch.float32 and torch.equal(net[0].freq, freq)
    assert net[0].axis.dtype is torch.int32 and torch.equal(net[0].axis, axis)


def test_frequencies_of_ones_own_keep_their_bits():
    layer = hnn.HexPixelAttention(64, 2)
    mine = torch.rand(16)
    layer.freq.copy_(mine)
    layer.to(torch.bfloat16)
    assert layer.qkv.weight.dtype is torch.bfloat16 and torch.equal(layer.freq, mine)


@pytest.mark.parametrize("lead,trail", [(0, 0), (0, 4), (6, 0), (3, 2)])
def test_prefill_with_unused_tokens(plain_library, lead, trail):
    cases.unused_tokens("cpu", lead, trail)


def test_prefill_refuses_other_offsets(plain_library):
    """As many offsets as streams and one; nothing is counted before."""
    st = cases.Streams("cpu", [4, 4])
    c = st.cache(8)
    x, pos, start = st.pack([range(4), range(4)])
    with pytest.raises(ValueError, match="start has shape"):
        st.layer.prefill(x, pos, start[:2], c, 4)
    assert c.most == 0 and c.length.tolist() == [0, 0]
    none = st.layer.new_cache(0, 8)
    assert torch.equal(st.layer.prefill(x, pos, start[:1], none, 4), x)


@pytest.mark.parametrize("capacity,longest,lens,kept", [
    (8, 8, [11, 2, 2], [8, 2, 2]), (8, 5, [11, 2, 0], [5, 2, 0]), (9, 6, [7, 6, 20], [6, 6, 6]),
    (5, 0, [3, 1, 0], [0, 0, 0]), (12, 9, [9, 1, 4], [9, 1, 4])])
def test_prompts_past_their_room(plain_library, capacity, longest, lens, kept):
    cases.cut_prompts("cpu", capacity, longest, lens, kept)


def test_second_prompt_past_its_room(plain_library):
    cases.second_prompt_cut("cpu")


def test_refused_calls_leave_the_cache(plain_library, monkeypatch):
    """Calls that the library refuses (here: positions of another type) count
    no token."""
    def refuse(*a, **kw):
        raise TypeError("pos has dtype torch.float64")
    st = cases.Streams("cpu", [4, 4])
    c = st.cache(6)
    x, pos, start = st.pack([range(4), range(4)])
    rotary = hnn.hx.hexrotary_fwd
    for _ in range(3):
        monkeypatch.setattr(hnn.hx, "hexrotary_fwd", refuse)
        with pytest.raises(TypeError):
            st.layer.prefill(x, pos.double(), start, c, 4)
        with pytest.raises(TypeError):
            st.layer.step(x[:2, None], pos[:2, None].double(), c)
        monkeypatch.setattr(hnn.hx, "hexrotary_fwd", rotary)
        assert c.most == 0 and c.length.tolist() == [0, 0]
    y = st.layer.prefill(x, pos, start, c, 4)
    cases.near(y[4:], st.whole(1, list(range(4))))
    with pytest.raises(ValueError, match="capacity"):
        st.layer.step(x.view(2, 4, 32)[:, :3], pos.view(2, 4, 3)[:, :3], c)
    assert c.most == 4 and c.length.tolist() == [4, 4]


def test_streams_in_turn(plain_library):
    cases.streams_in_turn("cpu")


def test_bounds_of_each_stream():
    """One number for all streams or one for each; what does not fit changes
    nothing."""
    c = hnn.HexCache(3, 10, 1, 8)
    c.reserve([4, 0, 7])
    c.reserve(3)
    assert c.most == 10
    c.reserve([3, 5, 0])
    for more in (1, [0, 3, 0], [0, 0, 1]):
        with pytest.raises(ValueError, match="do not fit the capacity of 10"):
            c.reserve(more)
    for bad in ([1, 2], [0, 0, 0, 0], -1, [0, -1, 0]):
        with pytest.raises(ValueError):
            c.reserve(bad)
    c.reserve((0, 2, 0))
    assert c.most == 10
    c.most = 4
    c.reserve([6, 6, 0]), c.reserve([0, 0, 6])
    with pytest.raises(ValueError, match="capacity"):
        c.reserve(1)


def test_nothing_to_do(plain_library):
    with torch.no_grad():
        cases.nothing_to_do("cpu")
