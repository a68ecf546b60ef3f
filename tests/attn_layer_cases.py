"""Prompts and steps of HexPixelAttention over a cache, on a given device, held
against its whole-sequence forward.  A stream's tokens are random rows of x with
positions of their own.  float32: projections and sums of up to 64 products in
another order, 2e-5 of values up to 4."""
import torch

from paper_1903_01814_amd import nn as hnn

TOL = 2e-5


class Streams:
    """Streams of tokens for a causal layer, and what it gives for them whole."""

    def __init__(self, device, lens, seed=0):
        torch.manual_seed(seed)
        self.device = device
        self.layer = hnn.HexPixelAttention(32, 4, 2, 8, causal=True).eval().to(device)
        self.x = [torch.randn(n, 32).to(device) for n in lens]
        self.pos = [(torch.rand(n, 3) * 9).to(device) for n in lens]

    def ints(self, a):
        return torch.tensor(a, dtype=torch.int32, device=self.device)

    @torch.no_grad()
    def whole(self, s, tokens):
        """The forward of these tokens of stream s as one sequence."""
        return self.layer(self.x[s][tokens], self.pos[s][tokens], self.ints([0, len(tokens)]))

    def pack(self, parts, lead=0, trail=0):
        """x, pos and offsets of parts[s], tokens of stream s, between `lead`
        and `trail` tokens of no sequence."""
        junk = lambda n, w: torch.full((n, w), 3.0, device=self.device)  # noqa: E731
        cat = lambda t, w: torch.cat(  # noqa: E731
            [junk(lead, w)] + [t[s][p] for s, p in enumerate(parts)] + [junk(trail, w)])
        start = [lead]
        for p in parts:
            start.append(start[-1] + len(p))
        return cat(self.x, 32), cat(self.pos, 3), self.ints(start)

    def cache(self, capacity):
        c = self.layer.new_cache(len(self.x), capacity)
        c.k.fill_(7.0), c.v.fill_(7.0)
        return c

    def untouched(self, c):
        """Slots past every stream's length hold what was there."""
        for s, n in enumerate(c.length.tolist()):
            rest = slice(s * c.capacity + n, (s + 1) * c.capacity)
            assert bool((c.k[rest] == 7).all()) and bool((c.v[rest] == 7).all()), s


def near(a, b):
    assert a.shape == b.shape
    if a.numel():
        assert float((a - b).abs().max()) <= TOL


def unused_tokens(device, lead, trail):
    """Tokens before the first stream's and after the last one's: they pass as
    they are and are stored nowhere."""
    st = Streams(device, [5, 0, 9, 3])
    c = st.cache(12)
    parts = [list(range(len(x))) for x in st.x]
    x, pos, start = st.pack(parts, lead, trail)
    y = st.layer.prefill(x, pos, start, c, 9)
    assert c.length.tolist() == [5, 0, 9, 3]
    assert torch.equal(y[:lead], x[:lead]) and torch.equal(y[len(x) - trail:], x[len(x) - trail:])
    at = lead
    for s, p in enumerate(parts):
        if p:
            near(y[at:at + len(p)], st.whole(s, p))
        at += len(p)
    st.untouched(c)
    # the next tokens see the cached ones
    st.x = [torch.cat([x, torch.ones(1, 32, device=device)]) for x in st.x]
    st.pos = [torch.cat([p, torch.ones(1, 3, device=device)]) for p in st.pos]
    y = st.layer.step(torch.stack([x[-1:] for x in st.x]), torch.stack([p[-1:] for p in st.pos]), c)
    for s in range(4):
        near(y[s], st.whole(s, list(range(len(st.x[s]))))[-1:])


def cut_prompts(device, capacity, longest, lens, kept):
    """Prompts past `longest` or their stream's room: the first tokens, as many
    as fit, are stored and see what they would see alone; the others pass as
    they are.  Steps go on behind them."""
    st = Streams(device, [n + 2 for n in lens], seed=1)
    c = st.cache(capacity)
    x, pos, start = st.pack([range(n) for n in lens], lead=1)
    y = st.layer.prefill(x, pos, start, c, longest)
    assert c.length.tolist() == kept and c.most >= max(kept)
    at = 1
    for s, n in enumerate(lens):
        near(y[at:at + kept[s]], st.whole(s, list(range(kept[s]))))
        assert torch.equal(y[at + kept[s]:at + n], x[at + kept[s]:at + n])
        at += n
    st.untouched(c)
    steps = capacity - c.most
    for i in range(min(steps, 2)):
        new = [slice(n + i, n + i + 1) for n in lens]
        y = st.layer.step(torch.stack([a[p] for a, p in zip(st.x, new)]),
                          torch.stack([a[p] for a, p in zip(st.pos, new)]), c)
        for s, n in enumerate(lens):
            near(y[s], st.whole(s, list(range(kept[s])) + list(range(n, n + i + 1)))[-1:])
        st.untouched(c)
    assert c.most <= capacity and max(c.length.tolist()) <= c.most


def second_prompt_cut(device):
    """A second prompt of streams that already hold tokens: it sees them, and is
    cut where the streams are full."""
    st = Streams(device, [9, 9, 9], seed=2)
    c = st.cache(8)
    parts = [[0, 1, 2, 3, 4], [0], []]
    x, pos, start = st.pack(parts)
    st.layer.prefill(x, pos, start, c, 5)
    more = [[5, 6, 7, 8], [1, 2, 3], [0, 1, 2, 3, 4, 5]]
    x, pos, start = st.pack(more, trail=2)
    y = st.layer.prefill(x, pos, start, c, 3)
    assert c.length.tolist() == [8, 4, 3] and c.most == 8
    near(y[:3], st.whole(0, list(range(8)))[5:])
    near(y[4:7], st.whole(1, list(range(4)))[1:])
    near(y[7:10], st.whole(2, list(range(3))))
    assert torch.equal(y[3:4], x[3:4]) and torch.equal(y[10:], x[10:])
    st.untouched(c)


def streams_in_turn(device):
    """Prompts of one stream after another, each with its own bound: the cache
    holds as many tokens of every stream as it has room for."""
    st = Streams(device, [6, 8, 7], seed=3)
    c = st.cache(8)
    for s, parts in ((0, [[0, 1, 2], [], []]), (1, [[], list(range(8)), []]),
                     (2, [[], [], [0, 1, 2, 3]]), (0, [[3, 4, 5], [], []]),
                     (2, [[], [], [4, 5, 6]])):
        x, pos, start = st.pack(parts)
        y = st.layer.prefill(x, pos, start, c, [len(p) for p in parts])
        near(y, st.whole(s, list(range(parts[s][-1] + 1)))[parts[s][0]:])
    assert c.length.tolist() == [6, 8, 7] and c.most == 8
    # a bound of its own cuts a stream's prompt too
    x, pos, start = st.pack([[0, 1], [], []])
    y = st.layer.prefill(x, pos, start, c, (1, 0, 1))
    assert c.length.tolist() == [7, 8, 7] and torch.equal(y[1], x[1])
    st.untouched(c)


def nothing_to_do(device):
    """No tokens, no streams: empty results, and a cache that stays empty."""
    st = Streams(device, [2, 2])
    c = st.cache(4)
    x, pos, start = st.pack([[], []])
    assert st.layer.prefill(x, pos, start, c, 3).shape == (0, 32)
    assert c.length.tolist() == [0, 0]
    for offsets in (start, start[:1]):
        assert st.layer(x, pos, offsets).shape == (0, 32)
    none = st.layer.new_cache(0, 4)
    assert st.layer.prefill(x, pos, start[:1], none, 1).shape == (0, 32)
    y = st.layer.step(x.view(0, 2, 32), pos.view(0, 2, 3), none)
    assert y.shape == (0, 2, 32) and none.most == 2
    st.untouched(c)
