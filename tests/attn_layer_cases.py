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
