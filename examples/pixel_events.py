"""Camera events as sequences of lit pixels: convolution, attention, streams.

Synthetic events on a 16 x 16 hexagonal camera: a shape (filled hexagon, ring
or line) lights up somewhere, its pixels in random order of time, over weak
noise.  A hexagonal convolution makes features of the whole image, the lit
pixels become packed tokens with (time, down, right) positions, two attention
layers exchange between them, and the mean of an event's tokens gives its
class.

    python examples/pixel_events.py         # trains, then replays a stream

``train`` returns the accuracy on fresh events; ``stream_error`` feeds events
pixel by pixel through a causal layer and its cache and returns the largest
difference from the whole-event forward.
"""
import os
import sys

import torch
from torch import nn

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1903_01814_amd import nn as hnn  # noqa: E402

H = W = 16
SHAPES = 3


def _cells(shape):
    """Axial cells (dq, ds) of a shape around its centre."""
    out = []
    for dq in range(-3, 4):
        for ds in range(-3, 4):
            d = max(abs(dq), abs(ds), abs(dq + ds))
            if (shape == 0 and d <= 2) or (shape == 1 and d == 3) or (shape == 2 and ds == 0):
                out.append((dq, ds))
    return out


def events(n, gen):
    """n events: images [n][1][H][W], classes, and the packed lit pixels: image
    and pixel number of every token, positions [T][3], offsets [n + 1]."""
    label = torch.randint(SHAPES, (n,), generator=gen)
    img = torch.randn((n, 1, H, W), generator=gen) * 0.1
    centre = torch.randint(4, H - 4, (n, 2), generator=gen)
    image, pixel, time, start = [], [], [], [0]
    for i in range(n):
        r0, c0 = centre[i].tolist()
        lit = []
        for dq, ds in _cells(int(label[i])):
            c = c0 + dq
            lit.append((r0 - c0 // 2 + ds + c // 2) * W + c)  # axial to offset columns
        lit = torch.tensor(lit)
        lit = lit[(lit >= 0) & (lit < H * W)]
        lit = lit[torch.randperm(len(lit), generator=gen)]
        img[i].view(-1)[lit] += 1.0
        image.append(torch.full_like(lit, i))
        pixel.append(lit)
        time.append(torch.arange(len(lit)).float())
        start.append(start[-1] + len(lit))
    image, pixel = torch.cat(image), torch.cat(pixel)
    pos = torch.cat([torch.cat(time)[:, None], hnn.hex_pixel_positions(H, W)[pixel]], dim=1)
    return img, label, image, pixel, pos, torch.tensor(start, dtype=torch.int32)


class PixelNet(nn.Module):
    def __init__(self, dim=64, heads=4, kv_heads=2, dropout=0.1, device=None, dtype=None):
        super().__init__()
        kw = {"device": device, "dtype": dtype}
        self.conv = hnn.HexConv2d(1, dim, 1, relu=True, **kw)
        self.blocks = nn.ModuleList(
            hnn.HexPixelAttention(dim, heads, kv_heads, dim // heads, dropout=dropout, **kw)
            for _ in range(2))
        self.head = nn.Linear(dim, SHAPES, **kw)

    def forward(self, img, image, pixel, pos, start):
        f = self.conv(img).flatten(2)  # [n][dim][H W]
        x = f[image, :, pixel]         # tokens [T][dim]
        for b in self.blocks:
            x = b(x, pos, start)
        n = start.shape[0] - 1
        event = torch.zeros((n, x.shape[1]), dtype=torch.float32, device=x.device)
        event.index_add_(0, image, x.float())
        event /= (start[1:] - start[:-1])[:, None].clamp(min=1)
        return self.head(event.to(x.dtype))


def train(steps=120, batch=96, dtype=torch.float32, device="cuda", seed=0, log=None):
    torch.manual_seed(seed)
    gen = torch.Generator().manual_seed(seed)
    net = PixelNet(device=device, dtype=dtype)
    opt = torch.optim.Adam(net.parameters(), lr=2e-3)

    def load(n):
        img, label, *rest = events(n, gen)
        return [img.to(dtype).to(device), label.to(device)] + [t.to(device) for t in rest]

    for i in range(steps):
        img, label, *rest = load(batch)
        loss = nn.functional.cross_entropy(net(img, *rest).float(), label)
        opt.zero_grad(set_to_none=True)
        loss.backward()
        opt.step()
        if log and i % 20 == 0:
            log("step %d loss %.3f" % (i, float(loss.detach())))
    net.eval()
    with torch.no_grad():
        img, label, *rest = load(512)
        return float((net(img, *rest).argmax(1) == label).float().mean())


@torch.no_grad()
def stream_error(streams=5, prompt=7, tokens=9, dtype=torch.float32, device="cuda", seed=1):
    torch.manual_seed(seed)
    dim, T = 64, prompt + tokens
    layer = hnn.HexPixelAttention(dim, 4, 2, 16, causal=True, device=device, dtype=dtype).eval()
    x = torch.randn(streams, T, dim, device=device).to(dtype)
    pos = torch.rand(streams, T, 3, device=device) * 16
    start = torch.arange(0, streams * T + 1, T, dtype=torch.int32, device=device)
    whole = layer(x.view(-1, dim), pos.view(-1, 3), start).view(streams, T, dim)
    cache = layer.new_cache(streams, T)
    first = torch.arange(0, streams * prompt + 1, prompt, dtype=torch.int32, device=device)
    got = [layer.prefill(x[:, :prompt].reshape(-1, dim), pos[:, :prompt].reshape(-1, 3), first,
                         cache, prompt).view(streams, prompt, dim)]
    t = prompt
    while t < T:
        n = min(T - t, 1 + t % 2)  # one or two tokens at a time
        got.append(layer.step(x[:, t:t + n].contiguous(), pos[:, t:t + n].contiguous(), cache))
        t += n
    return float((torch.cat(got, 1).float() - whole.float()).abs().max())


if __name__ == "__main__":
    print("accuracy on fresh events: %.3f" % train(log=print))
    print("streamed against whole events: largest difference %.2e" % stream_error())
