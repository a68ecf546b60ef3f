"""PyTorch layers over libhexconv: hexagonal convolution, pooling, and
attention over lit pixels, as ``torch.autograd.Function``s and
``nn.Module``s, so that they drop into models written with the PyTorch API the
way the paper's layers do (Sec. 2.4).

Tensors are NCHW in the offset-column layout of Sec. 2.1 (odd columns shifted
half a pitch down); weights are ``[C_out, C_in, T]`` with T = 1 + 3k(k+1)
taps in the library's canonical order.  Forward and backward are libhexconv
calls through the ``hexconv`` binding: this module allocates their outputs
and workspaces with torch and keeps what the backward needs, nothing else.
Inputs must live on the GPU in float32 or bfloat16, with weights and bias of
the same dtype; weight and bias gradients are computed in float32 and handed
to autograd in the parameter's dtype.
"""
from __future__ import annotations

import math

import torch
from torch import nn

from . import hexconv as hx


def _empty(shape, like, dtype=None):
    return torch.empty(shape, dtype=like.dtype if dtype is None else dtype,
                       device=like.device)


def _relu_backward(gy, y):
    """gy * [y > 0] by the pooling gradient of the one-tap (k = 0, stride 1)
    average pool, whose gradient is its input, masked by relu_y > 0."""
    g = _empty(gy.shape, gy)
    hx.hexpool_bwd(gy, None, y, g, 0, 1, hx.HEX_POOL_AVG)
    return g


class HexConv2dFunction(torch.autograd.Function):
    """y = hexagonal convolution of x with w (+ b), optionally followed by
    ReLU (fused into the forward kernel's epilogue)."""

    @staticmethod
    def forward(ctx, x, w, b, k, stride, relu):
        x = x.contiguous()
        w = w.contiguous()
        b = None if b is None else b.contiguous()
        if w.dtype != x.dtype or (b is not None and b.dtype != x.dtype):
            raise TypeError("hex_conv2d: x, weight and bias must share a dtype")
        N, _, H, W = x.shape
        Ho, Wo = hx.hex_out_shape(H, W, k, stride)
        y = _empty((N, w.shape[0], Ho, Wo), x)
        hx.hexconv_fwd(x, w, b, y, k, stride, relu=relu)
        ctx.save_for_backward(x, w, y if relu else None)
        ctx.k, ctx.stride, ctx.relu = k, stride, relu
        ctx.has_bias = b is not None
        ctx.bias_dtype = None if b is None else b.dtype
        return y

    @staticmethod
    def backward(ctx, gy):
        x, w, y = ctx.saved_tensors
        k, s = ctx.k, ctx.stride
        gy = gy.contiguous()
        if ctx.relu:
            gy = _relu_backward(gy, y)
        need_x, need_w, need_b = ctx.needs_input_grad[:3]
        need_b = need_b and ctx.has_bias
        dx = dw = db = None
        if not (need_w or need_b):
            if need_x:
                dx = _empty(x.shape, x)
                hx.hexconv_bwd_data(gy, w, dx, k, s)
            return dx, None, None, None, None, None
        N, Ci, H, W = x.shape
        Co = w.shape[0]
        dt = hx.HEX_F32 if x.dtype == torch.float32 else hx.HEX_BF16
        dx = _empty(x.shape, x) if need_x else None
        dw = _empty(w.shape, x, torch.float32)
        db = _empty((Co,), x, torch.float32) if ctx.has_bias else None
        nbytes = hx.hexconv_bwd_workspace(N, Ci, Co, H, W, k, s, dt)
        ws = _empty((nbytes,), x, torch.uint8) if nbytes else None
        hx.hexconv_bwd(x, gy, w, dx, dw, db, ws, k, s)
        gw = dw.to(w.dtype) if need_w else None
        gb = db.to(ctx.bias_dtype) if need_b else None
        return dx, gw, gb, None, None, None


class HexPool2dFunction(torch.autograd.Function):
    """y = hexagonal max or average pooling of x; max pooling keeps the
    winning tap of every output (uint8) for its backward."""

    @staticmethod
    def forward(ctx, x, k, stride, mode):
        x = x.contiguous()
        N, C, H, W = x.shape
        Ho, Wo = hx.hex_out_shape(H, W, k, stride)
        y = _empty((N, C, Ho, Wo), x)
        am = _empty(y.shape, x, torch.uint8) if mode == hx.HEX_POOL_MAX else None
        hx.hexpool_fwd(x, y, am, k, stride, mode)
        ctx.save_for_backward(am)
        ctx.k, ctx.stride, ctx.mode, ctx.in_shape = k, stride, mode, x.shape
        return y

    @staticmethod
    def backward(ctx, gy):
        (am,) = ctx.saved_tensors
        if not ctx.needs_input_grad[0]:
            return None, None, None, None
        dx = _empty(ctx.in_shape, gy)
        hx.hexpool_bwd(gy.contiguous(), am, None, dx, ctx.k, ctx.stride, ctx.mode)
        return dx, None, None, None


def hex_conv2d(x, weight, bias=None, kernel_size=1, stride=1, relu=False):
    """Hexagonal convolution (Sec. 2.3) with a caller-supplied kernel:
    weight [C_out, C_in, 1 + 3k(k+1)], bias [C_out] or None."""
    return HexConv2dFunction.apply(x, weight, bias, int(kernel_size), int(stride),
                                   bool(relu))


def hex_max_pool2d(x, kernel_size, stride):
    """Hexagonal max pooling over the size-k hexagon (Sec. 2.4); taps outside
    the tensor take part as zeros."""
    return HexPool2dFunction.apply(x, int(kernel_size), int(stride), hx.HEX_POOL_MAX)


def hex_avg_pool2d(x, kernel_size, stride):
    """Hexagonal average pooling: the sum over the size-k hexagon divided by
    its tap count, taps outside the tensor counting as zeros (Sec. 2.4)."""
    return HexPool2dFunction.apply(x, int(kernel_size), int(stride), hx.HEX_POOL_AVG)


class HexConv2d(nn.Module):
    """Hexagonal convolution layer of size ``kernel_size`` (the hexagon's
    radius k) and ``stride`` (Sec. 2.3).  ``relu`` fuses a ReLU into the
    forward kernel.  ``debug`` sets every kernel element to 1 and drops the
    bias, the layer then summing each hexagonal neighbourhood (Sec. 3); its
    weights take no gradient.  Initial weights and bias are uniform in
    +-1/sqrt(fan_in) with the hexagonal fan-in C_in * T."""

    def __init__(self, in_channels, out_channels, kernel_size=1, stride=1, bias=True,
                 relu=False, debug=False, device=None, dtype=None):
        super().__init__()
        self.in_channels, self.out_channels = int(in_channels), int(out_channels)
        self.kernel_size, self.stride = int(kernel_size), int(stride)
        self.relu, self.debug = bool(relu), bool(debug)
        T = hx.hex_num_taps(self.kernel_size)
        kw = {"device": device, "dtype": dtype}
        self.weight = nn.Parameter(torch.empty((self.out_channels, self.in_channels, T), **kw),
                                   requires_grad=not self.debug)
        if bias and not self.debug:
            self.bias = nn.Parameter(torch.empty((self.out_channels,), **kw))
        else:
            self.register_parameter("bias", None)
        self.reset_parameters()

    def reset_parameters(self):
        with torch.no_grad():
            if self.debug:
                self.weight.fill_(1.0)
                return
            bound = 1.0 / math.sqrt(self.in_channels * self.weight.shape[2])
            self.weight.uniform_(-bound, bound)
            if self.bias is not None:
                self.bias.uniform_(-bound, bound)

    def forward(self, x):
        return hex_conv2d(x, self.weight, self.bias, self.kernel_size, self.stride,
                          self.relu)

    def extra_repr(self):
        return ("%d, %d, kernel_size=%d, stride=%d, bias=%s, relu=%s, debug=%s"
                % (self.in_channels, self.out_channels, self.kernel_size, self.stride,
                   self.bias is not None, self.relu, self.debug))


class HexMaxPool2d(nn.Module):
    """Hexagonal max pooling of size ``kernel_size`` and ``stride``."""

    def __init__(self, kernel_size, stride):
        super().__init__()
        self.kernel_size, self.stride = int(kernel_size), int(stride)

    def forward(self, x):
        return hex_max_pool2d(x, self.kernel_size, self.stride)

    def extra_repr(self):
        return "kernel_size=%d, stride=%d" % (self.kernel_size, self.stride)


class HexAvgPool2d(nn.Module):
    """Hexagonal average pooling of size ``kernel_size`` and ``stride``."""

    def __init__(self, kernel_size, stride):
        super().__init__()
        self.kernel_size, self.stride = int(kernel_size), int(stride)

    def forward(self, x):
        return hex_avg_pool2d(x, self.kernel_size, self.stride)

    def extra_repr(self):
        return "kernel_size=%d, stride=%d" % (self.kernel_size, self.stride)


# ------------------------------------------------------- three dimensions
# Sec. 2.4: hexagonal x-y planes, equidistant samples along z.  Tensors are
# NCDHW; a kernel of size (k, kz) is the size-k hexagon in the plane times
# the 2kz+1 planes around the centre plane; weights [C_out, C_in, 2kz+1, T];
# stride (s, s_z).

def _pair(v):
    if isinstance(v, (tuple, list)):
        a, b = v
        return int(a), int(b)
    return int(v), int(v)


def _relu_backward3d(gy, y):
    """gy * [y > 0] via the gradient of the one-tap 3-D average pool."""
    g = _empty(gy.shape, gy)
    hx.hexpool3d_bwd(gy, None, y, g, 0, 0, 1, 1, hx.HEX_POOL_AVG)
    return g


class HexConv3dFunction(torch.autograd.Function):
    """y = 3-D hexagonal convolution of x with w (+ b), optionally ReLU."""

    @staticmethod
    def forward(ctx, x, w, b, k, kz, stride, stride_z, relu):
        x = x.contiguous()
        w = w.contiguous()
        b = None if b is None else b.contiguous()
        if w.dtype != x.dtype or (b is not None and b.dtype != x.dtype):
            raise TypeError("hex_conv3d: x, weight and bias must share a dtype")
        N, _, D, H, W = x.shape
        Do, Ho, Wo = hx.hex_out_shape3d(D, H, W, k, kz, stride, stride_z)
        y = _empty((N, w.shape[0], Do, Ho, Wo), x)
        hx.hexconv3d_fwd(x, w, b, y, k, kz, stride, stride_z, relu=relu)
        ctx.save_for_backward(x, w, y if relu else None)
        ctx.geom = (k, kz, stride, stride_z)
        ctx.relu, ctx.has_bias = relu, b is not None
        ctx.bias_dtype = None if b is None else b.dtype
        return y

    @staticmethod
    def backward(ctx, gy):
        x, w, y = ctx.saved_tensors
        k, kz, s, sz = ctx.geom
        gy = gy.contiguous()
        if ctx.relu:
            gy = _relu_backward3d(gy, y)
        need_x, need_w, need_b = ctx.needs_input_grad[:3]
        dx = gw = gb = None
        if need_x:
            dx = _empty(x.shape, x)
            hx.hexconv3d_bwd_data(gy, w, dx, k, kz, s, sz)
        if need_w or (need_b and ctx.has_bias):
            N, Ci, D, H, W = x.shape
            Co = w.shape[0]
            dt = hx.HEX_F32 if x.dtype == torch.float32 else hx.HEX_BF16
            dw = _empty(w.shape, x, torch.float32)
            db = _empty((Co,), x, torch.float32) if ctx.has_bias else None
            nbytes = hx.hexconv3d_bwd_weight_workspace(N, Ci, Co, D, H, W, k, kz, s, sz, dt)
            ws = _empty((nbytes,), x, torch.uint8) if nbytes else None
            hx.hexconv3d_bwd_weight(x, gy, dw, db, ws, k, kz, s, sz)
            gw = dw.to(w.dtype) if need_w else None
            gb = db.to(ctx.bias_dtype) if need_b and ctx.has_bias else None
        return dx, gw, gb, None, None, None, None, None


class HexPool3dFunction(torch.autograd.Function):
    """y = 3-D hexagonal max or average pooling; max pooling keeps the
    winning tap (a 16-bit index) for its backward."""

    @staticmethod
    def forward(ctx, x, k, kz, stride, stride_z, mode):
        x = x.contiguous()
        N, C, D, H, W = x.shape
        Do, Ho, Wo = hx.hex_out_shape3d(D, H, W, k, kz, stride, stride_z)
        y = _empty((N, C, Do, Ho, Wo), x)
        am = _empty(y.shape, x, torch.int16) if mode == hx.HEX_POOL_MAX else None
        hx.hexpool3d_fwd(x, y, am, k, kz, stride, stride_z, mode)
        ctx.save_for_backward(am)
        ctx.geom = (k, kz, stride, stride_z)
        ctx.mode, ctx.in_shape = mode, x.shape
        return y

    @staticmethod
    def backward(ctx, gy):
        (am,) = ctx.saved_tensors
        if not ctx.needs_input_grad[0]:
            return None, None, None, None, None, None
        dx = _empty(ctx.in_shape, gy)
        hx.hexpool3d_bwd(gy.contiguous(), am, None, dx, *ctx.geom, ctx.mode)
        return dx, None, None, None, None, None


def hex_conv3d(x, weight, bias=None, kernel_size=(1, 0), stride=(1, 1), relu=False):
    """3-D hexagonal convolution (Sec. 2.4) with a caller-supplied kernel
    weight [C_out, C_in, 2kz+1, 1 + 3k(k+1)]; kernel_size = (k, kz), stride
    = (s, s_z) (an int applies to both)."""
    k, kz = _pair(kernel_size)
    s, sz = _pair(stride)
    return HexConv3dFunction.apply(x, weight, bias, k, kz, s, sz, bool(relu))


def hex_max_pool3d(x, kernel_size, stride):
    """3-D hexagonal max pooling over the (k, kz) window (Sec. 2.4)."""
    k, kz = _pair(kernel_size)
    s, sz = _pair(stride)
    return HexPool3dFunction.apply(x, k, kz, s, sz, hx.HEX_POOL_MAX)


def hex_avg_pool3d(x, kernel_size, stride):
    """3-D hexagonal average pooling over the (k, kz) window (Sec. 2.4)."""
    k, kz = _pair(kernel_size)
    s, sz = _pair(stride)
    return HexPool3dFunction.apply(x, k, kz, s, sz, hx.HEX_POOL_AVG)


class HexConv3d(nn.Module):
    """3-D hexagonal convolution layer: kernel_size = (k, kz), stride = (s,
    s_z); initial weights uniform in +-1/sqrt(C_in (2kz+1) T)."""

    def __init__(self, in_channels, out_channels, kernel_size=(1, 1), stride=(1, 1), bias=True,
                 relu=False, device=None, dtype=None):
        super().__init__()
        self.in_channels, self.out_channels = int(in_channels), int(out_channels)
        self.kernel_size, self.stride = _pair(kernel_size), _pair(stride)
        self.relu = bool(relu)
        k, kz = self.kernel_size
        T = hx.hex_num_taps(k)
        kw = {"device": device, "dtype": dtype}
        self.weight = nn.Parameter(torch.empty((self.out_channels, self.in_channels, 2 * kz + 1, T),
                                               **kw))
        if bias:
            self.bias = nn.Parameter(torch.empty((self.out_channels,), **kw))
        else:
            self.register_parameter("bias", None)
        self.reset_parameters()

    def reset_parameters(self):
        with torch.no_grad():
            fan_in = self.in_channels * self.weight.shape[2] * self.weight.shape[3]
            bound = 1.0 / math.sqrt(fan_in)
            self.weight.uniform_(-bound, bound)
            if self.bias is not None:
                self.bias.uniform_(-bound, bound)

    def forward(self, x):
        return hex_conv3d(x, self.weight, self.bias, self.kernel_size, self.stride, self.relu)

    def extra_repr(self):
        return ("%d, %d, kernel_size=%s, stride=%s, bias=%s, relu=%s"
                % (self.in_channels, self.out_channels, self.kernel_size, self.stride,
                   self.bias is not None, self.relu))


class HexMaxPool3d(nn.Module):
    """3-D hexagonal max pooling, kernel_size = (k, kz), stride = (s, s_z)."""

    def __init__(self, kernel_size, stride):
        super().__init__()
        self.kernel_size, self.stride = _pair(kernel_size), _pair(stride)

    def forward(self, x):
        return hex_max_pool3d(x, self.kernel_size, self.stride)


class HexAvgPool3d(nn.Module):
    """3-D hexagonal average pooling, kernel_size = (k, kz), stride = (s, s_z)."""

    def __init__(self, kernel_size, stride):
        super().__init__()
        self.kernel_size, self.stride = _pair(kernel_size), _pair(stride)

    def forward(self, x):
        return hex_avg_pool3d(x, self.kernel_size, self.stride)


# ------------------------------------------- attention over lit pixels
# The lit pixels of camera events as packed sequences of tokens [T][...]: the
# events one after another, ``start`` (int32 [S + 1], on the device) their
# offsets.  Positions are float32 [T][axes], e.g. time and the pixel's centre.

def hex_pixel_positions(H, W, device=None):
    """Centres [H * W][2] (down, right) of the pixels of an H x W tensor in
    units of the pixel pitch: odd columns lie half a pitch lower, columns are
    sqrt(3)/2 apart (Sec. 2.1)."""
    r = torch.arange(H, dtype=torch.float32, device=device)[:, None]
    c = torch.arange(W, device=device)[None]
    y = r + 0.5 * (c % 2).float()
    x = (c.float() * (math.sqrt(3.0) / 2.0)).expand(H, W)
    return torch.stack([y, x], dim=2).reshape(H * W, 2)


def hex_frequencies(head_dim, bases=(10000.0, 100.0, 100.0), device=None):
    """Frequencies (radians a unit) and axes of a head's head_dim / 2 pairs
    for rotary positions of len(bases) axes: each axis owns a run of pairs
    whose wavelengths grow geometrically from 2 pi up to 2 pi times its
    base."""
    pairs, axes = head_dim // 2, len(bases)
    freq, axis = [], []
    for a, base in enumerate(bases):
        n = pairs // axes + (a < pairs % axes)
        freq += [base ** (-i / n) for i in range(n)]
        axis += [a] * n
    return (torch.tensor(freq, dtype=torch.float32, device=device),
            torch.tensor(axis, dtype=torch.int32, device=device))


def _workspace(nbytes, like):
    return _empty((nbytes,), like, torch.uint8) if nbytes else None


class HexRotaryFunction(torch.autograd.Function):
    """Norm and rotation of query and key heads (hexrotary_fwd)."""

    @staticmethod
    def forward(ctx, q, k, wq, wk, pos, freq, axis, eps, norm):
        qo, ko = _empty(q.shape, q), _empty(k.shape, k)
        hx.hexrotary_fwd(q, k, pos, freq, axis, wq, wk, qo, ko, eps=eps, norm=norm)
        ctx.save_for_backward(q if norm else None, k if norm else None, wq, wk, pos, freq, axis)
        ctx.eps, ctx.norm = eps, norm
        return qo, ko

    @staticmethod
    def backward(ctx, gq, gk):
        q, k, wq, wk, pos, freq, axis = ctx.saved_tensors
        gq, gk = gq.contiguous(), gk.contiguous()
        dq, dk = _empty(gq.shape, gq), _empty(gk.shape, gk)
        dwq, dwk = _rotary_bwd(q, k, pos, freq, axis, wq, wk, gq, gk, dq, dk, ctx.eps, ctx.norm)
        return dq, dk, dwq, dwk, None, None, None, None, None


def _rotary_bwd(q, k, pos, freq, axis, wq, wk, gq, gk, dq, dk, eps, norm):
    """dq and dk written; the weights' gradients in their dtype."""
    T, Hq, D = gq.shape
    dwq = _empty((D,), gq, torch.float32) if norm and wq is not None else None
    dwk = _empty((D,), gk, torch.float32) if norm and wk is not None else None
    ws = None
    if norm:
        ws = _workspace(hx.hexrotary_bwd_workspace(T, Hq, gk.shape[1], D, hx._dtype_code(gq)), gq)
    hx.hexrotary_bwd(q, k, pos, freq, axis, wq, wk, gq, gk, dq, dk, dwq, dwk, ws, eps=eps,
                     norm=norm)
    return (None if dwq is None else dwq.to(wq.dtype), None if dwk is None else dwk.to(wk.dtype))


class HexAttentionFunction(torch.autograd.Function):
    """Softmax attention over packed sequences (hexattn_fwd)."""

    @staticmethod
    def forward(ctx, q, k, v, q_start, k_start, scale, causal):
        o, lse = _attention_outputs(q)
        hx.hexattn_fwd(q, k, v, o, lse, q_start, k_start, scale=scale, causal=causal)
        ctx.save_for_backward(q, k, v, o, lse, q_start, k_start)
        ctx.scale, ctx.causal = scale, causal
        return o

    @staticmethod
    def backward(ctx, g):
        q, k, v, o, lse, q_start, k_start = ctx.saved_tensors
        dq, dk, dv = (torch.zeros(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
        _attention_bwd(q, k, v, o, lse, g.contiguous(), dq, dk, dv, q_start, k_start, ctx.scale,
                       ctx.causal)
        return dq, dk, dv, None, None, None, None


def _attention_outputs(q):
    """o and lse as rows of no sequence have them: zeros, and no gradient."""
    return (torch.zeros(q.shape, dtype=q.dtype, device=q.device),
            torch.full(q.shape[:2], -math.inf, dtype=torch.float32, device=q.device))


def _attention_bwd(q, k, v, o, lse, g, dq, dk, dv, q_start, k_start, scale, causal):
    Tq, Hq, D = q.shape
    Tk, Hkv = k.shape[:2]
    ws = _workspace(hx.hexattn_bwd_workspace(Tq, Tk, q_start.shape[0] - 1, Hq, Hkv, D,
                                             hx._dtype_code(q)), q)
    hx.hexattn_bwd(q, k, v, o, lse, g, dq, dk, dv, ws, q_start, k_start, scale=scale,
                   causal=causal)


class HexPixelAttentionFunction(torch.autograd.Function):
    """Norm, rotation and attention of one projection's queries, keys and
    values, qkv [T][Hq + 2 Hkv][D]: the gradients are written into one tensor
    of that layout, with no copies between the parts."""

    @staticmethod
    def forward(ctx, qkv, wq, wk, pos, freq, axis, start, heads, eps, causal):
        Hq, Hkv = heads
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        qo, ko = _empty(q.shape, q), _empty(k.shape, k)
        hx.hexrotary_fwd(q, k, pos, freq, axis, wq, wk, qo, ko, eps=eps)
        o, lse = _attention_outputs(q)
        hx.hexattn_fwd(qo, ko, v, o, lse, start, causal=causal)
        ctx.save_for_backward(qkv, wq, wk, pos, freq, axis, start, qo, ko, o, lse)
        ctx.heads, ctx.eps, ctx.causal = heads, eps, causal
        return o

    @staticmethod
    def backward(ctx, g):
        qkv, wq, wk, pos, freq, axis, start, qo, ko, o, lse = ctx.saved_tensors
        Hq, Hkv = ctx.heads
        parts = lambda t: (t[:, :Hq], t[:, Hq:Hq + Hkv], t[:, Hq + Hkv:])  # noqa: E731
        d = torch.zeros_like(qkv)
        (q, k, v), (dq, dk, dv) = parts(qkv), parts(d)
        gq, gk = torch.zeros_like(qo), torch.zeros_like(ko)
        _attention_bwd(qo, ko, v, o, lse, g.contiguous(), gq, gk, dv, start, start, None,
                       ctx.causal)
        dwq, dwk = _rotary_bwd(q, k, pos, freq, axis, wq, wk, gq, gk, dq, dk, ctx.eps, True)
        return d, dwq, dwk, None, None, None, None, None, None, None


class HexDropoutFunction(torch.autograd.Function):
    """Dropout with a residual (hexdropout); the backward makes the mask again
    from the generator's words as they were."""

    @staticmethod
    def forward(ctx, x, residual, p, rng, call):
        x = x.contiguous()
        y = _empty(x.shape, x)
        hx.hexdropout(x, None if residual is None else residual.contiguous(), y, p, rng, call)
        ctx.save_for_backward(rng)
        ctx.p, ctx.call = p, call
        return y

    @staticmethod
    def backward(ctx, g):
        (rng,) = ctx.saved_tensors
        dx = None
        if ctx.needs_input_grad[0]:
            g = g.contiguous()
            dx = _empty(g.shape, g)
            hx.hexdropout(g, None, dx, ctx.p, rng, ctx.call)
        return dx, g if ctx.needs_input_grad[1] else None, None, None, None


def hex_rotary(q, k, pos, freq, axis, wq=None, wk=None, eps=1e-6, norm=True):
    """Query heads q [T][Hq][D] and key heads k [T][Hkv][D], normed (weights
    wq and wk [D], or ones) and turned by their positions pos [T][axes].
    Positions and frequencies take no gradient."""
    return HexRotaryFunction.apply(q, k, wq, wk, pos, freq, axis, float(eps), bool(norm))


def hex_attention(q, k, v, q_start, k_start=None, scale=None, causal=False):
    """Softmax attention of packed sequences, q [Tq][Hq][D] over k and v
    [Tk][Hkv][D], offsets int32 [S + 1] (k_start: q_start by default)."""
    return HexAttentionFunction.apply(q, k, v, q_start, q_start if k_start is None else k_start,
                                      scale, bool(causal))


def hex_dropout(x, p, rng, residual=None, call=0):
    """residual + dropout of x with probability p.  rng: int64 [2] on the
    device, seed and call number; the same words (and call) give the same
    mask.  It must keep its values until the backward."""
    return HexDropoutFunction.apply(x, residual, float(p), rng, int(call))


class HexCache:
    """Keys and values of S streams, `capacity` tokens each, for
    HexPixelAttention.prefill and .step."""

    def __init__(self, streams, capacity, kv_heads, head_dim, device=None, dtype=None):
        shape = (int(streams) * int(capacity), int(kv_heads), int(head_dim))
        self.k = torch.empty(shape, device=device, dtype=dtype)
        self.v = torch.empty(shape, device=device, dtype=dtype)
        self.capacity = int(capacity)
        self.start = (torch.arange(int(streams), device=device) * self.capacity).to(torch.int32)
        self.length = torch.zeros(int(streams), dtype=torch.int32, device=device)
        # the host's count, no stream holds more: tokens of every stream, and
        # beside them of each, the largest
        self.count = (0, [0] * int(streams), 0)
        # what prefill's offsets are made of: `far` names no slot, whatever token
        # is added; a first and a last column; the starts with a sequence of no
        # key before and behind every stream
        none, far, last = torch.zeros_like(self.start), -(1 << 31), (1 << 31) - 1
        column = lambda *a: torch.tensor(a, dtype=torch.int32, device=device)[:, None]  # noqa: E731
        self.parts = (none + far, none, column(0, far, 0), column(last, far, 0))
        self.starts = nn.functional.pad(torch.stack([self.start, none], 1).view(-1), (1, 0))

    @property
    def most(self):
        """No stream holds more tokens, by the host's count."""
        return self.count[0] + self.count[2]

    @most.setter
    def most(self, n):
        self.count = (int(n), [0] * len(self.count[1]), 0)

    def reserve(self, n):
        """Room for n more tokens of every stream, or n[s] (a list or tuple) of
        stream s, by the host's count."""
        self.count = self.with_more(n)

    def with_more(self, n):
        """The count with so many tokens more, refused where they do not fit."""
        every, each, top = self.count
        if isinstance(n, (list, tuple)):
            if len(n) != len(each):
                raise ValueError("HexCache: %d numbers of tokens for %d streams"
                                 % (len(n), len(each)))
            each = [a + int(b) for a, b in zip(each, n)]
            top, least = max(each, default=0), min(n, default=0)
        else:
            every, least = every + int(n), n
        if least < 0:
            raise ValueError("HexCache: %d more tokens" % least)
        if every + top > self.capacity:
            raise ValueError("HexCache: %d tokens do not fit the capacity of %d"
                             % (every + top, self.capacity))
        return every, each, top


class HexPixelAttention(nn.Module):
    """Attention layer over packed sequences of lit pixels: projection to
    heads, root-mean-square norm of every query and key head, rotation by
    positions of len(bases) axes, softmax attention (grouped heads), output
    projection, and with ``dropout`` the residual branch's dropout.  The
    projections are torch's linear layers.

    forward(x [T][dim], pos, start): x + dropout(projection(attention(x))),
    the mask by torch's generator of x's device (torch.manual_seed).
    prefill and step do the same over a HexCache, without dropout."""

    def __init__(self, dim, heads, kv_heads=None, head_dim=None, bases=(10000.0, 100.0, 100.0),
                 causal=False, dropout=0.0, eps=1e-6, device=None, dtype=None):
        super().__init__()
        self.heads = (int(heads), int(kv_heads or heads))
        self.head_dim = int(head_dim or dim // heads)
        self.causal, self.dropout, self.eps = bool(causal), float(dropout), float(eps)
        Hq, Hkv = self.heads
        kw = {"device": device, "dtype": dtype}
        self.qkv = nn.Linear(dim, (Hq + 2 * Hkv) * self.head_dim, bias=False, **kw)
        self.out = nn.Linear(Hq * self.head_dim, dim, bias=False, **kw)
        self.q_norm = nn.Parameter(torch.ones(self.head_dim, **kw))
        self.k_norm = nn.Parameter(torch.ones(self.head_dim, **kw))
        self.bases = tuple(bases)
        freq, axis = hex_frequencies(self.head_dim, self.bases, device)
        self.register_buffer("freq", freq, persistent=False)
        self.register_buffer("axis", axis, persistent=False)

    def _apply(self, fn, *args, **kw):
        # whatever type the layer gets, its frequencies stay float32 as they are
        freq, axis = self.freq, self.axis
        super()._apply(fn, *args, **kw)
        device = self.freq.device
        if freq.is_meta:
            freq, axis = hex_frequencies(self.head_dim, self.bases)
        self.freq, self.axis = freq.to(device), axis.to(device)
        return self

    def _load_from_state_dict(self, state_dict, prefix, *args):
        # states of before hold the dropout's words
        state_dict.pop(prefix + "rng", None)
        super()._load_from_state_dict(state_dict, prefix, *args)

    def _project(self, x):
        Hq, Hkv = self.heads
        return self.qkv(x).view(-1, Hq + 2 * Hkv, self.head_dim)

    def forward(self, x, pos, start):
        o = HexPixelAttentionFunction.apply(self._project(x), self.q_norm, self.k_norm, pos,
                                            self.freq, self.axis, start, self.heads, self.eps,
                                            self.causal)
        y = self.out(o.flatten(1))
        if not (self.training and self.dropout > 0):
            return x + y
        # both words from torch's generator of the device, as its own dropout
        # draws: who saves and restores that (activation checkpointing) gets the
        # same mask again, and a captured graph draws a new one in every replay
        rng = torch.empty(2, dtype=torch.int64, device=x.device).random_()
        return hex_dropout(y, self.dropout, rng, residual=x)

    def new_cache(self, streams, capacity):
        return HexCache(streams, capacity, self.heads[1], self.head_dim, self.qkv.weight.device,
                        self.qkv.weight.dtype)

    def _into_cache(self, qkv, pos, slot, cache):
        Hq, Hkv = self.heads
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        qo = _empty(q.shape, q)
        hx.hexrotary_fwd(q, k, pos, self.freq, self.axis, self.q_norm, self.k_norm, qo, cache.k,
                         eps=self.eps, v=v, vo=cache.v, slot=slot)
        return qo

    @torch.no_grad()
    def prefill(self, x, pos, start, cache, longest):
        """Packed prompts x [T][dim] of all streams, appended to their caches:
        of each at most ``longest`` tokens (``longest[s]``, where it is a list of
        one number for each stream), and what its stream has room for.
        A longer one is cut; the tokens past the cut, as those of no sequence,
        are not stored, see nothing, and pass as they are."""
        T, S = x.shape[0], cache.start.shape[0]
        if start.shape != (S + 1,):
            raise ValueError("HexPixelAttention: start has shape %s, expected (%d,)"
                             % (tuple(start.shape), S + 1))
        count = cache.with_more(longest)
        if S == 0:
            return x.clone()
        first = start.clamp(0, T)
        if isinstance(longest, (list, tuple)):
            longest = torch.tensor(longest, dtype=torch.int32).to(x.device)
        else:
            longest = int(longest)
        room = (cache.capacity - cache.length).clamp_(min=0).clamp_(max=longest)
        kept = torch.minimum(first.diff().clamp_(min=0), room)
        first = first[:-1]
        slots = cache.start + cache.length - first  # token t goes to slots + t
        length = cache.length + kept
        # The packed tokens as 2 S + 1 sequences: those before the first stream's,
        # every stream's kept ones, and the rest behind them, which see no key.
        # Rows: their offsets; their tokens' slots less the token, a column late,
        # as a search of the offsets counts those up to a token; their keys.
        far, none, left, right = cache.parts
        table = torch.stack([first, first + kept, far, slots, length, none])
        table = torch.cat([left, table.view(3, 2, S).transpose(1, 2).reshape(3, 2 * S), right], 1)
        q_start, slots, k_len = table.unbind()
        token = torch.arange(T, dtype=torch.int32, device=x.device)
        slot = slots[torch.searchsorted(q_start, token, right=True)] + token
        qo = self._into_cache(self._project(x), pos, slot, cache)
        cache.length.copy_(length)
        cache.count = count
        o = _empty(qo.shape, qo)
        hx.hexattn_fwd(qo, cache.k, cache.v, o, None, q_start, cache.starts, k_len[:-1],
                       causal=self.causal)
        return x + self.out(o.flatten(1))

    @torch.no_grad()
    def step(self, x, pos, cache):
        """n new tokens of every stream, x [S][n][dim] and pos [S][n][axes]:
        each sees its stream's tokens up to itself."""
        if not self.causal:
            raise ValueError("HexPixelAttention: steps need a causal layer")
        S, n = x.shape[:2]
        count = cache.with_more(n)
        at = cache.start + cache.length
        slot = (at[:, None] + torch.arange(n, dtype=torch.int32, device=x.device)).view(-1)
        qo = self._into_cache(self._project(x.flatten(0, 1)), pos.flatten(0, 1), slot, cache)
        cache.length += n
        cache.count = count
        most = cache.most
        q = qo.view(S, n, self.heads[0], self.head_dim)
        o = torch.empty_like(q)
        ws = _workspace(hx.hexattn_step_workspace(S, n, *self.heads, self.head_dim, most,
                                                  hx._dtype_code(q)), q)
        hx.hexattn_step(q, cache.k, cache.v, o, ws, cache.start, cache.length, most)
        return x + self.out(o.flatten(2))

    def extra_repr(self):
        return ("heads=%d, kv_heads=%d, head_dim=%d, causal=%s, dropout=%g"
                % (self.heads + (self.head_dim, self.causal, self.dropout)))
