"""Python binding of libhexconv (include/hexconv.h).

Argument marshalling only: every function has the name of the C entry point
it calls, takes torch tensors for device buffers (torch supplies device
memory and the current HIP stream), checks dtypes/shapes/contiguity, and
raises HexError when the library returns a non-zero status.  All arithmetic
happens in the HIP kernels of libhexconv.so; there is no fallback.  If the
shared library has not been built, loading fails with an error.
"""
from __future__ import annotations

import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libhexconv.so")

HEX_OK = 0
HEX_ERR_INVALID_ARG = -1
HEX_ERR_UNSUPPORTED = -2
HEX_ERR_LAUNCH = -3
HEX_F32 = 0
HEX_BF16 = 1
HEX_POOL_MAX = 0
HEX_POOL_AVG = 1
HEX_FLAG_RELU = 1
HEX_MAX_K = 8
HEX_MAX_STRIDE = 8
HEX_MAX_KZ = 4
HEX_ATTN_CAUSAL = 1
HEX_ROTARY_NORM = 1
HEX_ATTN_MAX_DIM = 128
HEX_ROTARY_MAX_AXES = 8
HEX_NORM_MAX_DIM = 16384
HEX_LINEAR_MAX_DIM = 1 << 20
HEX_ACT_NONE = 0
HEX_ACT_RELU = 1
HEX_ACT_GELU = 2
HEX_ACT_SILU = 3

# (name, argtypes, restype) of every exported symbol
_P = ctypes.c_void_p
_I = ctypes.c_int
_IP = ctypes.POINTER(ctypes.c_int)
_S = ctypes.c_size_t
_L = ctypes.c_int64
_F = ctypes.c_float
SIGNATURES = {
    "hex_num_taps": ([_I], _I),
    "hex_out_shape": ([_I, _I, _I, _I, _IP, _IP], _I),
    "hex_tap_table": ([_I, _I, _IP, _IP], _I),
    "hexconv_fwd": ([_P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _I, _I, _P], _I),
    "hexconv_bwd_data": ([_P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _I, _P], _I),
    "hexconv_bwd_weight_workspace": ([_I, _I, _I, _I, _I, _I, _I, _I], _S),
    "hexconv_bwd_weight": ([_P, _P, _P, _P, _P, _S, _I, _I, _I, _I, _I, _I, _I,
                            _I, _P], _I),
    "hexconv_bwd_workspace": ([_I, _I, _I, _I, _I, _I, _I, _I], _S),
    "hexconv_bwd": ([_P, _P, _P, _P, _P, _P, _P, _S, _I, _I, _I, _I, _I, _I, _I,
                     _I, _P], _I),
    "hexconv_bwd_noalloc": ([_P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _I, _P],
                            _I),
    "hexpool_fwd": ([_P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _I, _P], _I),
    "hexpool_bwd": ([_P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _I, _P], _I),
    "hex_status_string": ([_I], ctypes.c_char_p),
    "hex_last_launch_error": ([], ctypes.c_char_p),
    "hex_out_shape3d": ([_I] * 7 + [_IP, _IP, _IP], _I),
    "hexconv3d_fwd": ([_P, _P, _P, _P] + [_I] * 12 + [_P], _I),
    "hexconv3d_bwd_data": ([_P, _P, _P] + [_I] * 11 + [_P], _I),
    "hexconv3d_bwd_weight_workspace": ([_I] * 11, _S),
    "hexconv3d_bwd_weight": ([_P, _P, _P, _P, _P, _S] + [_I] * 11 + [_P], _I),
    "hexpool3d_fwd": ([_P, _P, _P] + [_I] * 11 + [_P], _I),
    "hexpool3d_bwd": ([_P, _P, _P, _P] + [_I] * 11 + [_P], _I),
    "hexrotary_fwd": ([_P] * 12 + [_I] * 5 + [_L] * 6 + [_I, _F, _I, _I, _P], _I),
    "hexrotary_bwd_workspace": ([_I] * 5, _S),
    "hexrotary_bwd": ([_P] * 14 + [_S] + [_I] * 5 + [_L] * 6 + [_F, _I, _I, _P], _I),
    "hexattn_fwd": ([_P] * 8 + [_I] * 6 + [_L] * 4 + [_F, _I, _I, _P], _I),
    "hexattn_bwd_workspace": ([_I] * 7, _S),
    "hexattn_bwd": ([_P] * 10 + [_S] + [_P] * 2 + [_I] * 6 + [_L] * 8 + [_F, _I, _I, _P], _I),
    "hexattn_step_workspace": ([_I] * 7, _S),
    "hexattn_step": ([_P] * 5 + [_S] + [_P] * 2 + [_I] * 7 + [_L] * 2 + [_F, _I, _P], _I),
    "hexdropout": ([_P] * 3 + [_L, ctypes.c_double, _P, ctypes.c_uint64, _I, _P], _I),
    "hexnorm_fwd": ([_P] * 6 + [_I] * 2 + [_L] * 2 + [_F, _I, _P], _I),
    "hexnorm_bwd_workspace": ([_I] * 3, _S),
    "hexnorm_bwd": ([_P] * 10 + [_S] + [_I] * 2 + [_L] * 4 + [_I, _P], _I),
    "hexlinear_fwd_workspace": ([_I] * 3 + [_L, _I], _S),
    "hexlinear_fwd": ([_P] * 7 + [_S] + [_I] * 3 + [_L] * 3 + [_I, _I, _P], _I),
    "hexlinear_bwd_workspace": ([_I] * 3 + [_L] * 2 + [_I] * 2, _S),
    "hexlinear_bwd": ([_P] * 8 + [_S] + [_I] * 3 + [_L] * 3 + [_I] * 3 + [_P], _I),
    "hexffn_width": ([_I], _I),
    "hexffn_fwd_workspace": ([_I] * 4 + [_L, _I], _S),
    "hexffn_fwd": ([_P] * 10 + [_S] + [_I] * 4 + [_L] * 3 + [_I, _I, _P], _I),
    "hexffn_bwd_workspace": ([_I] * 4 + [_L] * 2 + [_I], _S),
    "hexffn_bwd": ([_P] * 12 + [_S] + [_I] * 4 + [_L] * 3 + [_I] * 3 + [_P], _I),
    "hexconv_timing_begin": ([], _I),
    "hexconv_timing_end": ([_I, ctypes.c_char_p, _IP, ctypes.POINTER(ctypes.c_double), _IP],
                           _I),
}

HEX_TIMING_NAME_LEN = 64

_lib = None


class HexError(RuntimeError):
    def __init__(self, fn, status):
        self.status = status
        msg = "%s: %s" % (fn, status_string(status))
        if status == HEX_ERR_LAUNCH:
            msg += " (%s)" % load().hex_last_launch_error().decode()
        super().__init__(msg)


def load():
    """Load libhexconv.so (must have been built, e.g. by build.build()).

    torch is imported first.  torch ships its own HIP runtime (needed under
    the name libamdhip64.so), while libhexconv links the system one
    (libamdhip64.so.7); both then share the HSA runtime that was loaded
    first.  With libhexconv loaded before torch, torch's HIP runtime ends up
    on the system HSA runtime and the system HIP runtime, initialised after
    it, finds no device.  Loading torch's libraries first keeps the one
    order that works."""
    global _lib
    if _lib is None:
        import torch  # noqa: F401  (load order of the HIP runtimes, above)
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                "libhexconv.so not found at %s: build it first "
                "(python -m paper_1903_01814_amd.build)" % LIB_PATH)
        lib = ctypes.CDLL(LIB_PATH)
        for name, (args, res) in SIGNATURES.items():
            f = getattr(lib, name)
            f.argtypes = args
            f.restype = res
        _lib = lib
    return _lib


def status_string(status: int) -> str:
    return load().hex_status_string(status).decode()


def _ok(fn, rc):
    if rc != HEX_OK:
        raise HexError(fn, rc)


# ----------------------------------------------------------- host helpers

def hex_num_taps(k: int) -> int:
    rc = load().hex_num_taps(k)
    if rc < 0:
        raise HexError("hex_num_taps", rc)
    return rc


def hex_out_shape(H: int, W: int, k: int, stride: int):
    ho, wo = ctypes.c_int(), ctypes.c_int()
    _ok("hex_out_shape", load().hex_out_shape(H, W, k, stride, ctypes.byref(ho),
                                              ctypes.byref(wo)))
    return ho.value, wo.value


def hexconv_timing_begin():
    """Start bracketing every kernel launch with HIP events (eager use only,
    not while a HIP graph is being captured)."""
    _ok("hexconv_timing_begin", load().hexconv_timing_begin())


def hexconv_timing_end(max_kernels: int = 32):
    """Stop recording; {kernel name: (launches, summed GPU ms)} in order of
    first launch."""
    names = ctypes.create_string_buffer(max_kernels * HEX_TIMING_NAME_LEN)
    counts = (ctypes.c_int * max_kernels)()
    total = (ctypes.c_double * max_kernels)()
    n = ctypes.c_int()
    _ok("hexconv_timing_end", load().hexconv_timing_end(max_kernels, names, counts, total,
                                                        ctypes.byref(n)))
    out = {}
    for i in range(n.value):
        raw = names.raw[i * HEX_TIMING_NAME_LEN:(i + 1) * HEX_TIMING_NAME_LEN]
        out[raw.split(b"\0", 1)[0].decode()] = (counts[i], total[i])
    return out


def hex_tap_table(k: int, parity: int):
    """(dcol, drow) lists of the taps of a size-k kernel for a centre column
    of the given parity."""
    T = hex_num_taps(k)
    dcol = (ctypes.c_int * T)()
    drow = (ctypes.c_int * T)()
    _ok("hex_tap_table", load().hex_tap_table(k, parity, dcol, drow))
    return list(dcol), list(drow)


# --------------------------------------------------------- device entries

_torch_module = None


def _torch():
    # looked up once: the statement takes 0.1 us each time
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _dtype_code(t):
    torch, dtype = _torch(), t.dtype
    if dtype is torch.float32:
        return HEX_F32
    if dtype is torch.bfloat16:
        return HEX_BF16
    raise TypeError("hexconv: unsupported dtype %s" % dtype)


def _dev(t, name, dt=None, shape=None):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("hexconv: %s must be a device tensor" % name)
    if not t.is_contiguous():
        raise ValueError("hexconv: %s must be contiguous" % name)
    if dt is not None and _dtype_code(t) != dt:
        raise TypeError("hexconv: %s has dtype %s" % (name, t.dtype))
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError("hexconv: %s has shape %s, expected %s"
                         % (name, tuple(t.shape), tuple(shape)))
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        # the handle alone: making a Stream object of it takes 3 us a call
        torch = _torch()
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def hexconv_fwd(x, w, bias, y, k: int, stride: int = 1, relu: bool = False,
                stream=None):
    """y <- hexagonal convolution of x with w (+ bias) (Sec. 2.3)."""
    N, Ci, H, W = x.shape
    Co = w.shape[0]
    dt = _dtype_code(x)
    T = hex_num_taps(k)
    Ho, Wo = hex_out_shape(H, W, k, stride)
    rc = load().hexconv_fwd(
        _dev(x, "x", dt), _dev(w, "w", dt, (Co, Ci, T)),
        _dev(bias, "bias", dt, (Co,)), _dev(y, "y", dt, (N, Co, Ho, Wo)),
        N, Ci, Co, H, W, k, stride, dt, HEX_FLAG_RELU if relu else 0,
        _stream(stream))
    _ok("hexconv_fwd", rc)
    return y


def hexconv_bwd_data(dy, w, dx, k: int, stride: int = 1, stream=None):
    """dx <- gradient of the forward map with respect to its input."""
    N, Ci, H, W = dx.shape
    Co = w.shape[0]
    dt = _dtype_code(dx)
    T = hex_num_taps(k)
    Ho, Wo = hex_out_shape(H, W, k, stride)
    rc = load().hexconv_bwd_data(
        _dev(dy, "dy", dt, (N, Co, Ho, Wo)), _dev(w, "w", dt, (Co, Ci, T)),
        _dev(dx, "dx", dt), N, Ci, Co, H, W, k, stride, dt, _stream(stream))
    _ok("hexconv_bwd_data", rc)
    return dx


def hexconv_bwd_weight_workspace(N, C_in, C_out, H, W, k, stride, dt):
    return load().hexconv_bwd_weight_workspace(N, C_in, C_out, H, W, k, stride,
                                               dt)


def hexconv_bwd_weight(x, dy, dw, db, ws, k: int, stride: int = 1,
                       stream=None):
    """dw, db <- gradients with respect to weights and bias (fp32).  ws is a
    uint8 device tensor of at least hexconv_bwd_weight_workspace bytes (or
    None when that is 0)."""
    torch = _torch()
    N, Ci, H, W = x.shape
    Co = dw.shape[0]
    dt = _dtype_code(x)
    T = hex_num_taps(k)
    Ho, Wo = hex_out_shape(H, W, k, stride)
    if dw.dtype != torch.float32 or (db is not None and db.dtype != torch.float32):
        raise TypeError("hexconv: dw and db must be float32")
    ws_ptr = _dev(ws, "ws")
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    rc = load().hexconv_bwd_weight(
        _dev(x, "x", dt), _dev(dy, "dy", dt, (N, Co, Ho, Wo)),
        _dev(dw, "dw", None, (Co, Ci, T)), _dev(db, "db", None, (Co,)),
        ws_ptr, ws_bytes, N, Ci, Co, H, W, k, stride, dt, _stream(stream))
    _ok("hexconv_bwd_weight", rc)
    return dw, db


def hexconv_bwd_workspace(N, C_in, C_out, H, W, k, stride, dt):
    return load().hexconv_bwd_workspace(N, C_in, C_out, H, W, k, stride, dt)


def hexconv_bwd(x, dy, w, dx, dw, db, ws, k: int, stride: int = 1,
                stream=None):
    """dx (may be None), dw, db (may be None) <- both gradients of one layer
    in one call.  ws: uint8 device tensor of at least hexconv_bwd_workspace
    bytes (or None when that is 0)."""
    torch = _torch()
    N, Ci, H, W = x.shape
    Co = dw.shape[0]
    dt = _dtype_code(x)
    T = hex_num_taps(k)
    Ho, Wo = hex_out_shape(H, W, k, stride)
    if dw.dtype != torch.float32 or (db is not None and db.dtype != torch.float32):
        raise TypeError("hexconv: dw and db must be float32")
    ws_ptr = _dev(ws, "ws")
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    rc = load().hexconv_bwd(
        _dev(x, "x", dt), _dev(dy, "dy", dt, (N, Co, Ho, Wo)),
        _dev(w, "w", dt, (Co, Ci, T)), _dev(dx, "dx", dt, (N, Ci, H, W)),
        _dev(dw, "dw", None, (Co, Ci, T)), _dev(db, "db", None, (Co,)),
        ws_ptr, ws_bytes, N, Ci, Co, H, W, k, stride, dt, _stream(stream))
    _ok("hexconv_bwd", rc)
    return dx, dw, db


HEX_NOALLOC_SCRATCH_BYTES = 64 << 20


def hexconv_bwd_noalloc(x, dy, w, dx, dw, db, k: int, stride: int = 1, stream=None):
    """hexconv_bwd without a workspace: the library's static scratch array
    serves instead (no allocation in the call; overlapping calls on one GPU
    race)."""
    torch = _torch()
    N, Ci, H, W = x.shape
    Co = dw.shape[0]
    dt = _dtype_code(x)
    T = hex_num_taps(k)
    Ho, Wo = hex_out_shape(H, W, k, stride)
    if dw.dtype != torch.float32 or (db is not None and db.dtype != torch.float32):
        raise TypeError("hexconv: dw and db must be float32")
    rc = load().hexconv_bwd_noalloc(
        _dev(x, "x", dt), _dev(dy, "dy", dt, (N, Co, Ho, Wo)),
        _dev(w, "w", dt, (Co, Ci, T)), _dev(dx, "dx", dt, (N, Ci, H, W)),
        _dev(dw, "dw", None, (Co, Ci, T)), _dev(db, "db", None, (Co,)),
        N, Ci, Co, H, W, k, stride, dt, _stream(stream))
    _ok("hexconv_bwd_noalloc", rc)
    return dx, dw, db


def hexpool_fwd(x, y, argmax_tap, k: int, stride: int, mode: int,
                stream=None):
    """y <- hexagonal max (mode 0) or average (mode 1) pooling of x."""
    torch = _torch()
    N, C, H, W = x.shape
    dt = _dtype_code(x)
    Ho, Wo = hex_out_shape(H, W, k, stride)
    if argmax_tap is not None and argmax_tap.dtype != torch.uint8:
        raise TypeError("hexconv: argmax_tap must be uint8")
    rc = load().hexpool_fwd(
        _dev(x, "x", dt), _dev(y, "y", dt, (N, C, Ho, Wo)),
        _dev(argmax_tap, "argmax_tap", None, (N, C, Ho, Wo)),
        N, C, H, W, k, stride, mode, dt, _stream(stream))
    _ok("hexpool_fwd", rc)
    return y


def hexpool_bwd(dy, argmax_tap, relu_y, dx, k: int, stride: int, mode: int,
                stream=None):
    """dx <- pooling gradient (optionally masked by relu_y > 0)."""
    torch = _torch()
    N, C, H, W = dx.shape
    dt = _dtype_code(dx)
    Ho, Wo = hex_out_shape(H, W, k, stride)
    if argmax_tap is not None and argmax_tap.dtype != torch.uint8:
        raise TypeError("hexconv: argmax_tap must be uint8")
    rc = load().hexpool_bwd(
        _dev(dy, "dy", dt, (N, C, Ho, Wo)),
        _dev(argmax_tap, "argmax_tap", None, (N, C, Ho, Wo)),
        _dev(relu_y, "relu_y", dt, (N, C, H, W)), _dev(dx, "dx", dt),
        N, C, H, W, k, stride, mode, dt, _stream(stream))
    _ok("hexpool_bwd", rc)
    return dx


# ------------------------------------------------------- three dimensions
# x[N][C][D][H][W]; window of size (k, kz): the size-k hexagon times the
# planes dz = -kz .. kz; w[C_out][C_in][2kz+1][T]; plane stride stride_z.

def hex_out_shape3d(D: int, H: int, W: int, k: int, kz: int, stride: int, stride_z: int):
    do, ho, wo = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    _ok("hex_out_shape3d", load().hex_out_shape3d(D, H, W, k, kz, stride, stride_z,
                                                  ctypes.byref(do), ctypes.byref(ho),
                                                  ctypes.byref(wo)))
    return do.value, ho.value, wo.value


def hexconv3d_fwd(x, w, bias, y, k: int, kz: int, stride: int = 1, stride_z: int = 1,
                  relu: bool = False, stream=None):
    """y <- 3-D hexagonal convolution of x with w (+ bias) (Sec. 2.4)."""
    N, Ci, D, H, W = x.shape
    Co = w.shape[0]
    dt = _dtype_code(x)
    T = hex_num_taps(k)
    Do, Ho, Wo = hex_out_shape3d(D, H, W, k, kz, stride, stride_z)
    rc = load().hexconv3d_fwd(
        _dev(x, "x", dt), _dev(w, "w", dt, (Co, Ci, 2 * kz + 1, T)),
        _dev(bias, "bias", dt, (Co,)), _dev(y, "y", dt, (N, Co, Do, Ho, Wo)),
        N, Ci, Co, D, H, W, k, kz, stride, stride_z, dt, HEX_FLAG_RELU if relu else 0,
        _stream(stream))
    _ok("hexconv3d_fwd", rc)
    return y


def hexconv3d_bwd_data(dy, w, dx, k: int, kz: int, stride: int = 1, stride_z: int = 1,
                       stream=None):
    N, Ci, D, H, W = dx.shape
    Co = w.shape[0]
    dt = _dtype_code(dx)
    T = hex_num_taps(k)
    Do, Ho, Wo = hex_out_shape3d(D, H, W, k, kz, stride, stride_z)
    rc = load().hexconv3d_bwd_data(
        _dev(dy, "dy", dt, (N, Co, Do, Ho, Wo)), _dev(w, "w", dt, (Co, Ci, 2 * kz + 1, T)),
        _dev(dx, "dx", dt), N, Ci, Co, D, H, W, k, kz, stride, stride_z, dt, _stream(stream))
    _ok("hexconv3d_bwd_data", rc)
    return dx


def hexconv3d_bwd_weight_workspace(N, C_in, C_out, D, H, W, k, kz, stride, stride_z, dt):
    return load().hexconv3d_bwd_weight_workspace(N, C_in, C_out, D, H, W, k, kz, stride,
                                                 stride_z, dt)


def hexconv3d_bwd_weight(x, dy, dw, db, ws, k: int, kz: int, stride: int = 1,
                         stride_z: int = 1, stream=None):
    torch = _torch()
    N, Ci, D, H, W = x.shape
    Co = dw.shape[0]
    dt = _dtype_code(x)
    T = hex_num_taps(k)
    Do, Ho, Wo = hex_out_shape3d(D, H, W, k, kz, stride, stride_z)
    if dw.dtype != torch.float32 or (db is not None and db.dtype != torch.float32):
        raise TypeError("hexconv: dw and db must be float32")
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    rc = load().hexconv3d_bwd_weight(
        _dev(x, "x", dt), _dev(dy, "dy", dt, (N, Co, Do, Ho, Wo)),
        _dev(dw, "dw", None, (Co, Ci, 2 * kz + 1, T)), _dev(db, "db", None, (Co,)),
        _dev(ws, "ws"), ws_bytes, N, Ci, Co, D, H, W, k, kz, stride, stride_z, dt,
        _stream(stream))
    _ok("hexconv3d_bwd_weight", rc)
    return dw, db


def hexpool3d_fwd(x, y, argmax, k: int, kz: int, stride: int, stride_z: int, mode: int,
                  stream=None):
    """y <- 3-D max (mode 0) or average (mode 1) pooling; argmax: int16
    tensor (the uint16 tap indices, bit for bit) or None."""
    torch = _torch()
    N, C, D, H, W = x.shape
    dt = _dtype_code(x)
    Do, Ho, Wo = hex_out_shape3d(D, H, W, k, kz, stride, stride_z)
    if argmax is not None and argmax.dtype not in (torch.int16, torch.uint16):
        raise TypeError("hexconv: 3-D argmax must be a 16-bit tensor")
    rc = load().hexpool3d_fwd(
        _dev(x, "x", dt), _dev(y, "y", dt, (N, C, Do, Ho, Wo)),
        _dev(argmax, "argmax", None, (N, C, Do, Ho, Wo)),
        N, C, D, H, W, k, kz, stride, stride_z, mode, dt, _stream(stream))
    _ok("hexpool3d_fwd", rc)
    return y


def hexpool3d_bwd(dy, argmax, relu_y, dx, k: int, kz: int, stride: int, stride_z: int,
                  mode: int, stream=None):
    torch = _torch()
    N, C, D, H, W = dx.shape
    dt = _dtype_code(dx)
    Do, Ho, Wo = hex_out_shape3d(D, H, W, k, kz, stride, stride_z)
    if argmax is not None and argmax.dtype not in (torch.int16, torch.uint16):
        raise TypeError("hexconv: 3-D argmax must be a 16-bit tensor")
    rc = load().hexpool3d_bwd(
        _dev(dy, "dy", dt, (N, C, Do, Ho, Wo)),
        _dev(argmax, "argmax", None, (N, C, Do, Ho, Wo)),
        _dev(relu_y, "relu_y", dt, (N, C, D, H, W)), _dev(dx, "dx", dt),
        N, C, D, H, W, k, kz, stride, stride_z, mode, dt, _stream(stream))
    _ok("hexpool3d_bwd", rc)
    return dx


# --------------------------------------- attention over packed sequences

def _tokens(t, name, dtype, heads, D, n=None):
    """Pointer and token stride of [tokens][heads][D] with dense heads (n
    tokens, or any number)."""
    if t is None:
        return None, 0
    shape, stride = t.shape, t.stride()
    if (t.dtype is not dtype or not t.is_cuda or len(shape) != 3 or shape[1] != heads
            or shape[2] != D or (n is not None and shape[0] != n)):
        _refuse(t, name, dtype, ("n" if n is None else n, heads, D))
    if (stride[2] != 1 or stride[1] != D) and t.numel() and (
            (D > 1 and stride[2] != 1) or (heads > 1 and stride[1] != D)):
        raise ValueError("hexconv: the heads of %s must be dense" % name)
    # one token, or none: any stride does
    return t.data_ptr(), stride[0] if shape[0] > 1 else heads * D


def _array(t, name, dtype, shape):
    """Pointer of a contiguous device tensor; None passes through."""
    if t is None:
        return None
    if t.dtype is not dtype or not t.is_cuda or t.shape != shape or not t.is_contiguous():
        _refuse(t, name, dtype, shape)
    return t.data_ptr()


def _refuse(t, name, dtype, shape):
    if not t.is_cuda:
        raise ValueError("hexconv: %s must be a device tensor" % name)
    if t.dtype is not dtype:
        raise TypeError("hexconv: %s has dtype %s, expected %s" % (name, t.dtype, dtype))
    if len(t.shape) != len(shape) or any(w != "n" and w != g for w, g in zip(shape, t.shape)):
        raise ValueError("hexconv: %s has shape %s, expected %s" % (name, tuple(t.shape), shape))
    raise ValueError("hexconv: %s must be contiguous" % name)


def _ws(ws):
    return _dev(ws, "ws"), 0 if ws is None else ws.numel() * ws.element_size()


def hexrotary_fwd(q, k, pos, freq, axis, wq, wk, qo, ko, eps: float = 1e-6, norm: bool = True,
                  v=None, vo=None, slot=None, stream=None):
    """qo, ko <- norm and rotation of the heads of q [T][Hq][D] and k
    [T][Hkv][D] by positions pos [T][A]; with slot (int32 [T]) the keys, and
    with v and vo the values, go to those rows of ko and vo."""
    torch = _torch()
    T, Hq, D = q.shape
    Hkv, A = k.shape[1], pos.shape[1]
    dt, ty = _dtype_code(q), q.dtype
    n = T if slot is None else ko.shape[0]
    pq, ldq = _tokens(q, "q", ty, Hq, D)
    pk, ldk = _tokens(k, "k", ty, Hkv, D, T)
    pv, ldv = _tokens(v, "v", ty, Hkv, D, T)
    pqo, ldqo = _tokens(qo, "qo", ty, Hq, D, T)
    pko, ldko = _tokens(ko, "ko", ty, Hkv, D, n)
    pvo, ldvo = _tokens(vo, "vo", ty, Hkv, D, n)
    rc = load().hexrotary_fwd(
        pq, pk, pv, _array(pos, "pos", torch.float32, (T, A)),
        _array(freq, "freq", torch.float32, (D // 2,)),
        _array(axis, "axis", torch.int32, (D // 2,)), _array(wq, "wq", ty, (D,)),
        _array(wk, "wk", ty, (D,)), pqo, pko, pvo, _array(slot, "slot", torch.int32, (T,)), T, Hq,
        Hkv, D, A, ldq, ldk, ldv, ldqo, ldko, ldvo, n, eps, HEX_ROTARY_NORM if norm else 0, dt,
        _stream(stream))
    _ok("hexrotary_fwd", rc)
    return qo, ko


def hexrotary_bwd_workspace(T, Hq, Hkv, D, dt):
    return load().hexrotary_bwd_workspace(T, Hq, Hkv, D, dt)


def hexrotary_bwd(q, k, pos, freq, axis, wq, wk, dqo, dko, dq, dk, dwq, dwk, ws,
                  eps: float = 1e-6, norm: bool = True, stream=None):
    """dq, dk and the float32 dwq, dwk (each may be None) <- gradients of
    hexrotary_fwd.  Without the norm q and k may be None."""
    torch = _torch()
    T, Hq, D = dqo.shape
    Hkv, A = dko.shape[1], pos.shape[1]
    dt, ty = _dtype_code(dqo), dqo.dtype
    pq, ldq = _tokens(q, "q", ty, Hq, D, T)
    pk, ldk = _tokens(k, "k", ty, Hkv, D, T)
    pgq, ldgq = _tokens(dqo, "dqo", ty, Hq, D)
    pgk, ldgk = _tokens(dko, "dko", ty, Hkv, D, T)
    pdq, lddq = _tokens(dq, "dq", ty, Hq, D, T)
    pdk, lddk = _tokens(dk, "dk", ty, Hkv, D, T)
    rc = load().hexrotary_bwd(
        pq, pk, _array(pos, "pos", torch.float32, (T, A)),
        _array(freq, "freq", torch.float32, (D // 2,)),
        _array(axis, "axis", torch.int32, (D // 2,)), _array(wq, "wq", ty, (D,)),
        _array(wk, "wk", ty, (D,)), pgq, pgk, pdq, pdk, _array(dwq, "dwq", torch.float32, (D,)),
        _array(dwk, "dwk", torch.float32, (D,)), *_ws(ws), T, Hq, Hkv, D, A, ldq, ldk, ldgq, ldgk,
        lddq, lddk, eps, HEX_ROTARY_NORM if norm else 0, dt, _stream(stream))
    _ok("hexrotary_bwd", rc)
    return dq, dk, dwq, dwk


def _scale(scale, D):
    return D ** -0.5 if scale is None else scale


def hexattn_fwd(q, k, v, o, lse, q_start, k_start=None, k_len=None, scale=None,
                causal: bool = False, stream=None):
    """o, lse (float32 [Tq][Hq], may be None) <- attention of the packed
    queries q [Tq][Hq][D] over k and v [Tk][Hkv][D].  q_start: int32 [S+1];
    k_start: the same for the keys (None: q_start), or int32 [S] with k_len.
    scale: 1 / sqrt(D) by default."""
    Tq, Hq, D = q.shape
    Tk, Hkv, _ = k.shape
    dt = _dtype_code(q)
    S = q_start.shape[0] - 1
    if k_start is None:
        if k_len is not None:
            raise ValueError("hexconv: k_len needs k_start")
        k_start = q_start
    i32, ty = _torch().int32, q.dtype
    pq, ldq = _tokens(q, "q", ty, Hq, D)
    pk, ldk = _tokens(k, "k", ty, Hkv, D)
    pv, ldv = _tokens(v, "v", ty, Hkv, D, Tk)
    po, ldo = _tokens(o, "o", ty, Hq, D, Tq)
    rc = load().hexattn_fwd(
        pq, pk, pv, po, _array(lse, "lse", _torch().float32, (Tq, Hq)),
        _array(q_start, "q_start", i32, (S + 1,)),
        _array(k_start, "k_start", i32, (S + 1,) if k_len is None else (S,)),
        _array(k_len, "k_len", i32, (S,)), S, Tq, Tk, Hq, Hkv, D, ldq, ldk, ldv, ldo,
        _scale(scale, D), HEX_ATTN_CAUSAL if causal else 0, dt, _stream(stream))
    _ok("hexattn_fwd", rc)
    return o, lse


def hexattn_bwd_workspace(Tq, Tk, S, Hq, Hkv, D, dt):
    return load().hexattn_bwd_workspace(Tq, Tk, S, Hq, Hkv, D, dt)


def hexattn_bwd(q, k, v, o, lse, dout, dq, dk, dv, ws, q_start, k_start=None, scale=None,
                causal: bool = False, stream=None):
    """dq, dk, dv <- gradients of hexattn_fwd from dout, o and lse."""
    Tq, Hq, D = q.shape
    Tk, Hkv, _ = k.shape
    dt = _dtype_code(q)
    S = q_start.shape[0] - 1
    if k_start is None:
        k_start = q_start
    i32, ty = _torch().int32, q.dtype
    pq, ldq = _tokens(q, "q", ty, Hq, D)
    pk, ldk = _tokens(k, "k", ty, Hkv, D)
    pv, ldv = _tokens(v, "v", ty, Hkv, D, Tk)
    po, ldo = _tokens(o, "o", ty, Hq, D, Tq)
    pg, ldg = _tokens(dout, "dout", ty, Hq, D, Tq)
    pdq, lddq = _tokens(dq, "dq", ty, Hq, D, Tq)
    pdk, lddk = _tokens(dk, "dk", ty, Hkv, D, Tk)
    pdv, lddv = _tokens(dv, "dv", ty, Hkv, D, Tk)
    rc = load().hexattn_bwd(
        pq, pk, pv, po, _array(lse, "lse", _torch().float32, (Tq, Hq)), pg, pdq, pdk, pdv,
        *_ws(ws), _array(q_start, "q_start", i32, (S + 1,)),
        _array(k_start, "k_start", i32, (S + 1,)), S, Tq, Tk, Hq, Hkv, D, ldq, ldk, ldv, ldo, ldg,
        lddq, lddk, lddv, _scale(scale, D), HEX_ATTN_CAUSAL if causal else 0, dt,
        _stream(stream))
    _ok("hexattn_bwd", rc)
    return dq, dk, dv


def hexattn_step_workspace(S, n, Hq, Hkv, D, max_len, dt):
    return load().hexattn_step_workspace(S, n, Hq, Hkv, D, max_len, dt)


def hexattn_step(q, k, v, o, ws, k_start, k_len, max_len: int, scale=None, stream=None):
    """o <- attention of n new tokens of every sequence, q [S][n][Hq][D],
    over the k_len[s] cached tokens from k_start[s] on of k and v
    [Tk][Hkv][D], at most max_len each."""
    S, n, Hq, D = q.shape
    Tk, Hkv, _ = k.shape
    dt = _dtype_code(q)
    i32, ty = _torch().int32, q.dtype
    pk, ldk = _tokens(k, "k", ty, Hkv, D)
    pv, ldv = _tokens(v, "v", ty, Hkv, D, Tk)
    rc = load().hexattn_step(
        _array(q, "q", ty, (S, n, Hq, D)), pk, pv, _array(o, "o", ty, (S, n, Hq, D)), *_ws(ws),
        _array(k_start, "k_start", i32, (S,)), _array(k_len, "k_len", i32, (S,)), S, n, Hq, Hkv,
        D, Tk, max_len, ldk, ldv, _scale(scale, D), dt, _stream(stream))
    _ok("hexattn_step", rc)
    return o


def hexdropout(x, res, y, p: float, rng, call: int = 0, stream=None):
    """y <- res (may be None) + dropout of x with probability p; rng: int64
    device tensor [seed, call number]."""
    dt, ty, shape = _dtype_code(x), x.dtype, x.shape
    if rng.dtype is not _torch().int64:
        raise TypeError("hexconv: rng must be int64")
    rc = load().hexdropout(_array(x, "x", ty, shape), _array(res, "res", ty, shape),
                           _array(y, "y", ty, shape), x.numel(), p,
                           _array(rng, "rng", rng.dtype, (2,)), call, dt, _stream(stream))
    _ok("hexdropout", rc)
    return y


# --------------------------------------- operators on tokens by themselves

def _rows(t, name, dtype, n, cols):
    """Pointer and row stride of [n][cols] with dense rows; None passes through."""
    if t is None:
        return None, cols
    shape, stride = t.shape, t.stride()
    if t.dtype is not dtype or not t.is_cuda or shape != (n, cols):
        _refuse(t, name, dtype, (n, cols))
    if cols > 1 and stride[1] != 1 and n > 0:
        raise ValueError("hexconv: the rows of %s must be dense" % name)
    # one row, or none: any stride does
    return t.data_ptr(), stride[0] if n > 1 else cols


def _stream_on(stream, x, *others):
    """The stream of a call on x's device, which has to be the current one and
    that of every other tensor."""
    torch = _torch()
    d = x.get_device()
    # without torch.cuda.current_device's check for a device, 0.3 us a call
    if d != torch._C._cuda_getDevice():
        raise ValueError("hexconv: tensors on device %d, the current one is %d"
                         % (d, torch.cuda.current_device()))
    for t in others:
        if t is not None and t.get_device() != d:
            raise ValueError("hexconv: tensors on devices %d and %d" % (d, t.get_device()))
    return torch._C._cuda_getCurrentRawStream(d) if stream is None else _stream(stream)


def _grad_dtype(ty, grads):
    """The one type of the weights' gradients that are given, float32 or ty."""
    torch = _torch()
    got = [t.dtype for t in grads if t is not None] or [torch.float32]
    if any(t is not got[0] for t in got) or (got[0] is not torch.float32 and got[0] is not ty):
        raise TypeError("hexconv: the gradients of weights must be all float32 or all %s" % ty)
    return got[0]


def hexnorm_fwd(x, w, b, y, mean=None, rstd=None, eps: float = 1e-5, stream=None):
    """y (and mean, rstd, float32 [T]) <- layer norm of the rows of x [T][C],
    weights w and b [C] (each may be None)."""
    T, C = x.shape
    dt, ty, f32 = _dtype_code(x), x.dtype, _torch().float32
    px, ldx = _rows(x, "x", ty, T, C)
    py, ldy = _rows(y, "y", ty, T, C)
    rc = load().hexnorm_fwd(px, _array(w, "w", ty, (C,)), _array(b, "b", ty, (C,)), py,
                            _array(mean, "mean", f32, (T,)), _array(rstd, "rstd", f32, (T,)), T, C,
                            ldx, ldy, eps, dt, _stream_on(stream, x, w, b, y, mean, rstd))
    _ok("hexnorm_fwd", rc)
    return y


def hexnorm_bwd_workspace(T, C, dt):
    return load().hexnorm_bwd_workspace(T, C, dt)


def hexnorm_bwd(x, w, mean, rstd, dy, res, dx, dw, db, ws, stream=None):
    """dx and the float32 dw, db [C] (each may be None) <- gradients of
    hexnorm_fwd; res (may be None): added to dx."""
    T, C = x.shape
    dt, ty, f32 = _dtype_code(x), x.dtype, _torch().float32
    px, ldx = _rows(x, "x", ty, T, C)
    pg, ldg = _rows(dy, "dy", ty, T, C)
    pr, ldr = _rows(res, "res", ty, T, C)
    pd, ldd = _rows(dx, "dx", ty, T, C)
    rc = load().hexnorm_bwd(px, _array(w, "w", ty, (C,)), _array(mean, "mean", f32, (T,)),
                            _array(rstd, "rstd", f32, (T,)), pg, pr, pd,
                            _array(dw, "dw", f32, (C,)), _array(db, "db", f32, (C,)), *_ws(ws), T, C,
                            ldx, ldg, ldr, ldd, dt,
                            _stream_on(stream, x, w, mean, rstd, dy, res, dx, dw, db, ws))
    _ok("hexnorm_bwd", rc)
    return dx, dw, db


def hexlinear_fwd_workspace(M, N, K, ldx, dt):
    return load().hexlinear_fwd_workspace(M, N, K, ldx, dt)


def hexlinear_fwd(x, w, bias, res, y, z=None, ws=None, act: int = HEX_ACT_NONE, stream=None):
    """y <- act(z) + res with z = x w^T + bias, x [M][K] and w [N][K]; bias,
    res and z (which receives it) may be None."""
    M, K = x.shape
    N = w.shape[0]
    dt, ty = _dtype_code(x), x.dtype
    px, ldx = _rows(x, "x", ty, M, K)
    pr, ldr = _rows(res, "res", ty, M, N)
    py, ldy = _rows(y, "y", ty, M, N)
    rc = load().hexlinear_fwd(px, _array(w, "w", ty, (N, K)), _array(bias, "bias", ty, (N,)), pr,
                              py, _array(z, "z", ty, (M, N)), *_ws(ws), M, N, K, ldx, ldr, ldy, act,
                              dt, _stream_on(stream, x, w, bias, res, y, z, ws))
    _ok("hexlinear_fwd", rc)
    return y


def hexlinear_bwd_workspace(M, N, K, ldx, lddy, act, dt):
    return load().hexlinear_bwd_workspace(M, N, K, ldx, lddy, act, dt)


def hexlinear_bwd(x, w, z, dy, dx, dw, db, ws, act: int = HEX_ACT_NONE, stream=None):
    """dx, dw and db (each may be None; dw and db float32 or of x's type) <-
    gradients of hexlinear_fwd; z for an activation only."""
    M, K = x.shape
    N = dy.shape[1]
    dt, ty = _dtype_code(x), x.dtype
    gt = _grad_dtype(ty, (dw, db))
    px, ldx = _rows(x, "x", ty, M, K)
    pg, ldg = _rows(dy, "dy", ty, M, N)
    pd, ldd = _rows(dx, "dx", ty, M, K)
    rc = load().hexlinear_bwd(px, _array(w, "w", ty, (N, K)), _array(z, "z", ty, (M, N)), pg, pd,
                              _array(dw, "dw", gt, (N, K)), _array(db, "db", gt, (N,)), *_ws(ws), M,
                              N, K, ldx, ldg, ldd, act, dt if gt is ty else HEX_F32, dt,
                              _stream_on(stream, x, w, z, dy, dx, dw, db, ws))
    _ok("hexlinear_bwd", rc)
    return dx, dw, db


def hexffn_width(F: int) -> int:
    """Columns of h for F hidden features (gu has twice as many)."""
    rc = load().hexffn_width(F)
    if rc < 0:
        raise HexError("hexffn_width", rc)
    return rc


def hexffn_fwd_workspace(M, K, F, N, ldx, dt):
    return load().hexffn_fwd_workspace(M, K, F, N, ldx, dt)


def hexffn_fwd(x, w1, b1, w2, b2, res, y, gu, h, ws=None, act: int = HEX_ACT_SILU, stream=None):
    """y <- h w2^T + b2 + res, h = act(x w1[:F]^T + b1[:F]) (x w1[F:]^T + b1[F:]);
    x [M][K], w1 [2F][K], w2 [N][F]; b1, b2, res and gu may be None.  h
    [M][hexffn_width(F)] and gu [M][2 hexffn_width(F)] are for the backward."""
    M, K = x.shape
    N, F = w2.shape
    dt, ty, Fp = _dtype_code(x), x.dtype, hexffn_width(F)
    px, ldx = _rows(x, "x", ty, M, K)
    pr, ldr = _rows(res, "res", ty, M, N)
    py, ldy = _rows(y, "y", ty, M, N)
    rc = load().hexffn_fwd(px, _array(w1, "w1", ty, (2 * F, K)), _array(b1, "b1", ty, (2 * F,)),
                           _array(w2, "w2", ty, (N, F)), _array(b2, "b2", ty, (N,)), pr, py,
                           _array(gu, "gu", ty, (M, 2 * Fp)), _array(h, "h", ty, (M, Fp)), *_ws(ws),
                           M, K, F, N, ldx, ldr, ldy, act, dt,
                           _stream_on(stream, x, w1, b1, w2, b2, res, y, gu, h, ws))
    _ok("hexffn_fwd", rc)
    return y


def hexffn_bwd_workspace(M, K, F, N, ldx, lddy, dt):
    return load().hexffn_bwd_workspace(M, K, F, N, ldx, lddy, dt)


def hexffn_bwd(x, w1, w2, gu, h, dy, dx, dw1, db1, dw2, db2, ws, act: int = HEX_ACT_SILU,
               stream=None):
    """dx and the weights' gradients (each may be None; float32 or of x's
    type) <- gradients of hexffn_fwd."""
    M, K = x.shape
    N, F = w2.shape
    dt, ty, Fp = _dtype_code(x), x.dtype, hexffn_width(F)
    gt = _grad_dtype(ty, (dw1, db1, dw2, db2))
    px, ldx = _rows(x, "x", ty, M, K)
    pg, ldg = _rows(dy, "dy", ty, M, N)
    pd, ldd = _rows(dx, "dx", ty, M, K)
    rc = load().hexffn_bwd(px, _array(w1, "w1", ty, (2 * F, K)), _array(w2, "w2", ty, (N, F)),
                           _array(gu, "gu", ty, (M, 2 * Fp)), _array(h, "h", ty, (M, Fp)), pg, pd,
                           _array(dw1, "dw1", gt, (2 * F, K)), _array(db1, "db1", gt, (2 * F,)),
                           _array(dw2, "dw2", gt, (N, F)), _array(db2, "db2", gt, (N,)), *_ws(ws),
                           M, K, F, N, ldx, ldg, ldd, act, dt if gt is ty else HEX_F32, dt,
                           _stream_on(stream, x, w1, w2, gu, h, dy, dx, dw1, db1, dw2, db2, ws))
    _ok("hexffn_bwd", rc)
    return dx, dw1, db1, dw2, db2
