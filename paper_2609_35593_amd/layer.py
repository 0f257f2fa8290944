"""Python binding of include/ress_layer.h: layer norm, rotary positions with several
axes, and attention over a sliding window of frames with sink tokens.

As in the package's other functions, a function carries its C entry point's name,
checks tensor metadata, allocates outputs (and workspaces) with torch when the caller
passes none, and passes pointers and the current stream of the tensors' device, or the
caller's `stream` (a torch stream or an address; that its inputs are ready there, and its
outputs before they are used elsewhere, is the caller's to order). Nothing is recorded
for autograd: gradients are the calls ending in _bwd and the inverse of ress_rope."""
from __future__ import annotations

import ctypes as C
import math
import struct

import torch

from . import RESS_OK, RessError, lib
from .memory import empty, raw_stream

DTYPE_BF16, DTYPE_F32 = 0, 1
MAX_NORM_WIDTH = 16384
ROPE_LAYOUTS = {"split": 0, "interleaved": 1, "sections": 2}
_DTYPES = {torch.bfloat16: DTYPE_BF16, torch.float32: DTYPE_F32}


def _packer(fields):
    pack = struct.Struct(fields).pack

    def packed(*values):
        try:
            return pack(*values)
        except struct.error as e:
            raise ValueError(f"an argument is no number of its C type: {e}") from None

    return packed


# The shapes of ress_layer.h, packed as C lays them out (strides are pairs head, token). Packing takes a tenth of the
# time that filling in ctypes structures does, which shows in calls of a few microseconds.
_NORM = _packer("@q3i2qd")     # rows; width, x_dtype, y_dtype; x_stride, y_stride; eps
_ROPE = _packer("@12id8q")     # H, H_kv, N, D, n_axes, dims[4], layout, inverse, dtype; base; q, k, q_out, k_out
_WINDOW = _packer("@10i8q")    # H, H_kv, n_q, n_k, D, q_offset, frame, window, n_sink, causal; q, k, v, o
_GRADS = _packer("@8q")        # d_o, dq, dk, dv
_DECODE = _packer("@8i10q")    # B, H, H_kv, capacity, D, frame, window, n_sink; q_batch, q_head, k_batch, v_batch, k, v,
                               # o_batch, o_head


def _declare():
    vp, f, sz = C.c_void_p, C.c_float, C.c_size_t
    for name, args in (
            ("ress_layer_norm", [vp] * 8),
            ("ress_layer_norm_bwd_workspace_size", [vp, vp]),
            ("ress_layer_norm_bwd", [vp] * 10 + [sz, vp]),
            ("ress_rope", [vp] * 7),
            ("ress_window_attn_workspace_size", [vp, vp]),
            ("ress_window_attn", [vp] * 4 + [f, vp, vp, vp, sz, vp]),
            ("ress_window_attn_bwd_workspace_size", [vp, vp]),
            ("ress_window_attn_bwd", [vp] * 8 + [f] + [vp] * 4 + [sz, vp]),
            ("ress_window_attn_decode_workspace_size", [vp, vp]),
            ("ress_window_attn_decode", [vp] * 5 + [f, vp, vp, sz, vp])):
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = args, C.c_int


_declare()
# The current device, without a check, where torch offers that.
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _call(fn, device, stream, *args):
    """Calls an entry point on `stream` (default: the device's current one) with the tensors' device
    current, as the C ABI asks."""
    index = device.index
    if stream is None:
        stream = raw_stream(index)
    elif hasattr(stream, "cuda_stream"):
        stream = stream.cuda_stream
    if index == _current_device():
        st = fn(*args, stream)
    else:
        with torch.cuda.device(device):
            st = fn(*args, stream)
    if st != RESS_OK:
        raise RessError(st, fn.__name__)


def _size(name, shape) -> int:
    n = C.c_size_t(0)
    st = getattr(lib, name)(shape, C.byref(n))
    if st != RESS_OK:
        raise RessError(st, name)
    return n.value


def _workspace(workspace, size, shape, device, stream):
    """The caller's workspace, or one of torch's, or none where the call needs none; its address; its bytes. Callers hold
    the tensor until their kernels are enqueued: only then may torch give the block to another call."""
    if workspace is None:
        n = _size(size, shape)
        if n == 0:
            return None, None, 0
        workspace = empty(n, torch.uint8, device, stream, output=False)
    elif not (workspace.is_cuda and workspace.device == device and workspace.is_contiguous()):
        raise ValueError(f"workspace must be a contiguous tensor on {device}")
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _dense(name, t, dtype, shape, device):
    """Address of a contiguous tensor whose metadata must be these; of none without one."""
    if t is None:
        return None
    if t.dtype is dtype and t.shape == shape and t.device == device and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {device}")


def _device(name, t):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    return t.device


def _all_strides(name, t, dtype, shape, device):
    """The strides of a tensor whose metadata must be these and whose channels, the last dimension, must be contiguous."""
    st = t.stride()
    if t.dtype is dtype and t.shape == shape and t.device == device and (st[-1] == 1 or shape[-1] <= 1):
        return st
    raise ValueError(f"{name} must be a {dtype} tensor of shape {tuple(shape)} on {device} with contiguous channels")


def _strides(name, t, dtype, shape, device):
    """The strides (heads, tokens) of a [heads][tokens][channels] tensor. (The stride of a dimension of one entry says
    nothing: torch may give any.)"""
    head, token, _ = _all_strides(name, t, dtype, shape, device)
    return head if shape[0] > 1 else 0, token if shape[1] > 1 else 0


# ---------------------------------------------------------------- layer norm


def _norm_view(name, t, shape, device):
    """Rows, their stride and the type of [rows][width] with any row stride, or of a contiguous tensor of any rank."""
    dtype = _DTYPES.get(t.dtype)
    if dtype is None or t.shape != shape or t.device != device:
        raise ValueError(f"{name} must be a bfloat16 or float32 tensor of shape {tuple(shape)} on {device}")
    if len(shape) == 2:
        rows, width = shape
        stride, channel = t.stride()
        if channel != 1 and width > 1:
            raise ValueError(f"{name}: a row's channels must be contiguous")
        return rows, stride if rows > 1 else width, dtype
    if not shape or not t.is_contiguous():
        raise ValueError(f"{name}: tensors of other ranks than [rows][width] must be contiguous")
    return (t.numel() // shape[-1] if shape[-1] else 0), shape[-1], dtype


def ress_layer_norm(x, gamma=None, beta=None, *, eps: float = 1e-5, out=None, out_dtype=torch.bfloat16, mean=None,
                    rstd=None, want_stats: bool = False, stream=None) -> dict:
    """Layer norm over the last dimension (see include/ress_layer.h). x: bfloat16 or float32, [rows][width]
    with any row stride, or contiguous of any rank; gamma, beta: float32 [width] or None; out: as x, of
    out_dtype when it is made here. Returns y and, with want_stats or given buffers, mean and rstd
    (float32, one per row) for ress_layer_norm_bwd."""
    dev, dims = _device("x", x), x.shape
    rows, xs, xt = _norm_view("x", x, dims, dev)
    if out is None:
        out = empty(dims, out_dtype, dev, stream)
    _, ys, yt = _norm_view("out", out, dims, dev)
    width, each = dims[-1:], dims[:-1]
    if want_stats and mean is None and rstd is None:
        mean, rstd = (empty(each, torch.float32, dev, stream) for _ in range(2))
    _call(lib.ress_layer_norm, dev, stream, _NORM(rows, *width, xt, yt, xs, ys, eps), x.data_ptr(),
          _dense("gamma", gamma, torch.float32, width, dev), _dense("beta", beta, torch.float32, width, dev),
          out.data_ptr(), _dense("mean", mean, torch.float32, each, dev), _dense("rstd", rstd, torch.float32, each, dev))
    return dict(y=out, mean=mean, rstd=rstd)


def ress_layer_norm_bwd_workspace_size(rows: int, width: int) -> int:
    return _size("ress_layer_norm_bwd_workspace_size",
                 _NORM(rows, width, DTYPE_BF16, DTYPE_BF16, width, width, 1.0))


def ress_layer_norm_bwd(dy, x, gamma, mean, rstd, *, dx=None, dgamma=None, dbeta=None, want_weights: bool = True,
                        workspace=None, stream=None) -> dict:
    """Gradients of ress_layer_norm (see include/ress_layer.h). dy: of y's type; x, mean, rstd: as given to
    and made by the forward pass. Returns dx (of x's type and with its row stride; given, it may be a slice of
    a packed gradient) and, with want_weights, dgamma and dbeta (float32 [width])."""
    dev, dims = _device("x", x), x.shape
    rows, xs, xt = _norm_view("x", x, dims, dev)
    _, ys, yt = _norm_view("dy", dy, dims, dev)
    width, each = dims[-1:], dims[:-1]
    if dx is None:
        dx = empty(dims, x.dtype, dev, stream, x.stride())
    if _norm_view("dx", dx, dims, dev)[1:] != (xs, xt):
        raise ValueError("dx must have x's type and row stride")
    if mean is None or rstd is None:
        raise ValueError("mean and rstd must be given")
    if want_weights:
        dgamma = empty(width, torch.float32, dev, stream) if dgamma is None else dgamma
        dbeta = empty(width, torch.float32, dev, stream) if dbeta is None else dbeta
    shape = _NORM(rows, *width, xt, yt, xs, ys, 1.0)
    args = (dy.data_ptr(), x.data_ptr(), _dense("gamma", gamma, torch.float32, width, dev),
            _dense("mean", mean, torch.float32, each, dev), _dense("rstd", rstd, torch.float32, each, dev), dx.data_ptr(),
            _dense("dgamma", dgamma, torch.float32, width, dev), _dense("dbeta", dbeta, torch.float32, width, dev))
    ws, ws_bytes = None, 0
    if dgamma is not None or dbeta is not None:
        workspace, ws, ws_bytes = _workspace(workspace, "ress_layer_norm_bwd_workspace_size", shape, dev, stream)
    _call(lib.ress_layer_norm_bwd, dev, stream, shape, *args, ws, ws_bytes)
    return dict(dx=dx, dgamma=dgamma, dbeta=dbeta)


# --------------------------------------------------------- rotary positions


def ress_rope(q, k, pos, *, dims, layout: str = "split", base: float = 100.0, inverse: bool = False, q_out=None,
              k_out=None, stream=None) -> dict:
    """Rotary positions of q [H][N][D] and k [H_kv][N][D] (either may be None; any strides with contiguous
    channels) by pos int32 [N][axes] (see include/ress_layer.h). dims: channels of each axis; layout: "split",
    "interleaved" or "sections"; inverse: turn back (the pass of the gradients). Outputs may be the inputs (in
    place). Returns q and k. (ress_select of turned ones pools them itself: the state in ress_qkv_proj_pool's
    workspace is of those that it wrote.)"""
    first = q if q is not None else k
    if first is None:
        raise ValueError("one of q and k must be given")
    if layout not in ROPE_LAYOUTS:
        raise ValueError(f"layout must be one of {sorted(ROPE_LAYOUTS)}")
    if first.dtype not in _DTYPES or first.dim() != 3:
        raise ValueError("q and k must be bfloat16 or float32 tensors [heads][tokens][channels]")
    dev, (_, N, D) = _device("q and k", first), first.shape
    axes = len(dims)
    if not 1 <= axes <= 4:
        raise ValueError("one to four axes")
    if pos is None:
        raise ValueError("pos must be given")
    H = H_kv = 0
    qs = ks = qo = ko = (0, 0)
    q_in = k_in = q_to = k_to = None
    if q is not None:
        H = q.shape[0]
        qs = _strides("q", q, first.dtype, (H, N, D), dev)
        q_out = empty(q.shape, q.dtype, dev, stream) if q_out is None else q_out
        qo = _strides("q_out", q_out, first.dtype, (H, N, D), dev)
        q_in, q_to = q.data_ptr(), q_out.data_ptr()
    else:
        q_out = None
    if k is not None:
        H_kv = k.shape[0]
        ks = _strides("k", k, first.dtype, (H_kv, N, D), dev)
        k_out = empty(k.shape, k.dtype, dev, stream) if k_out is None else k_out
        ko = _strides("k_out", k_out, first.dtype, (H_kv, N, D), dev)
        k_in, k_to = k.data_ptr(), k_out.data_ptr()
    else:
        k_out = None
    shape = _ROPE(H, H_kv, N, D, axes, *dims, *(0,) * (4 - axes), ROPE_LAYOUTS[layout], bool(inverse), _DTYPES[first.dtype],
                  base, *qs, *ks, *qo, *ko)
    _call(lib.ress_rope, dev, stream, shape, _dense("pos", pos, torch.int32, (N, axes), dev), q_in, k_in, q_to, k_to)
    return dict(q=q_out, k=k_out)


# -------------------------------------------- sliding window with sink tokens


def _int32(n):
    """Windows, frames and sink counts beyond every position act alike: the largest int stands for them."""
    return n if n < 2147483647 else 2147483647


def _window_shape(H, H_kv, n_q, n_k, D, q_offset, frame, window, n_sink, causal, strides=(0,) * 8):
    return _WINDOW(H, H_kv, n_q, n_k, D, q_offset, _int32(frame), _int32(window), _int32(n_sink), bool(causal), *strides)


def _qkv_strides(q, k, v):
    dev, qn, kn = _device("q", q), q.shape, k.shape
    if len(qn) != 3 or len(kn) != 3 or qn[2] != kn[2]:
        raise ValueError("q, k and v must be [heads][tokens][channels]")
    return dev, qn, kn, (_strides("q", q, torch.bfloat16, qn, dev) + _strides("k", k, torch.bfloat16, kn, dev)
                         + _strides("v", v, torch.bfloat16, kn, dev))


def ress_window_attn(q, k, v, *, window: int, frame: int = 1, n_sink: int = 0, q_offset: int = 0, causal: bool = True,
                     scale: float | None = None, out=None, lse=None, want_lse: bool = False, workspace=None, stream=None) -> dict:
    """Attention over a sliding window of frames and the first n_sink tokens (see include/ress_layer.h). q: bf16
    [H][n_q][64] at positions q_offset ..; k, v: bf16 [H_kv][n_k][64]; any strides with contiguous channels.
    Returns o (bf16, as q) and, with want_lse or a given buffer, lse (float32 [H][n_q])."""
    dev, qn, kn, st = _qkv_strides(q, k, v)
    H, n_q, D = qn
    H_kv, n_k, _ = kn
    if out is None:
        out = empty(qn, torch.bfloat16, dev, stream)
    st += _strides("out", out, torch.bfloat16, qn, dev)
    if lse is None and want_lse:
        lse = empty((H, n_q), torch.float32, dev, stream)
    lse_to = _dense("lse", lse, torch.float32, (H, n_q), dev)
    shape = _window_shape(H, H_kv, n_q, n_k, D, q_offset, frame, window, n_sink, causal, st)
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    workspace, ws, ws_bytes = _workspace(workspace, "ress_window_attn_workspace_size", shape, dev, stream)
    _call(lib.ress_window_attn, dev, stream, shape, q.data_ptr(), k.data_ptr(), v.data_ptr(), float(scale), out.data_ptr(),
          lse_to, ws, ws_bytes)
    return dict(o=out, lse=lse)


def ress_window_attn_workspace_size(H: int, H_kv: int, n_q: int, n_k: int, *, window: int, frame: int = 1, n_sink: int = 0,
                                    q_offset: int = 0, causal: bool = True) -> int:
    return _size("ress_window_attn_workspace_size",
                 _window_shape(H, H_kv, n_q, n_k, 64, q_offset, frame, window, n_sink, causal))


def ress_window_attn_bwd_workspace_size(H: int, H_kv: int, n_q: int, n_k: int, *, window: int, frame: int = 1,
                                        n_sink: int = 0, q_offset: int = 0, causal: bool = True) -> int:
    return _size("ress_window_attn_bwd_workspace_size",
                 _window_shape(H, H_kv, n_q, n_k, 64, q_offset, frame, window, n_sink, causal))


def ress_window_attn_bwd(d_o, q, k, v, o, lse, *, window: int, frame: int = 1, n_sink: int = 0, q_offset: int = 0,
                         causal: bool = True, scale: float | None = None, dq=None, dk=None, dv=None, workspace=None,
                         stream=None) -> dict:
    """Gradients of ress_window_attn (see include/ress_layer.h): o and lse as it made them, the other arguments
    as it was given. Returns dq, dk, dv (bf16, as q, k, v)."""
    dev, qn, kn, st = _qkv_strides(q, k, v)
    H, n_q, D = qn
    H_kv, n_k, _ = kn
    st += _strides("o", o, torch.bfloat16, qn, dev)
    gst = _strides("d_o", d_o, torch.bfloat16, qn, dev)
    if lse is None:
        raise ValueError("lse must be given")
    grads = []
    for name, t, like in (("dq", dq, qn), ("dk", dk, kn), ("dv", dv, kn)):
        t = empty(like, torch.bfloat16, dev, stream) if t is None else t
        gst += _strides(name, t, torch.bfloat16, like, dev)
        grads.append(t)
    dq, dk, dv = grads
    shape = _window_shape(H, H_kv, n_q, n_k, D, q_offset, frame, window, n_sink, causal, st)
    g = _GRADS(*gst)
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    workspace, ws, ws_bytes = _workspace(workspace, "ress_window_attn_bwd_workspace_size", shape, dev, stream)
    _call(lib.ress_window_attn_bwd, dev, stream, shape, g, d_o.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(),
          o.data_ptr(), _dense("lse", lse, torch.float32, (H, n_q), dev), float(scale), dq.data_ptr(), dk.data_ptr(),
          dv.data_ptr(), ws, ws_bytes)
    return dict(dq=dq, dk=dk, dv=dv)


def ress_window_attn_decode_workspace_size(B: int, H: int, H_kv: int, capacity: int, *, window: int, frame: int = 1,
                                           n_sink: int = 0) -> int:
    return _size("ress_window_attn_decode_workspace_size",
                 _DECODE(B, H, H_kv, capacity, 64, _int32(frame), _int32(window), _int32(n_sink), *(0,) * 10))


def ress_window_attn_decode(q, k, v, lens, *, window: int, frame: int = 1, n_sink: int = 0, scale: float | None = None,
                            out=None, workspace=None, stream=None):
    """One new token per sequence over its cache (see include/ress_layer.h). q: bf16 [B][H][64]; k, v: bf16
    [B][H_kv][capacity][64], any strides with contiguous channels; lens: int32 [B] on the device, the new tokens
    counted. Returns o (bf16 [B][H][64])."""
    dev, qn, kn = _device("q", q), q.shape, k.shape
    if len(qn) != 3 or len(kn) != 4 or kn[0] != qn[0] or kn[3] != qn[2]:
        raise ValueError("q must be [B][H][64], k and v [B][H_kv][capacity][64]")
    B, H, D = qn
    _, H_kv, capacity, _ = kn
    q_b, q_h, _ = _all_strides("q", q, torch.bfloat16, qn, dev)
    k_b, k_h, k_t, _ = _all_strides("k", k, torch.bfloat16, kn, dev)
    v_b, v_h, v_t, _ = _all_strides("v", v, torch.bfloat16, kn, dev)
    if lens is None:
        raise ValueError("lens must be given")
    if out is None:
        out = empty(qn, torch.bfloat16, dev, stream)
    o_b, o_h, _ = _all_strides("out", out, torch.bfloat16, qn, dev)
    if B <= 1:  # (the stride of a dimension of one entry says nothing)
        q_b = k_b = v_b = o_b = 0
    if H <= 1:
        q_h = o_h = 0
    if H_kv <= 1:
        k_h = v_h = 0
    if capacity <= 1:
        k_t = v_t = 0
    shape = _DECODE(B, H, H_kv, capacity, D, _int32(frame), _int32(window), _int32(n_sink), q_b, q_h, k_b, v_b, k_h, k_t,
                    v_h, v_t, o_b, o_h)
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    workspace, ws, ws_bytes = _workspace(workspace, "ress_window_attn_decode_workspace_size", shape, dev, stream)
    _call(lib.ress_window_attn_decode, dev, stream, shape, q.data_ptr(), k.data_ptr(), v.data_ptr(),
          _dense("lens", lens, torch.int32, (B,), dev), float(scale), out.data_ptr(), ws, ws_bytes)
    return out
