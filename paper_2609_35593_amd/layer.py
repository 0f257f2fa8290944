"""Python binding of include/ress_layer.h: layer norm, rotary positions with several
axes, and attention over a sliding window of frames with sink tokens.

As in the package's other functions, a function carries its C entry point's name,
checks tensor metadata, allocates outputs (and workspaces) with torch when the caller
passes none, and passes pointers and the current stream of the tensors' device."""
from __future__ import annotations

import ctypes as C
import math
import struct

import torch

from . import RESS_OK, RessError, lib

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
# The current stream of a device as an address, without a Stream object around it where torch offers that.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _call(fn, device, stream, *args):
    """Calls an entry point on `stream` (default: the device's current one) with the tensors' device
    current, as the C ABI asks."""
    if stream is None:
        stream = _raw_stream(device.index)
    elif hasattr(stream, "cuda_stream"):
        stream = stream.cuda_stream
    if device.index == torch.cuda.current_device():
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
    """Address and bytes of the caller's workspace, or of one of torch's (marked as in use on a stream that is not its
    own), or none where the call needs none."""
    if workspace is None:
        n = _size(size, shape)
        if n == 0:
            return None, 0
        workspace = torch.empty(n, dtype=torch.uint8, device=device)
        if stream is not None:
            workspace.record_stream(_as_stream(stream, device))
    elif not (workspace.is_cuda and workspace.device == device and workspace.is_contiguous()):
        raise ValueError(f"workspace must be a contiguous tensor on {device}")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _as_stream(stream, device):
    return stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream), device=device)


def _empty(shape, dtype, device, stream):
    """An output, marked as in use on a stream that is not torch's current one."""
    t = torch.empty(shape, dtype=dtype, device=device)
    if stream is not None:
        t.record_stream(_as_stream(stream, device))
    return t


def _check(name, t, dtype, shape, device):
    """Metadata of a strided tensor whose last dimension is contiguous."""
    if not (t.dtype is dtype and t.shape == shape and t.device == device and (t.stride(-1) == 1 or t.shape[-1] <= 1)):
        raise ValueError(f"{name} must be a {dtype} tensor of shape {tuple(shape)} on {device} with contiguous channels")


def _check_dense(name, t, dtype, shape, device):
    if not (t.dtype is dtype and t.shape == shape and t.device == device and t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {device}")


def _device(name, t):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    return t.device


def _ptr(t):
    return None if t is None else t.data_ptr()


def _strides(name, t, dtype, shape, device):
    """The strides (heads, tokens) of a [heads][tokens][channels] tensor whose metadata must be these. (The stride of a
    dimension of one entry says nothing: torch may give any.)"""
    if t.dtype is dtype and t.shape == shape and t.device == device:
        head, token, channel = t.stride()
        if channel == 1 or shape[2] <= 1:
            return head if shape[0] > 1 else 0, token if shape[1] > 1 else 0
    raise ValueError(f"{name} must be a {dtype} tensor of shape {tuple(shape)} on {device} with contiguous channels")


# ---------------------------------------------------------------- layer norm


def _norm_view(name, t, like):
    """Rows, their stride and the type of [rows][width] with any row stride, or of a contiguous tensor of any rank; of
    `like`'s shape and device where that is given."""
    dtype = _DTYPES.get(t.dtype)
    if dtype is None or (like is not None and (t.shape != like.shape or t.device != like.device)):
        raise ValueError(f"{name} must be a bfloat16 or float32 CUDA tensor"
                         + ("" if like is None else f" of shape {tuple(like.shape)} on {like.device}"))
    if t.dim() == 2:
        rows, width = t.shape
        stride, channel = t.stride()
        if channel != 1 and width > 1:
            raise ValueError(f"{name}: a row's channels must be contiguous")
        return rows, stride if rows > 1 else width, dtype
    if t.dim() == 0 or not t.is_contiguous():
        raise ValueError(f"{name}: tensors of other ranks than [rows][width] must be contiguous")
    return (t.numel() // t.shape[-1] if t.shape[-1] else 0), t.shape[-1], dtype


def ress_layer_norm(x, gamma=None, beta=None, *, eps: float = 1e-5, out=None, out_dtype=torch.bfloat16, mean=None,
                    rstd=None, want_stats: bool = False, stream=None) -> dict:
    """Layer norm over the last dimension (see include/ress_layer.h). x: bfloat16 or float32, [rows][width]
    with any row stride, or contiguous of any rank; gamma, beta: float32 [width] or None; out: as x, of
    out_dtype when it is made here. Returns y and, with want_stats or given buffers, mean and rstd
    (float32, one per row) for ress_layer_norm_bwd."""
    dev = _device("x", x)
    rows, xs, xt = _norm_view("x", x, None)
    if out is None:
        out = _empty(x.shape, out_dtype, dev, stream)
    _, ys, yt = _norm_view("out", out, x)
    shape = _NORM(rows, x.shape[-1], xt, yt, xs, ys, eps)
    if want_stats and mean is None and rstd is None:
        mean, rstd = (_empty(x.shape[:-1], torch.float32, dev, stream) for _ in range(2))
    if gamma is not None:
        _check_dense("gamma", gamma, torch.float32, x.shape[-1:], dev)
    if beta is not None:
        _check_dense("beta", beta, torch.float32, x.shape[-1:], dev)
    if mean is not None:
        _check_dense("mean", mean, torch.float32, x.shape[:-1], dev)
    if rstd is not None:
        _check_dense("rstd", rstd, torch.float32, x.shape[:-1], dev)
    _call(lib.ress_layer_norm, dev, stream, shape, _ptr(x), _ptr(gamma), _ptr(beta), _ptr(out), _ptr(mean),
          _ptr(rstd))
    return dict(y=out, mean=mean, rstd=rstd)


def ress_layer_norm_bwd_workspace_size(rows: int, width: int) -> int:
    return _size("ress_layer_norm_bwd_workspace_size",
                 _NORM(rows, width, DTYPE_BF16, DTYPE_BF16, width, width, 1.0))


def ress_layer_norm_bwd(dy, x, gamma, mean, rstd, *, dx=None, dgamma=None, dbeta=None, want_weights: bool = True,
                        workspace=None, stream=None) -> dict:
    """Gradients of ress_layer_norm (see include/ress_layer.h). dy: of y's type; x, mean, rstd: as given to
    and made by the forward pass. Returns dx (of x's type) and, with want_weights, dgamma and dbeta
    (float32 [width])."""
    dev = _device("x", x)
    rows, xs, xt = _norm_view("x", x, None)
    _, ys, yt = _norm_view("dy", dy, x)
    width = x.shape[-1]
    if dx is None:
        dx = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=dev)
        if stream is not None:
            dx.record_stream(_as_stream(stream, dev))
    if _norm_view("dx", dx, x)[1:] != (xs, xt):
        raise ValueError("dx must have x's type and row stride")
    shape = _NORM(rows, width, xt, yt, xs, ys, 1.0)
    for name, t in (("mean", mean), ("rstd", rstd)):
        _check_dense(name, t, torch.float32, x.shape[:-1], dev)
    if gamma is not None:
        _check_dense("gamma", gamma, torch.float32, (width,), dev)
    if want_weights:
        dgamma = _empty(width, torch.float32, dev, stream) if dgamma is None else dgamma
        dbeta = _empty(width, torch.float32, dev, stream) if dbeta is None else dbeta
    for name, t in (("dgamma", dgamma), ("dbeta", dbeta)):
        if t is not None:
            _check_dense(name, t, torch.float32, (width,), dev)
    ws, ws_bytes = None, 0
    if dgamma is not None or dbeta is not None:
        ws, ws_bytes = _workspace(workspace, "ress_layer_norm_bwd_workspace_size", shape, dev, stream)
    _call(lib.ress_layer_norm_bwd, dev, stream, shape, _ptr(dy), _ptr(x), _ptr(gamma), _ptr(mean), _ptr(rstd),
          _ptr(dx), _ptr(dgamma), _ptr(dbeta), ws, ws_bytes)
    return dict(dx=dx, dgamma=dgamma, dbeta=dbeta)


# --------------------------------------------------------- rotary positions


def ress_rope(q, k, pos, *, dims, layout: str = "split", base: float = 100.0, inverse: bool = False, q_out=None,
              k_out=None, stream=None) -> dict:
    """Rotary positions of q [H][N][D] and k [H_kv][N][D] (either may be None; any strides with contiguous
    channels) by pos int32 [N][axes] (see include/ress_layer.h). dims: channels of each axis; layout: "split",
    "interleaved" or "sections"; inverse: turn back (the pass of the gradients). Outputs may be the inputs (in
    place). Returns q and k."""
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
    _check_dense("pos", pos, torch.int32, (N, axes), dev)
    H = H_kv = 0
    qs = ks = qo = ko = (0, 0)
    if q is not None:
        H = q.shape[0]
        qs = _strides("q", q, first.dtype, (H, N, D), dev)
        q_out = _empty(q.shape, q.dtype, dev, stream) if q_out is None else q_out
        qo = _strides("q_out", q_out, q.dtype, q.shape, dev)
    else:
        q_out = None
    if k is not None:
        H_kv = k.shape[0]
        ks = _strides("k", k, first.dtype, (H_kv, N, D), dev)
        k_out = _empty(k.shape, k.dtype, dev, stream) if k_out is None else k_out
        ko = _strides("k_out", k_out, k.dtype, k.shape, dev)
    else:
        k_out = None
    shape = _ROPE(H, H_kv, N, D, axes, *dims, *(0,) * (4 - axes), ROPE_LAYOUTS[layout], bool(inverse), _DTYPES[first.dtype],
                  base, *qs, *ks, *qo, *ko)
    _call(lib.ress_rope, dev, stream, shape, _ptr(pos), _ptr(q), _ptr(k), _ptr(q_out), _ptr(k_out))
    return dict(q=q_out, k=k_out)


# -------------------------------------------- sliding window with sink tokens


def _int32(n):
    """Windows, frames and sink counts beyond every position act alike: the largest int stands for them."""
    return n if n < 2147483647 else 2147483647


def _window_shape(H, H_kv, n_q, n_k, D, q_offset, frame, window, n_sink, causal, strides=(0,) * 8):
    return _WINDOW(H, H_kv, n_q, n_k, D, q_offset, _int32(frame), _int32(window), _int32(n_sink), bool(causal), *strides)


def _qkv_strides(q, k, v):
    dev = _device("q", q)
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("q, k and v must be [heads][tokens][channels]")
    return dev, (_strides("q", q, torch.bfloat16, q.shape, dev)
                 + _strides("k", k, torch.bfloat16, (k.shape[0], k.shape[1], q.shape[2]), dev)
                 + _strides("v", v, torch.bfloat16, k.shape, dev))


def ress_window_attn(q, k, v, *, window: int, frame: int = 1, n_sink: int = 0, q_offset: int = 0, causal: bool = True,
                     scale: float | None = None, out=None, lse=None, want_lse: bool = False, workspace=None, stream=None) -> dict:
    """Attention over a sliding window of frames and the first n_sink tokens (see include/ress_layer.h). q: bf16
    [H][n_q][64] at positions q_offset ..; k, v: bf16 [H_kv][n_k][64]; any strides with contiguous channels.
    Returns o (bf16, as q) and, with want_lse or a given buffer, lse (float32 [H][n_q])."""
    dev, st = _qkv_strides(q, k, v)
    H, n_q, D = q.shape
    if out is None:
        out = _empty(q.shape, torch.bfloat16, dev, stream)
    st += _strides("out", out, torch.bfloat16, q.shape, dev)
    if lse is None and want_lse:
        lse = _empty((H, n_q), torch.float32, dev, stream)
    if lse is not None:
        _check_dense("lse", lse, torch.float32, (H, n_q), dev)
    shape = _window_shape(H, k.shape[0], n_q, k.shape[1], D, q_offset, frame, window, n_sink, causal, st)
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    ws, ws_bytes = _workspace(workspace, "ress_window_attn_workspace_size", shape, dev, stream)
    _call(lib.ress_window_attn, dev, stream, shape, _ptr(q), _ptr(k), _ptr(v), float(scale), _ptr(out), _ptr(lse), ws,
          ws_bytes)
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
    dev, st = _qkv_strides(q, k, v)
    H, n_q, D = q.shape
    st += _strides("o", o, torch.bfloat16, q.shape, dev)
    gst = _strides("d_o", d_o, torch.bfloat16, q.shape, dev)
    _check_dense("lse", lse, torch.float32, (H, n_q), dev)
    grads = []
    for name, t, like in (("dq", dq, q), ("dk", dk, k), ("dv", dv, v)):
        t = _empty(like.shape, torch.bfloat16, dev, stream) if t is None else t
        gst += _strides(name, t, torch.bfloat16, like.shape, dev)
        grads.append(t)
    dq, dk, dv = grads
    shape = _window_shape(H, k.shape[0], n_q, k.shape[1], D, q_offset, frame, window, n_sink, causal, st)
    g = _GRADS(*gst)
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    ws, ws_bytes = _workspace(workspace, "ress_window_attn_bwd_workspace_size", shape, dev, stream)
    _call(lib.ress_window_attn_bwd, dev, stream, shape, g, _ptr(d_o), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse),
          float(scale), _ptr(dq), _ptr(dk), _ptr(dv), ws, ws_bytes)
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
    if q.dim() != 3 or k.dim() != 4 or v.dim() != 4:
        raise ValueError("q must be [B][H][64], k and v [B][H_kv][capacity][64]")
    dev, (B, H, D) = _device("q", q), q.shape
    _, H_kv, capacity, _ = k.shape
    _check("q", q, torch.bfloat16, q.shape, dev)
    _check("k", k, torch.bfloat16, (B, H_kv, capacity, D), dev)
    _check("v", v, torch.bfloat16, k.shape, dev)
    _check_dense("lens", lens, torch.int32, (B,), dev)
    if out is None:
        out = _empty(q.shape, torch.bfloat16, dev, stream)
    _check("out", out, torch.bfloat16, q.shape, dev)
    q_b, q_h, _ = q.stride()
    k_b, k_h, k_t, _ = k.stride()
    v_b, v_h, v_t, _ = v.stride()
    o_b, o_h, _ = out.stride()
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
    ws, ws_bytes = _workspace(workspace, "ress_window_attn_decode_workspace_size", shape, dev, stream)
    _call(lib.ress_window_attn_decode, dev, stream, shape, _ptr(q), _ptr(k), _ptr(v), _ptr(lens), float(scale), _ptr(out), ws,
          ws_bytes)
    return out
