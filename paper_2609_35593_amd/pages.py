"""Python binding of include/ress_pages.h: the norm of every head of Q and K with the rotary positions, a cache in
pages, and attention of new tokens over it.

As in the package's other functions, a function carries its C entry point's name, checks tensor metadata, allocates
outputs (and workspaces) with torch when the caller passes none, and passes pointers and the current stream of the
tensors' device, or the caller's `stream` (see layer.py). Nothing is recorded for autograd: the gradients of
ress_qk_norm_rope are ress_qk_norm_rope_bwd's."""
from __future__ import annotations

import ctypes as C
import math

import torch

from . import lib
from .layer import _DTYPES, ROPE_LAYOUTS, _call, _dense, _device, _int32, _packer, _size, _workspace
from .memory import empty

HEAD_NORMS = {"layer": 0, "rms": 1}
_BF16, _F32, _I32 = torch.bfloat16, torch.float32, torch.int32

# The shapes of ress_pages.h, packed as C lays them out.
_HEADS = _packer("@12id8qid0q")  # H, H_kv, N, D, n_axes, dims[4], layout, inverse, dtype; base; q, k, q_out, k_out; norm; eps
_CACHE = _packer("@2i8q")        # n_pages, page; k, v (page, head, token), v_in
_GRADS = _packer("@8q")          # dq_out, dk_out, dq, dk
_TABLE = _packer("@5iqi0q")      # B, N, page, n_pages, max_pages; table_stride; clear
_PAGED = _packer("@11i11q")      # B, N, H, H_kv, D, page, n_pages, max_pages, frame, window, n_sink; table_stride, q, o, k, v


def _declare():
    vp, f, sz = C.c_void_p, C.c_float, C.c_size_t
    for name, args in (
            ("ress_qk_norm_rope", [vp] * 11),
            ("ress_qk_norm_rope_pages", [vp] * 15),
            ("ress_qk_norm_rope_bwd_workspace_size", [vp, vp]),
            ("ress_qk_norm_rope_bwd", [vp] * 16 + [sz, vp]),
            ("ress_page_tables", [vp] * 13),
            ("ress_pages_release_workspace_size", [vp, vp]),
            ("ress_pages_release", [vp] * 8 + [sz, vp]),
            ("ress_paged_attn_workspace_size", [vp, vp]),
            ("ress_paged_attn", [vp] * 7 + [f, vp, vp, vp, sz, vp])):
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = args, C.c_int


_declare()


# (Metadata is read once a tensor, and no further than a call needs it: a check costs a tenth to a quarter of a
# microsecond, which shows in calls of a few.)


def _rows(name, t, dtype, H, N, D, dev):
    """Strides (heads, tokens) and the address of a [heads][tokens][channels] tensor whose metadata must be these. (The
    stride of a dimension of one entry says nothing: torch may give any.)"""
    if t is None:
        raise ValueError(f"{name} must be given")
    head, token, channel = t.stride()
    if t.dtype is not dtype or t.shape != (H, N, D) or t.device != dev or channel != 1:
        raise ValueError(f"{name} must be a {dtype} tensor of shape {(H, N, D)} on {dev} with contiguous channels")
    return head if H > 1 else 0, token if N > 1 else 0, t.data_ptr()


def _flat(name, t, dtype, n, dev):
    """Address of a contiguous tensor [n]; of none without one."""
    if t is None:
        return None
    if t.dtype is dtype and t.shape == (n,) and t.device == dev and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {(n,)} on {dev}")


def _ints(name, t, n, dev):
    """Address of an int32 tensor [n] that must be there."""
    if t is None:
        raise ValueError(f"{name} must be given")
    return _flat(name, t, _I32, n, dev)


# ----------------------------------------------------------- norm of heads


def _head_shape(H, H_kv, N, D, dims, layout, dtype, base, norm, eps, strides=(0,) * 8):
    axes = len(dims)
    if not 1 <= axes <= 4:
        raise ValueError("one to four axes")
    if layout not in ROPE_LAYOUTS:
        raise ValueError(f"layout must be one of {sorted(ROPE_LAYOUTS)}")
    if norm not in HEAD_NORMS:
        raise ValueError(f"norm must be one of {sorted(HEAD_NORMS)}")
    return _HEADS(H, H_kv, N, D, axes, *dims, *_NO_DIMS[axes], ROPE_LAYOUTS[layout], 0, dtype, base, *strides,
                  HEAD_NORMS[norm], eps)


_NO_DIMS = {n: (0,) * (4 - n) for n in range(5)}


def _first(q, k):
    """Of the tensor of q and k that is there: its type and that type's number, device, tokens, channels."""
    x = q if q is not None else k
    if x is None:
        raise ValueError("one of q and k must be given")
    dtype, shape = x.dtype, x.shape
    code = _DTYPES.get(dtype)
    if code is None or len(shape) != 3:
        raise ValueError("q and k must be bfloat16 or float32 tensors [heads][tokens][channels]")
    return dtype, code, _device("q and k", x), shape[1], shape[2]


def _pos(pos, N, dims, dev):
    if pos is None:
        raise ValueError("pos must be given")
    return _dense("pos", pos, _I32, (N, len(dims)), dev)


def ress_qk_norm_rope(q, k, pos, *, dims, norm: str = "layer", q_gamma=None, q_beta=None, k_gamma=None, k_beta=None,
                      eps: float = 1e-5, layout: str = "split", base: float = 100.0, q_out=None, k_out=None,
                      stream=None) -> dict:
    """Norm of every head of q [H][N][D] and k [H_kv][N][D] (either may be None; any strides with contiguous channels)
    and their turn by pos int32 [N][axes], in one pass (see include/ress_pages.h). norm: "layer" or "rms"; gamma, beta:
    float32 [D] or None; dims, layout, base: as for ress_rope. Outputs may be the inputs (in place). Returns q and k."""
    dtype, code, dev, N, D = _first(q, k)
    H = H_kv = qh = qt = kh = kt = qoh = qot = koh = kot = 0
    q_in = k_in = q_to = k_to = None
    if q is not None:
        H = q.shape[0]
        qh, qt, q_in = _rows("q", q, dtype, H, N, D, dev)
        if q_out is None:
            q_out = empty((H, N, D), dtype, dev, stream)
        qoh, qot, q_to = _rows("q_out", q_out, dtype, H, N, D, dev)
    else:
        q_out = None
    if k is not None:
        H_kv = k.shape[0]
        kh, kt, k_in = _rows("k", k, dtype, H_kv, N, D, dev)
        if k_out is None:
            k_out = empty((H_kv, N, D), dtype, dev, stream)
        koh, kot, k_to = _rows("k_out", k_out, dtype, H_kv, N, D, dev)
    else:
        k_out = None
    shape = _head_shape(H, H_kv, N, D, dims, layout, code, base, norm, eps, (qh, qt, kh, kt, qoh, qot, koh, kot))
    _call(lib.ress_qk_norm_rope, dev, stream, shape, _pos(pos, N, dims, dev), q_in, k_in,
          _flat("q_gamma", q_gamma, _F32, D, dev), _flat("q_beta", q_beta, _F32, D, dev),
          _flat("k_gamma", k_gamma, _F32, D, dev), _flat("k_beta", k_beta, _F32, D, dev), q_to, k_to)
    return dict(q=q_out, k=k_out)


def _paged(name, t, dtype, shape, dev):
    """Strides (pages, heads, tokens) and the address of [pages][heads][tokens][channels] with this metadata."""
    if t is None:
        raise ValueError(f"{name} must be given")
    page, head, token, channel = t.stride()
    if t.dtype is not dtype or t.shape != shape or t.device != dev or (channel != 1 and shape[3] > 1):
        raise ValueError(f"{name} must be a {dtype} tensor of shape {tuple(shape)} on {dev} with contiguous channels")
    n, H, size, _ = shape
    return page if n > 1 else 0, head if H > 1 else 0, token if size > 1 else 0, t.data_ptr()


def ress_qk_norm_rope_pages(q, k, v, pos, slots, k_pages, v_pages, *, dims, norm: str = "layer", q_gamma=None, q_beta=None,
                            k_gamma=None, k_beta=None, eps: float = 1e-5, layout: str = "split", base: float = 100.0,
                            q_out=None, stream=None) -> dict:
    """ress_qk_norm_rope with k written into k_pages and v [H_kv][N][D] copied into v_pages (both [n_pages][H_kv][page][D],
    any strides with contiguous channels), token t at slots[t] (int32 [N]; a token without a slot in the cache is left
    out). q may be None. Returns q, k_pages and v_pages."""
    if k is None or v is None or k_pages is None:
        raise ValueError("k, v and k_pages must be given")
    dtype, code, dev, N, D = _first(k, None)
    H, H_kv, pages = 0, k.shape[0], k_pages.shape
    if len(pages) != 4 or pages[1] != H_kv or pages[3] != D:
        raise ValueError("k_pages and v_pages must be [n_pages][H_kv][page][D]")
    qh = qt = qoh = qot = 0
    q_in = q_to = None
    if q is not None:
        H = q.shape[0]
        qh, qt, q_in = _rows("q", q, dtype, H, N, D, dev)
        if q_out is None:
            q_out = empty((H, N, D), dtype, dev, stream)
        qoh, qot, q_to = _rows("q_out", q_out, dtype, H, N, D, dev)
    else:
        q_out = None
    kh, kt, k_in = _rows("k", k, dtype, H_kv, N, D, dev)
    vh, vt, v_in = _rows("v", v, dtype, H_kv, N, D, dev)
    kps, kph, kpt, k_to = _paged("k_pages", k_pages, dtype, pages, dev)
    vps, vph, vpt, v_to = _paged("v_pages", v_pages, dtype, pages, dev)
    shape = _head_shape(H, H_kv, N, D, dims, layout, code, base, norm, eps, (qh, qt, kh, kt, qoh, qot, 0, 0))
    cache = _CACHE(pages[0], pages[2], kps, kph, kpt, vps, vph, vpt, vh, vt)
    _call(lib.ress_qk_norm_rope_pages, dev, stream, shape, cache, _pos(pos, N, dims, dev), _ints("slots", slots, N, dev), q_in,
          k_in, v_in, _flat("q_gamma", q_gamma, _F32, D, dev), _flat("q_beta", q_beta, _F32, D, dev),
          _flat("k_gamma", k_gamma, _F32, D, dev), _flat("k_beta", k_beta, _F32, D, dev), q_to, k_to, v_to)
    return dict(q=q_out, k_pages=k_pages, v_pages=v_pages)


def ress_qk_norm_rope_bwd_workspace_size(H: int, H_kv: int, N: int, D: int) -> int:
    return _size("ress_qk_norm_rope_bwd_workspace_size",
                 _head_shape(H, H_kv, N, D, (0,), "split", 0, 1.0, "layer", 1.0))


def ress_qk_norm_rope_bwd(dq_out, dk_out, q, k, pos, *, dims, norm: str = "layer", q_gamma=None, k_gamma=None,
                          eps: float = 1e-5, layout: str = "split", base: float = 100.0, dq=None, dk=None, q_dgamma=None,
                          q_dbeta=None, k_dgamma=None, k_dbeta=None, want_weights: bool = True, workspace=None,
                          stream=None) -> dict:
    """Gradients of ress_qk_norm_rope (see include/ress_pages.h): dq_out, dk_out of its outputs; q, k and the other
    arguments as it was given (either pair may be None). Returns dq and dk (of q's and k's type; given, they may be dq_out
    and dk_out, or q and k) and, with want_weights or given buffers, q_dgamma, q_dbeta, k_dgamma, k_dbeta (float32 [D];
    with given ones, those alone)."""
    dtype, code, dev, N, D = _first(q, k)
    H = H_kv = qh = qt = kh = kt = gqh = gqt = gkh = gkt = dqh = dqt = dkh = dkt = 0
    q_in = k_in = gq = gk = dq_to = dk_to = None
    if q is not None:
        H = q.shape[0]
        qh, qt, q_in = _rows("q", q, dtype, H, N, D, dev)
        gqh, gqt, gq = _rows("dq_out", dq_out, dtype, H, N, D, dev)
        if dq is None:
            dq = empty((H, N, D), dtype, dev, stream)
        dqh, dqt, dq_to = _rows("dq", dq, dtype, H, N, D, dev)
    else:
        dq = None
    if k is not None:
        H_kv = k.shape[0]
        kh, kt, k_in = _rows("k", k, dtype, H_kv, N, D, dev)
        gkh, gkt, gk = _rows("dk_out", dk_out, dtype, H_kv, N, D, dev)
        if dk is None:
            dk = empty((H_kv, N, D), dtype, dev, stream)
        dkh, dkt, dk_to = _rows("dk", dk, dtype, H_kv, N, D, dev)
    else:
        dk = None
    shape = _head_shape(H, H_kv, N, D, dims, layout, code, base, norm, eps, (qh, qt, kh, kt, 0, 0, 0, 0))
    grads = _GRADS(gqh, gqt, gkh, gkt, dqh, dqt, dkh, dkt)
    if want_weights and q_dgamma is q_dbeta is k_dgamma is k_dbeta is None:
        q_dgamma, q_dbeta, k_dgamma, k_dbeta = (empty((D,), _F32, dev, stream) for _ in range(4))
    sums = (_flat("q_dgamma", q_dgamma, _F32, D, dev), _flat("q_dbeta", q_dbeta, _F32, D, dev),
            _flat("k_dgamma", k_dgamma, _F32, D, dev), _flat("k_dbeta", k_dbeta, _F32, D, dev))
    ws, ws_bytes = None, 0
    if sums != _NONE:
        workspace, ws, ws_bytes = _workspace(workspace, "ress_qk_norm_rope_bwd_workspace_size", shape, dev, stream)
    _call(lib.ress_qk_norm_rope_bwd, dev, stream, shape, grads, _pos(pos, N, dims, dev), gq, gk, q_in, k_in,
          _flat("q_gamma", q_gamma, _F32, D, dev), _flat("k_gamma", k_gamma, _F32, D, dev), dq_to, dk_to, *sums, ws, ws_bytes)
    return dict(dq=dq, dk=dk, q_dgamma=q_dgamma, q_dbeta=q_dbeta, k_dgamma=k_dgamma, k_dbeta=k_dbeta)


_NONE = (None,) * 4


# --------------------------------------------------------- pages of a step


def _tables(tables, dev=None):
    """Device, sequences, entries, row stride and address of tables int32 [B][max_pages]."""
    if tables is None or tables.dtype is not _I32:
        raise ValueError("tables must be an int32 tensor [B][max_pages]")
    shape, st = tables.shape, tables.stride()
    if dev is None:
        dev = _device("tables", tables)
    elif tables.device != dev:
        raise ValueError(f"tables must be on {dev}")
    if len(shape) != 2 or (st[1] != 1 and shape[1] > 1):
        raise ValueError("tables must be an int32 tensor [B][max_pages] with contiguous rows")
    B, n = shape
    return dev, B, n, st[0] if B > 1 else n, tables.data_ptr()


def ress_page_tables(lens, new_lens, tables, free_pages, n_free, *, page: int, tokens: int | None = None, lens_out=None,
                     n_free_out=None, cu_q=None, slots=None, pos=None, n_refused=None, stream=None) -> dict:
    """Tables, slots and positions of a step (see include/ress_pages.h). lens, new_lens: int32 [B]; tables: int32
    [B][max_pages] with any row stride, updated; free_pages: int32 [n_pages]; n_free: int32 [1]. tokens: entries of slots
    and pos where these are made here. lens_out may be lens, n_free_out n_free. Returns lens, n_free, cu_q, slots, pos,
    n_refused."""
    dev, B, max_pages, stride, table = _tables(tables)
    if tokens is None:
        if slots is None and pos is None:
            raise ValueError("tokens, or slots and pos, must be given")
        tokens = (slots if slots is not None else pos).shape[0]
    if free_pages is None:
        raise ValueError("free_pages must be given")
    n_pages = free_pages.shape[0]
    make = lambda n: empty((n,), _I32, dev, stream)
    lens_out = make(B) if lens_out is None else lens_out
    n_free_out = make(1) if n_free_out is None else n_free_out
    cu_q = make(B + 1) if cu_q is None else cu_q
    slots = make(tokens) if slots is None else slots
    pos = make(tokens) if pos is None else pos
    n_refused = make(1) if n_refused is None else n_refused
    _call(lib.ress_page_tables, dev, stream, _TABLE(B, tokens, page, n_pages, max_pages, stride, 0), _ints("lens", lens, B, dev),
          _ints("new_lens", new_lens, B, dev), _flat("free_pages", free_pages, _I32, n_pages, dev), _ints("n_free", n_free, 1, dev),
          table, _flat("lens_out", lens_out, _I32, B, dev), _flat("n_free_out", n_free_out, _I32, 1, dev),
          _flat("cu_q", cu_q, _I32, B + 1, dev), _flat("slots", slots, _I32, tokens, dev), _flat("pos", pos, _I32, tokens, dev),
          _flat("n_refused", n_refused, _I32, 1, dev))
    return dict(lens=lens_out, n_free=n_free_out, cu_q=cu_q, slots=slots, pos=pos, n_refused=n_refused)


def ress_pages_release_workspace_size(B: int) -> int:
    return _size("ress_pages_release_workspace_size", _TABLE(B, 0, 1, 0, 0, 0, 0))


def ress_pages_release(first, last, tables, free_pages, n_free, *, clear: bool = True, n_free_out=None, workspace=None,
                       stream=None):
    """Gives entries [first[b], last[b]) of every table back to the stack of free pages (see include/ress_pages.h).
    first, last: int32 [B]; clear: mark them with -1. n_free_out may be n_free. Returns the stack's new height (int32
    [1])."""
    dev, B, max_pages, stride, table = _tables(tables)
    if free_pages is None:
        raise ValueError("free_pages must be given")
    n_pages = free_pages.shape[0]
    ins = _ints("first", first, B, dev), _ints("last", last, B, dev)
    stack = _flat("free_pages", free_pages, _I32, n_pages, dev), _ints("n_free", n_free, 1, dev)
    out = empty((1,), _I32, dev, stream) if n_free_out is None else n_free_out
    to = _flat("n_free_out", out, _I32, 1, dev)
    shape = _TABLE(B, 0, 1, n_pages, max_pages, stride, bool(clear))
    workspace, ws, ws_bytes = _workspace(workspace, "ress_pages_release_workspace_size", shape, dev, stream)
    _call(lib.ress_pages_release, dev, stream, shape, *ins, table, *stack, to, ws, ws_bytes)
    return out


# --------------------------------------------------------------- attention


def ress_paged_attn_workspace_size(B: int, H: int, H_kv: int, N: int, *, page: int, max_pages: int, n_pages: int, window: int,
                                   frame: int = 1, n_sink: int = 0) -> int:
    return _size("ress_paged_attn_workspace_size",
                 _PAGED(B, N, H, H_kv, 64, page, n_pages, max_pages, _int32(frame), _int32(window), _int32(n_sink), max_pages,
                        *(0,) * 10))


def ress_paged_attn(q, k_pages, v_pages, cu_q, lens, tables, *, window: int, frame: int = 1, n_sink: int = 0,
                    scale: float | None = None, out=None, lse=None, want_lse: bool = False, workspace=None, stream=None) -> dict:
    """Attention of new tokens of several sequences over their pages (see include/ress_pages.h). q: bf16 [H][N][64], the
    sequences' new tokens one behind the other, those of b from cu_q[b] (int32 [B + 1]) on; k_pages, v_pages: bf16
    [n_pages][H_kv][page][64]; any strides with contiguous channels; lens: int32 [B], the new tokens counted; tables: int32
    [B][max_pages]; window, frame, n_sink: as for ress_window_attn, causal. Returns o (bf16, as q) and, with want_lse or a
    given buffer, lse (float32 [H][N]); their rows outside every sequence are not written."""
    if q is None or k_pages is None:
        raise ValueError("q and k_pages must be given")
    dev, qn, kn = _device("q", q), q.shape, k_pages.shape
    if len(qn) != 3 or len(kn) != 4 or qn[2] != kn[3]:
        raise ValueError("q must be [H][N][64], k_pages and v_pages [n_pages][H_kv][page][64]")
    H, N, D = qn
    n_pages, H_kv, page, _ = kn
    _, B, max_pages, stride, table = _tables(tables, dev)
    if out is None:
        out = empty(qn, _BF16, dev, stream)
    if lse is None and want_lse:
        lse = empty((H, N), _F32, dev, stream)
    qh, qt, q_in = _rows("q", q, _BF16, H, N, D, dev)
    oh, ot, to = _rows("out", out, _BF16, H, N, D, dev)
    kps, kph, kpt, k_in = _paged("k_pages", k_pages, _BF16, kn, dev)
    vps, vph, vpt, v_in = _paged("v_pages", v_pages, _BF16, kn, dev)
    shape = _PAGED(B, N, H, H_kv, D, page, n_pages, max_pages, _int32(frame), _int32(window), _int32(n_sink), stride,
                   qh, qt, oh, ot, kps, kph, kpt, vps, vph, vpt)
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    workspace, ws, ws_bytes = _workspace(workspace, "ress_paged_attn_workspace_size", shape, dev, stream)
    _call(lib.ress_paged_attn, dev, stream, shape, q_in, k_in, v_in, _ints("cu_q", cu_q, B + 1, dev),
          _ints("lens", lens, B, dev), table, float(scale), to, _dense("lse", lse, _F32, (H, N), dev), ws, ws_bytes)
    return dict(o=out, lse=lse)
