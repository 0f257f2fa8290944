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
from .layer import (_DTYPES, ROPE_LAYOUTS, _all_strides, _call, _dense, _device, _int32, _packer, _size, _strides,
                    _workspace)
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


# ----------------------------------------------------------- norm of heads


def _head_shape(H, H_kv, N, D, dims, layout, dtype, base, norm, eps, strides=(0,) * 8):
    if layout not in ROPE_LAYOUTS:
        raise ValueError(f"layout must be one of {sorted(ROPE_LAYOUTS)}")
    if norm not in HEAD_NORMS:
        raise ValueError(f"norm must be one of {sorted(HEAD_NORMS)}")
    axes = len(dims)
    if not 1 <= axes <= 4:
        raise ValueError("one to four axes")
    return _HEADS(H, H_kv, N, D, axes, *dims, *(0,) * (4 - axes), ROPE_LAYOUTS[layout], 0, dtype, base, *strides,
                  HEAD_NORMS[norm], eps)


def _first(q, k):
    """The tensor of q and k that is there, its device, tokens, channels and type."""
    x = q if q is not None else k
    if x is None:
        raise ValueError("one of q and k must be given")
    if x.dtype not in _DTYPES or x.dim() != 3:
        raise ValueError("q and k must be bfloat16 or float32 tensors [heads][tokens][channels]")
    return x.dtype, _device("q and k", x), x.shape[1], x.shape[2]


def _pos(pos, N, dims, dev):
    if pos is None:
        raise ValueError("pos must be given")
    return _dense("pos", pos, _I32, (N, len(dims)), dev)


def _like(name, t, given, dtype, dev, stream):
    """An output laid out as the caller gives it, else a contiguous one; its strides and address."""
    out = empty(t.shape, dtype, dev, stream) if given is None else given
    return out, _strides(name, out, dtype, tuple(t.shape), dev), out.data_ptr()


def ress_qk_norm_rope(q, k, pos, *, dims, norm: str = "layer", q_gamma=None, q_beta=None, k_gamma=None, k_beta=None,
                      eps: float = 1e-5, layout: str = "split", base: float = 100.0, q_out=None, k_out=None,
                      stream=None) -> dict:
    """Norm of every head of q [H][N][D] and k [H_kv][N][D] (either may be None; any strides with contiguous channels)
    and their turn by pos int32 [N][axes], in one pass (see include/ress_pages.h). norm: "layer" or "rms"; gamma, beta:
    float32 [D] or None; dims, layout, base: as for ress_rope. Outputs may be the inputs (in place). Returns q and k."""
    dtype, dev, N, D = _first(q, k)
    H = H_kv = 0
    st, q_in, k_in, q_to, k_to = [(0, 0)] * 4, None, None, None, None
    if q is not None:
        H, st[0], q_in = q.shape[0], _strides("q", q, dtype, (q.shape[0], N, D), dev), q.data_ptr()
        q_out, st[2], q_to = _like("q_out", q, q_out, dtype, dev, stream)
    if k is not None:
        H_kv, st[1], k_in = k.shape[0], _strides("k", k, dtype, (k.shape[0], N, D), dev), k.data_ptr()
        k_out, st[3], k_to = _like("k_out", k, k_out, dtype, dev, stream)
    shape = _head_shape(H, H_kv, N, D, dims, layout, _DTYPES[dtype], base, norm, eps, [n for s in st for n in s])
    weights = [_dense(n, w, _F32, (D,), dev) for n, w in (("q_gamma", q_gamma), ("q_beta", q_beta), ("k_gamma", k_gamma),
                                                        ("k_beta", k_beta))]
    _call(lib.ress_qk_norm_rope, dev, stream, shape, _pos(pos, N, dims, dev), q_in, k_in, *weights, q_to, k_to)
    return dict(q=q_out if q is not None else None, k=k_out if k is not None else None)


def _page_strides(name, t, dtype, shape, dev):
    """The strides (pages, heads, tokens) of [pages][heads][tokens][channels]."""
    st = _all_strides(name, t, dtype, shape, dev)
    return tuple(s if n > 1 else 0 for s, n in zip(st[:3], shape[:3]))


def ress_qk_norm_rope_pages(q, k, v, pos, slots, k_pages, v_pages, *, dims, norm: str = "layer", q_gamma=None, q_beta=None,
                            k_gamma=None, k_beta=None, eps: float = 1e-5, layout: str = "split", base: float = 100.0,
                            q_out=None, stream=None) -> dict:
    """ress_qk_norm_rope with k written into k_pages and v [H_kv][N][D] copied into v_pages (both [n_pages][H_kv][page][D],
    any strides with contiguous channels), token t at slots[t] (int32 [N]; a token without a slot in the cache is left
    out). q may be None. Returns q, k_pages and v_pages."""
    if k is None or v is None or slots is None:
        raise ValueError("k, v and slots must be given")
    dtype, dev, N, D = _first(k, None)
    H, H_kv = 0, k.shape[0]
    if k_pages.dim() != 4:
        raise ValueError("k_pages and v_pages must be [n_pages][H_kv][page][D]")
    n_pages, page = k_pages.shape[0], k_pages.shape[2]
    like = (n_pages, H_kv, page, D)
    qs = qo = (0, 0)
    q_in = q_to = None
    if q is not None:
        H, qs, q_in = q.shape[0], _strides("q", q, dtype, (q.shape[0], N, D), dev), q.data_ptr()
        q_out, qo, q_to = _like("q_out", q, q_out, dtype, dev, stream)
    ks, vs = _strides("k", k, dtype, (H_kv, N, D), dev), _strides("v", v, dtype, (H_kv, N, D), dev)
    shape = _head_shape(H, H_kv, N, D, dims, layout, _DTYPES[dtype], base, norm, eps, (*qs, *ks, *qo, 0, 0))
    cache = _CACHE(n_pages, page, *_page_strides("k_pages", k_pages, dtype, like, dev),
                   *_page_strides("v_pages", v_pages, dtype, like, dev), *vs)
    weights = [_dense(n, w, _F32, (D,), dev) for n, w in (("q_gamma", q_gamma), ("q_beta", q_beta), ("k_gamma", k_gamma),
                                                        ("k_beta", k_beta))]
    _call(lib.ress_qk_norm_rope_pages, dev, stream, shape, cache, _pos(pos, N, dims, dev),
          _dense("slots", slots, _I32, (N,), dev), q_in, k.data_ptr(), v.data_ptr(), *weights, q_to, k_pages.data_ptr(),
          v_pages.data_ptr())
    return dict(q=q_out if q is not None else None, k_pages=k_pages, v_pages=v_pages)


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
    dtype, dev, N, D = _first(q, k)
    H = H_kv = 0
    xs, gs, ptr = [(0, 0)] * 2, [(0, 0)] * 4, [None] * 6  # dq_out, dk_out, q, k, dq, dk
    if q is not None:
        like = (q.shape[0], N, D)
        H, xs[0] = q.shape[0], _strides("q", q, dtype, like, dev)
        gs[0] = _strides("dq_out", dq_out, dtype, like, dev)
        dq, gs[2], to = _like("dq", q, dq, dtype, dev, stream)
        ptr[0], ptr[2], ptr[4] = dq_out.data_ptr(), q.data_ptr(), to
    if k is not None:
        like = (k.shape[0], N, D)
        H_kv, xs[1] = k.shape[0], _strides("k", k, dtype, like, dev)
        gs[1] = _strides("dk_out", dk_out, dtype, like, dev)
        dk, gs[3], to = _like("dk", k, dk, dtype, dev, stream)
        ptr[1], ptr[3], ptr[5] = dk_out.data_ptr(), k.data_ptr(), to
    shape = _head_shape(H, H_kv, N, D, dims, layout, _DTYPES[dtype], base, norm, eps, (*xs[0], *xs[1], 0, 0, 0, 0))
    grads = _GRADS(*[n for s in gs for n in s])
    sums = dict(q_dgamma=q_dgamma, q_dbeta=q_dbeta, k_dgamma=k_dgamma, k_dbeta=k_dbeta)
    if want_weights and all(t is None for t in sums.values()):
        sums = {n: empty((D,), _F32, dev, stream) for n in sums}
    to = [_dense(n, t, _F32, (D,), dev) for n, t in sums.items()]
    weights = [_dense("q_gamma", q_gamma, _F32, (D,), dev), _dense("k_gamma", k_gamma, _F32, (D,), dev)]
    ws, ws_bytes = None, 0
    if any(t is not None for t in to):
        workspace, ws, ws_bytes = _workspace(workspace, "ress_qk_norm_rope_bwd_workspace_size", shape, dev, stream)
    _call(lib.ress_qk_norm_rope_bwd, dev, stream, shape, grads, _pos(pos, N, dims, dev), *ptr[:4], *weights, *ptr[4:], *to, ws,
          ws_bytes)
    return dict(dq=dq if q is not None else None, dk=dk if k is not None else None, **sums)


# --------------------------------------------------------- pages of a step


def _ints(name, t, shape, dev):
    if t is None:
        raise ValueError(f"{name} must be given")
    return _dense(name, t, _I32, shape, dev)


def _tables(tables, dev=None):
    """Sequences, entries and the stride of tables int32 [B][max_pages]."""
    if tables is None or tables.dim() != 2 or tables.dtype is not _I32:
        raise ValueError("tables must be an int32 tensor [B][max_pages]")
    dev = _device("tables", tables) if dev is None else dev
    B, n = tables.shape
    stride, _ = _all_strides("tables", tables, _I32, (B, n), dev)
    return dev, B, n, stride if B > 1 else n


def ress_page_tables(lens, new_lens, tables, free_pages, n_free, *, page: int, tokens: int | None = None, lens_out=None,
                     n_free_out=None, cu_q=None, slots=None, pos=None, n_refused=None, stream=None) -> dict:
    """Tables, slots and positions of a step (see include/ress_pages.h). lens, new_lens: int32 [B]; tables: int32
    [B][max_pages] with any row stride, updated; free_pages: int32 [n_pages]; n_free: int32 [1]. tokens: entries of slots
    and pos where these are made here. lens_out may be lens, n_free_out n_free. Returns lens, n_free, cu_q, slots, pos,
    n_refused."""
    dev, B, max_pages, stride = _tables(tables)
    if slots is None and pos is None and tokens is None:
        raise ValueError("tokens, or slots and pos, must be given")
    N = tokens if tokens is not None else (slots if slots is not None else pos).shape[0]
    if free_pages is None:
        raise ValueError("free_pages must be given")
    n_pages = free_pages.shape[0]
    ins = (_ints("lens", lens, (B,), dev), _ints("new_lens", new_lens, (B,), dev),
           _ints("free_pages", free_pages, (n_pages,), dev), _ints("n_free", n_free, (1,), dev))
    outs = dict(lens=(lens_out, B), n_free=(n_free_out, 1), cu_q=(cu_q, B + 1), slots=(slots, N), pos=(pos, N),
                n_refused=(n_refused, 1))
    outs = {n: (empty((m,), _I32, dev, stream) if t is None else t, m) for n, (t, m) in outs.items()}
    to = [_ints(n, t, (m,), dev) for n, (t, m) in outs.items()]
    shape = _TABLE(B, N, page, n_pages, max_pages, stride, 0)
    _call(lib.ress_page_tables, dev, stream, shape, *ins, tables.data_ptr(), *to)
    return {n: t for n, (t, _) in outs.items()}


def ress_pages_release_workspace_size(B: int) -> int:
    return _size("ress_pages_release_workspace_size", _TABLE(B, 0, 1, 0, 0, 0, 0))


def ress_pages_release(first, last, tables, free_pages, n_free, *, clear: bool = True, n_free_out=None, workspace=None,
                       stream=None):
    """Gives entries [first[b], last[b]) of every table back to the stack of free pages (see include/ress_pages.h).
    first, last: int32 [B]; clear: mark them with -1. n_free_out may be n_free. Returns the stack's new height (int32
    [1])."""
    dev, B, max_pages, stride = _tables(tables)
    if free_pages is None:
        raise ValueError("free_pages must be given")
    n_pages = free_pages.shape[0]
    ins = _ints("first", first, (B,), dev), _ints("last", last, (B,), dev)
    stack = _ints("free_pages", free_pages, (n_pages,), dev), _ints("n_free", n_free, (1,), dev)
    out = empty((1,), _I32, dev, stream) if n_free_out is None else n_free_out
    to = _ints("n_free_out", out, (1,), dev)
    shape = _TABLE(B, 0, 1, n_pages, max_pages, stride, bool(clear))
    workspace, ws, ws_bytes = _workspace(workspace, "ress_pages_release_workspace_size", shape, dev, stream)
    _call(lib.ress_pages_release, dev, stream, shape, *ins, tables.data_ptr(), *stack, to, ws, ws_bytes)
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
    dev, qn, kn = _device("q", q), q.shape, k_pages.shape
    if len(qn) != 3 or len(kn) != 4 or qn[2] != kn[3]:
        raise ValueError("q must be [H][N][64], k_pages and v_pages [n_pages][H_kv][page][64]")
    H, N, D = qn
    n_pages, H_kv, page, _ = kn
    _, B, max_pages, stride = _tables(tables, dev)
    if out is None:
        out = empty(qn, _BF16, dev, stream)
    if lse is None and want_lse:
        lse = empty((H, N), _F32, dev, stream)
    shape = _PAGED(B, N, H, H_kv, D, page, n_pages, max_pages, _int32(frame), _int32(window), _int32(n_sink), stride,
                   *_strides("q", q, _BF16, qn, dev), *_strides("out", out, _BF16, qn, dev),
                   *_page_strides("k_pages", k_pages, _BF16, kn, dev), *_page_strides("v_pages", v_pages, _BF16, kn, dev))
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    workspace, ws, ws_bytes = _workspace(workspace, "ress_paged_attn_workspace_size", shape, dev, stream)
    _call(lib.ress_paged_attn, dev, stream, shape, q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
          _ints("cu_q", cu_q, (B + 1,), dev), _ints("lens", lens, (B,), dev), tables.data_ptr(), float(scale), out.data_ptr(),
          _dense("lse", lse, _F32, (H, N), dev), ws, ws_bytes)
    return dict(o=out, lse=lse)
