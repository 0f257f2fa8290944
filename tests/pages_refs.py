"""Plain float64 forms of the steps in include/ress_pages.h, on the CPU or the GPU, and the error bounds their
tests use (HALF: half a step of a type relative to the value)."""
import math

import torch

import layer_refs as R
from layer_refs import HALF, rope, rope_pairs

# ----------------------------------------------------------- norm of heads


def _norm(x, norm, eps):
    x = x.double()
    if norm == "layer":
        x = x - x.mean(-1, keepdim=True)
    rstd = ((x * x).mean(-1, keepdim=True) + eps).rsqrt()
    return x * rstd, rstd


def _row(w, D, none):
    return torch.full((D,), none, dtype=torch.float64) if w is None else w.double()


def _meet(x, dims, layout):
    """Every channel's value plus that of the channel which its pair turns it with (its own alone where none does)."""
    y = x.clone()
    for _, _, a, b in rope_pairs(dims, layout, 1.0):
        y[..., a] = y[..., b] = x[..., a] + x[..., b]
    return y


def heads(x, pos, gamma, beta, norm, eps, dims, layout, base):
    """y and its bound. The mean is off by at most 16 2^-24 of the row's mean |x| (sums of 2 to 8 values a lane, then of up to 64
    lanes in 6 steps, and the product with 1 / D); rstd by 12 2^-24 of itself (the squares' sum likewise, the root, the
    quotient); the products, the weights' and the coefficients' roundings by 6 2^-24, a cosine or sine by 2^-22. So of each
    of a pair's terms 2^-19, of the mean |x| that the means take 2^-19, and the output's own rounding."""
    D = x.shape[-1]
    g, b = (_row(w, D, n).to(x.device) for w, n in ((gamma, 1.0), (beta, 0.0)))
    xh, rstd = _norm(x, norm, eps)
    y = rope(xh * g + b, pos, dims, layout, base)
    mag = xh.abs() * g.abs() + b.abs()
    if norm == "layer":
        mag = mag + rstd * x.double().abs().mean(-1, keepdim=True) * g.abs()
    return y, HALF[x.dtype] * y.abs() + 2.0 ** -19 * _meet(mag, dims, layout)


def heads_bwd(dy, x, pos, gamma, norm, eps, dims, layout, base):
    """dx, dgamma, dbeta and their bounds: u is off by 2^-20 of its pair's |dy|, xh as in heads(); dx's three terms by 2^-18 of
    their magnitudes; the weights' sums by 2^-18 of each term and 2^-24 (256 + rows / 1024) of the terms' sum (a thread's
    chain of rows, its workgroup's, the join's)."""
    D = x.shape[-1]
    g = _row(gamma, D, 1.0).to(x.device)
    u = rope(dy.double(), pos, dims, layout, base, inverse=True)
    um = _meet(dy.double().abs(), dims, layout)
    xh, rstd = _norm(x, norm, eps)
    xm = xh.abs()
    if norm == "layer":
        xm = xm + rstd * x.double().abs().mean(-1, keepdim=True)
    gu, gm = u * g, um * g.abs()
    dx = gu - xh * (gu * xh).mean(-1, keepdim=True)
    mag = gm + xm * (gm * xm).mean(-1, keepdim=True)
    if norm == "layer":
        dx = dx - gu.mean(-1, keepdim=True)
        mag = mag + gm.mean(-1, keepdim=True)
    dx, mag = dx * rstd, mag * rstd
    lead, rows = tuple(range(x.dim() - 1)), x.numel() // max(D, 1)
    e = 2.0 ** -18 + 2.0 ** -24 * (256 + rows / 1024)
    return (dx, (u * xh).sum(lead), u.sum(lead)), (HALF[x.dtype] * dx.abs() + 2.0 ** -18 * mag, e * (um * xm).sum(lead),
                                                   e * um.sum(lead))


# ------------------------------------------------------------------- pages


def tables(lens, new_lens, table, free_pages, n_free, page, N):
    """The step of include/ress_pages.h, sequence by sequence, on lists; `table` is changed."""
    cap, n_pages = page * (len(table[0]) if table else 0), len(free_pages)
    height = min(max(n_free, 0), n_pages)
    out, cu, slots, pos, refused, stop = [], [0], [], [], 0, False
    tokens, wanted = 0, 0  # of the sequences whose tables suffice, those without room among them
    for b, (n, new) in enumerate(zip(lens, new_lens)):
        n, new = min(max(n, 0), cap), max(new, 0)
        fits = n + new <= cap
        had = -(-n // page)
        have = -(-(n + new) // page) if fits else had
        if fits:
            tokens, wanted = tokens + new, wanted + have - had
            stop = stop or tokens > N or wanted > min(max(n_free, 0), n_pages)
        if not fits or stop:
            refused += new > 0
            new, have = 0, had
        for i in range(had, have):
            height -= 1
            table[b][i] = free_pages[height]
        for p in range(n, n + new):
            e = table[b][p // page]
            slots.append(e * page + p % page if 0 <= e < n_pages else -1)
            pos.append(p)
        out.append(n + new)
        cu.append(len(slots))
    fill = N - len(slots)
    return dict(lens=out, n_free=[height], cu_q=cu, slots=slots + [-1] * fill, pos=pos + [0] * fill, n_refused=[refused])


def release(first, last, table, free_pages, n_free, clear):
    """Entries given back, on lists; `table` and `free_pages` are changed. The stack's height."""
    n_pages, most = len(free_pages), len(table[0]) if table else 0
    height = min(max(n_free, 0), n_pages)
    for b, (i0, i1) in enumerate(zip(first, last)):
        for i in range(min(max(i0, 0), most), min(max(i1, 0), most)):
            if 0 <= table[b][i] < n_pages:
                if height < n_pages:
                    free_pages[height] = table[b][i]
                    height += 1
                if clear:
                    table[b][i] = -1
    return height


# --------------------------------------------------------------- attention


def paged(q, k, v, cu, lens, table, frame, window, n_sink, scale=None):
    """o, lse, their bounds and which rows of q are some sequence's, float64: sequence by sequence, over the keys whose pages are
    there. o's bound is that of windowed attention (layer_refs.window_bound), lse's its test's."""
    H, N = q.shape[:2]
    n_pages, H_kv, page, D = k.shape
    kw = dict(dtype=torch.float64, device=q.device)
    o, bo = torch.zeros(H, N, D, **kw), torch.zeros(H, N, D, **kw)
    lse, bl = torch.full((H, N), -math.inf, **kw), torch.zeros(H, N, **kw)
    rows = torch.zeros(N, dtype=torch.bool, device=q.device)
    cap = table.shape[1] * page
    for b in range(len(lens)):
        c0 = min(max(cu[b], 0), N)
        c1 = min(max(cu[b + 1], c0), N)
        n = min(max(lens[b], 0), cap)
        if c1 == c0:
            continue
        rows[c0:c1] = True
        p = torch.arange(c0, c1, device=q.device) - c1 + n
        s = torch.arange(n, device=q.device)
        entry = table[b].long()[s // page] if n else s
        there = (entry >= 0) & (entry < n_pages)
        fp, fs = torch.div(p, frame, rounding_mode="floor")[:, None], s // frame
        vis = (fs <= fp) & ((fs > fp - window) | (s < n_sink)) & there & (p >= 0)[:, None]
        e, r = entry.clamp(0, max(n_pages - 1, 0)), s % page
        if n and n_pages:
            kb, vb = k[e, :, r].transpose(0, 1), v[e, :, r].transpose(0, 1)
        else:
            kb = vb = torch.zeros(H_kv, n, D, device=q.device)
        x, l, w, mag = R.window(q[:, c0:c1], kb, vb, vis, scale)
        o[:, c0:c1], lse[:, c0:c1] = x, l
        bo[:, c0:c1] = R.window_bound(x, w, mag)
        bl[:, c0:c1] = 2.0 ** -18 * (mag + 1) + 2.0 ** -22 * torch.where(torch.isinf(l), 0.0, l).abs()
    return o, lse, bo, bl, rows
