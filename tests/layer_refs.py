"""Plain float64 forms of the steps in include/ress_layer.h, on the CPU or the GPU, and the error
bounds their tests use. H(t) is half a step of a type relative to the value: 2^-8 for bf16, 2^-24
for float32."""
import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


# ---------------------------------------------------------------- layer norm


def norm(x, gamma, beta, eps):
    x = x.double()
    mean = x.mean(-1)
    var = ((x - mean[..., None]) ** 2).mean(-1)
    rstd = (var + eps).rsqrt()
    y = (x - mean[..., None]) * rstd[..., None]
    if gamma is not None:
        y = y * gamma.double()
    if beta is not None:
        y = y + beta.double()
    return y, mean, rstd


def norm_bwd(dy, x, gamma, mean, rstd):
    dy, xh = dy.double(), (x.double() - mean.double()[..., None]) * rstd.double()[..., None]
    g = dy if gamma is None else dy * gamma.double()
    dx = rstd.double()[..., None] * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    lead = tuple(range(dy.dim() - 1))
    return dx, (dy * xh).sum(lead), dy.sum(lead)


# --------------------------------------------------------- rotary positions


def rope_pairs(dims, layout, base):
    """(axis, frequency, first channel, second channel) of every pair."""
    out, at, n = [], 0, 0
    total = sum(dims)
    for axis, d in enumerate(dims):
        for i in range(d // 2):
            if layout == "split":
                out.append((axis, base ** (-2.0 * i / d), at + i, at + i + d // 2))
            elif layout == "interleaved":
                out.append((axis, base ** (-2.0 * i / d), at + 2 * i, at + 2 * i + 1))
            else:
                out.append((axis, base ** (-2.0 * n / total), n, n + total // 2))
            n += 1
        at += d
    return out


def rope(x, pos, dims, layout, base, inverse=False):
    y = x.double().clone()
    for axis, f, a, b in rope_pairs(dims, layout, base):
        t = pos[:, axis].double() * f * (-1.0 if inverse else 1.0)
        xa, xb = x[..., a].double(), x[..., b].double()
        y[..., a] = xa * torch.cos(t) - xb * torch.sin(t)
        y[..., b] = xa * torch.sin(t) + xb * torch.cos(t)
    return y


def rope_bound(x, y, pos, dims, layout, base):
    """Half a step of the output, and 2^-21 (|a| + |b|): a cosine and sine within 2^-22 (the turn's
    fraction rounded to 2^-24 of half a turn, the functions to 2 steps) and three roundings of the products."""
    mag = torch.zeros_like(y)
    for _, _, a, b in rope_pairs(dims, layout, base):
        m = x[..., a].double().abs() + x[..., b].double().abs()
        mag[..., a] = mag[..., b] = m
    return HALF[x.dtype] * y.abs() + 2.0 ** -21 * mag


# ------------------------------------------------------------------ windows


def visible(n_q, n_k, q_offset, frame, window, n_sink, causal, device="cpu"):
    fp = ((torch.arange(n_q, device=device) + q_offset) // frame)[:, None]
    s = torch.arange(n_k, device=device)
    fs = s // frame
    if causal:
        return (fs <= fp) & ((fp - fs < window) | (s < n_sink))
    return ((fp - fs).abs() < window) | (s < n_sink).expand(n_q, n_k)


def window(q, k, v, vis, scale=None):
    """o, lse, and the bound's weights sum p |v|, all float64 [H][n_q]..., head by head."""
    H, g = q.shape[0], q.shape[0] // max(k.shape[0], 1)
    scale = 1.0 / math.sqrt(q.shape[2]) if scale is None else scale
    o, lse, w, mag = [], [], [], []
    for h in range(H):
        qd, kd, vd = q[h].double(), k[h // g].double(), v[h // g].double()
        x = torch.where(vis, (qd @ kd.T) * scale, -math.inf)
        l = torch.logsumexp(x, 1) if x.shape[1] else torch.full((x.shape[0],), -math.inf, device=x.device).double()
        p = torch.where(vis, torch.exp(x - torch.where(l == -math.inf, 0.0, l)[:, None]), 0.0)
        # (keys that nothing sees have no part, whatever they hold)
        vd = torch.where(vis.any(0)[:, None], vd, 0.0)
        o.append(p @ vd)
        lse.append(l)
        w.append(p @ vd.abs())
        m = (qd.abs() @ torch.where(vis.any(0)[:, None], kd, 0.0).abs().T) * scale
        mag.append(m.amax(1) if m.shape[1] else m.sum(1))
    return tuple(torch.stack(t) for t in (o, lse, w, mag))


def window_bound(o, w, mag):
    """p, rounded to bf16 for its product (2^-8 of each) and normalised by the sum of the rounded or unrounded
    ones (2^-8 of o), and o's own rounding: 2^-8 (w + 2 |o|). Products of 64 channels in float32 move a logit by at
    most 64 2^-24 mag, both sides of the quotient: 2^-17 mag w. The rest (exp2, sums in float32): 2^-12 w."""
    return 2.0 ** -8 * (w + 2 * o.abs()) + (2.0 ** -17 * mag[..., None] + 2.0 ** -12) * w


def window_bwd(d_o, q, k, v, vis, scale=None):
    """dq, dk, dv and their bounds, float64.
    Bounds: ds and p rounded to bf16 for their products (2^-8 of each term), outputs once (2^-8); what float32 leaves in
    p (2^-17 mag) and in d_o v^T - delta; and for dq the product of the two roundings in delta and p (2^-15 of
    p (|d_o| |v| + its mean)), which bounds the float32 part too."""
    H, H_kv = q.shape[0], k.shape[0]
    g = H // max(H_kv, 1)
    scale = 1.0 / math.sqrt(q.shape[2]) if scale is None else scale
    kw = dict(dtype=torch.float64, device=q.device)
    dq, bq = torch.zeros(q.shape, **kw), torch.zeros(q.shape, **kw)
    dk, bk, dv, bv = (torch.zeros(k.shape, **kw) for _ in range(4))
    for h in range(H if k.shape[1] else 0):  # (without keys every gradient is zero)
        qd, kd, vd, do = q[h].double(), k[h // g].double(), v[h // g].double(), d_o[h].double()
        x = torch.where(vis, (qd @ kd.T) * scale, -math.inf)
        l = torch.logsumexp(x, 1, keepdim=True)
        p = torch.where(vis, torch.exp(x - torch.where(l == -math.inf, 0.0, l)), 0.0)
        dp = do @ vd.T
        ds = p * (dp - (p * dp).sum(1, keepdim=True))
        dq[h] = scale * (ds @ kd)
        dk[h // g] += scale * (ds.T @ qd)
        dv[h // g] += p.T @ do
        mag = (torch.where(vis, qd.abs() @ kd.abs().T, 0.0) * scale).amax(1, keepdim=True)
        dpm = do.abs() @ vd.abs().T
        rough = p * (dpm + (p * dpm).sum(1, keepdim=True)) * (2.0 ** -14 + 2.0 ** -17 * mag)
        e = 2.0 ** -8 * ds.abs() + rough
        ep = p * (2.0 ** -8 + 2.0 ** -14 + 2.0 ** -17 * mag)
        bq[h] = scale * (e @ kd.abs())
        bk[h // g] += scale * (e.T @ qd.abs())
        bv[h // g] += ep.T @ do.abs()
    return dq, dk, dv, bq + 2.0 ** -8 * dq.abs(), bk + 2.0 ** -8 * dk.abs(), bv + 2.0 ** -8 * dv.abs()


def within(got, ref, bound, what=""):
    """got (any type) within `bound` of ref everywhere; infinities must match."""
    got = got.double()
    fin = torch.isfinite(ref)
    assert torch.equal(torch.isfinite(got), fin), f"{what}: finite entries differ"
    assert torch.equal(got[~fin], ref[~fin]), f"{what}: infinities differ"
    err = (got - ref).abs()[fin]
    lim = bound.expand_as(ref)[fin] if torch.is_tensor(bound) else torch.full_like(err, bound)
    bad = err > lim
    if bool(bad.any()):
        i = int((err - lim).argmax())
        raise AssertionError(f"{what}: {int(bad.sum())} of {err.numel()} beyond the bound, e.g. {err[i].item():.3e} "
                             f"against {lim[i].item():.3e}")
