"""The steps of a layer around and beside its global attention, for timing and
for comparing them with their definitions: layer norm (forward, backward),
rotary positions with several axes, and attention over a sliding window of
frames with sink tokens (forward, backward, one token over a cache).

With `own` set, run() makes the calls a program makes of this package; without
it, the same operators in elementary torch operations in 32 bits (rotary angles
in 64). exact() is each operator's definition in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

D = 64
FRAME = 37 * 37 + 5  # a 518 x 518 view in 14-pixel patches, and its special tokens
RANK = 8
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------- cases


def _norm(name, rows, width, x="f32", y="bf16", stats=False, kind="norm"):
    return dict(name=name, kind=kind, rows=rows, width=width, x=x, y=y, stats=stats)


def _rope(name, tokens, heads, kv_heads, dims, layout, dtype="bf16", width=D, base=100.0, first=0, inverse=False,
          token_major=False):
    return dict(name=name, kind="rope", tokens=tokens, heads=heads, kv_heads=kv_heads, width=width,
                dims="/".join(str(d) for d in dims), layout=layout, dtype=dtype, base=base, first=first,
                inverse=inverse, token_major=token_major)


def _window(name, kind, n_q, n_k, heads, kv_heads, frame, window, sinks, causal=True, lse=False, token_major=False):
    return dict(name=name, kind=kind, n_q=n_q, n_k=n_k, heads=heads, kv_heads=kv_heads, frame=frame, window=window,
                sinks=sinks, causal=causal, lse=lse, token_major=token_major)


def _decode(name, batch, heads, kv_heads, capacity, shortest, longest, frame, window, sinks):
    return dict(name=name, kind="decode", batch=batch, heads=heads, kv_heads=kv_heads, capacity=capacity,
                shortest=shortest, longest=longest, frame=frame, window=window, sinks=sinks)


def listed():
    return [
        # The special tokens of one view before a small head: the smallest call, all latency.
        _norm("norm_5_tokens", 5, 1024),
        # The residual stream of the 32-view layer before its QKV projection.
        _norm("norm_32v", 32 * FRAME, 1024),
        # Training on a 16-view layer: the same step backward.
        _norm("norm_bwd_16v", 16 * FRAME, 1024, kind="norm_bwd"),
        # Training with per-head norms of Q: many short rows, one small weight gradient.
        _norm("norm_bwd_heads_8v", 16 * 8 * FRAME, D, x="bf16", kind="norm_bwd"),
        # Q and K of the 32-view layer turned by their patches' rows and columns.
        _rope("rope_32v", 32 * FRAME, 16, 16, (32, 32), "split"),
        # One new view of a stream in float32 (time, row, column sections), token-major, gradients of shared K heads.
        _rope("rope_view_f32", FRAME, 12, 4, (16, 24, 24), "sections", dtype="f32", base=1e4, first=977, inverse=True,
              token_major=True),
        # A 32-view stream: each view sees itself, the three before it and the first.
        _window("window_32v", "window", 32 * FRAME, 32 * FRAME, 16, 16, FRAME, 4, FRAME),
        # Training forward on an odd count of tokens with a token window and shared K/V heads.
        _window("window_tokens", "window", 10001, 10001, 16, 4, 1, 1024, 4, lse=True, token_major=True),
        # Training on an 8-view stream: the backward pass.
        _window("window_bwd_8v", "window_bwd", 8 * FRAME, 8 * FRAME, 16, 16, FRAME, 3, FRAME),
        # A short window on both sides, shared K/V heads, backward.
        _window("window_bwd_tokens", "window_bwd", 3001, 3001, 12, 4, 1, 257, 5, causal=False),
        # One token of one stream: the latency of a step.
        _decode("decode_1", 1, 16, 16, 32 * FRAME, 32 * FRAME - 7, 32 * FRAME - 7, FRAME, 4, FRAME),
        # One token for each of many streams of ragged lengths, shared K/V heads.
        _decode("decode_24", 24, 16, 4, 20000, 1, 20000, 1, 4096, 64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_bwd", "rope", "window", "window", "window_bwd", "decode"])
    if kind in ("norm", "norm_bwd"):
        width = rng.choice([D, D, 768, 1024, 1024, _log(rng, 1, 8192)])
        most = 32 * FRAME * 1024 if kind == "norm" else 16 * FRAME * 1024
        rows = _log(rng, 1, max(1, most // max(width, 48)))
        c = _norm("", rows, width, x=rng.choice(["f32", "bf16"]), y=rng.choice(["bf16", "bf16", "f32"]),
                  stats=rng.random() < 0.5, kind=kind)
    elif kind == "rope":
        layout = rng.choice(["split", "interleaved", "sections"])
        dims = rng.choice([(32, 32), (16, 24, 24), (64,), (20, 20, 24), (16, 16, 16), (10, 14)])
        kv = rng.choice([0, 1, 4])
        heads = max(1, kv) * rng.choice([1, 3, 4])
        c = _rope("", _log(rng, 1, 32 * FRAME * 32 // (heads + kv) // 2), heads, kv, dims, layout,
                  dtype=rng.choice(["bf16", "bf16", "f32"]), base=rng.choice([100.0, 1e4, 5e5]),
                  first=rng.choice([0, rng.randint(0, 1 << 20)]), inverse=rng.random() < 0.4,
                  token_major=rng.random() < 0.4)
    elif kind in ("window", "window_bwd"):
        most = 3.5e9 if kind == "window" else 7e8  # pairs times heads, below the largest listed
        while True:
            heads, kv = rng.choice([(1, 1), (4, 1), (6, 2), (8, 8), (12, 4), (16, 4), (16, 8), (16, 16)])
            n_k = _log(rng, 1, 32 * FRAME if kind == "window" else 8 * FRAME)
            n_q = n_k if kind == "window_bwd" or rng.random() < 0.6 else _log(rng, 1, n_k)
            frame = rng.choice([1, 1, rng.randint(2, 300), FRAME])
            window = _log(rng, 1, max(1, 8192 // frame) + 1)
            sinks = rng.choice([0, rng.randint(1, 64), frame])
            c = _window("", kind, n_q, n_k, heads, kv, frame, window, sinks, causal=rng.random() < 0.7,
                        lse=rng.random() < 0.4, token_major=rng.random() < 0.4)
            if 0 < _pairs(c) * heads <= most:
                break
    else:
        heads, kv = rng.choice([(1, 1), (8, 1), (6, 2), (16, 4), (32, 4), (16, 8), (16, 16)])
        batch = _log(rng, 1, 48)
        longest = min(_log(rng, 1, 32 * FRAME), 24 * 4 * 20000 // (batch * kv) + 1)
        frame = rng.choice([1, rng.randint(2, 300), FRAME])
        c = _decode("", batch, heads, kv, longest + rng.randint(0, 100),
                    rng.choice([1, longest]), longest, frame, _log(rng, 1, max(1, 16384 // frame)),
                    rng.choice([0, rng.randint(1, 64), frame]))
    del c["name"]
    return c


def _ranges(c):
    """For every query of a window case: its window of keys [lo, hi) and its sinks [0, sk)."""
    at = np.arange(c["n_q"], dtype=np.int64) + (c["n_k"] - c["n_q"])
    f = at // c["frame"]
    lo = np.maximum(0, (f - c["window"] + 1) * c["frame"])
    hi = np.minimum(c["n_k"], (f + (1 if c["causal"] else c["window"])) * c["frame"])
    sk = np.minimum(c["sinks"], hi if c["causal"] else np.full_like(hi, c["n_k"]))
    return lo, hi, sk


def _pairs(c):
    lo, hi, sk = _ranges(c)
    lo, hi = np.minimum(lo, hi), hi
    return int((hi - lo + np.minimum(sk, lo)).sum() + np.maximum(sk - np.maximum(hi, 0), 0).sum())


def _lengths(c):
    """The lengths of a decode case's streams, spread evenly (their order goes by the seed)."""
    return np.rint(np.linspace(c["shortest"], c["longest"], c["batch"])).astype(np.int64)


def _seen(c):
    n = _lengths(c)
    lo = np.maximum(0, ((n - 1) // c["frame"] - c["window"] + 1) * c["frame"])
    return int((n - lo + np.minimum(np.minimum(c["sinks"], n), lo)).sum())


def work(case):
    c, kind = case, case["kind"]
    size = {"bf16": 2, "f32": 4}
    if kind == "norm":
        n = c["rows"] * c["width"]
        return {"bytes": n * (size[c["x"]] + size[c["y"]]) + 8 * c["width"] + 8 * c["rows"] * c["stats"], "flops": 8 * n}
    if kind == "norm_bwd":
        n = c["rows"] * c["width"]
        return {"bytes": n * (2 * size[c["x"]] + size[c["y"]]) + 12 * c["width"] + 8 * c["rows"], "flops": 14 * n}
    if kind == "rope":
        n = c["tokens"] * (c["heads"] + c["kv_heads"]) * c["width"]
        return {"bytes": 2 * n * size[c["dtype"]] + 4 * c["tokens"] * len(_dims(c)), "flops": 3 * n}
    if kind == "decode":
        seen = _seen(c)
        return {"bytes": seen * c["kv_heads"] * D * 4 + c["batch"] * c["heads"] * D * 4 + 4 * c["batch"],
                "flops": 4 * D * seen * c["heads"]}
    q, k = c["n_q"] * c["heads"] * D * 2, c["n_k"] * c["kv_heads"] * D * 2
    lse = 4 * c["n_q"] * c["heads"]
    if kind == "window":
        return {"bytes": 2 * q + 2 * k + lse * c["lse"], "flops": 4 * D * _pairs(c) * c["heads"]}
    return {"bytes": 4 * q + 4 * k + lse, "flops": 10 * D * _pairs(c) * c["heads"]}


# ------------------------------------------------------------------ inputs


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _place(t, token_major):
    """[heads][tokens][width], with the tokens outermost in memory if token_major."""
    return t.transpose(0, 1).contiguous().transpose(0, 1) if token_major else t.contiguous()


def _states(gen, heads, tokens, frame, dtype, width=D, amp=0.5):
    """Head-major activations with a low-rank part that views share, so that attention is peaked."""
    frames = -(-tokens // frame) if frame > 1 else 1
    fac = torch.randn(heads, RANK, width, generator=gen, device="cuda") * RANK ** -0.5
    code = torch.randn(heads, frames, RANK, generator=gen, device="cuda")
    code = code.repeat_interleave(frame if frame > 1 else tokens, 1)[:, :tokens]
    z = code + torch.randn(heads, tokens, RANK, generator=gen, device="cuda")
    return (amp * torch.matmul(z, fac) + 0.5 * torch.randn(heads, tokens, width, generator=gen, device="cuda")).to(dtype)


def _dims(c):
    return tuple(int(d) for d in c["dims"].split("/"))


def _inputs(c, seed):
    gen, kind = _gen(seed), c["kind"]
    if kind in ("norm", "norm_bwd"):
        rows, w = c["rows"], c["width"]
        x = torch.randn(rows, w, generator=gen, device="cuda") * 1.5 + torch.randn(w, generator=gen, device="cuda")
        s = dict(x=x.to(DTYPES[c["x"]]), gamma=1 + 0.2 * torch.randn(w, generator=gen, device="cuda"),
                 beta=0.1 * torch.randn(w, generator=gen, device="cuda"))
        if kind == "norm_bwd":
            s["dy"] = torch.randn(rows, w, generator=gen, device="cuda").to(DTYPES[c["y"]])
            x = s["x"].double()
            s["mean"] = x.mean(1).float()
            s["rstd"] = (x.var(1, unbiased=False) + 1e-5).rsqrt().float()
        return s
    if kind == "rope":
        n, axes = c["tokens"], len(_dims(c))
        t = torch.arange(n, device="cuda")
        grid = [c["first"] + t // FRAME, 1 + t % FRAME // 37, 1 + t % 37]  # time, patch row, patch column
        pos = torch.stack({1: [c["first"] + t], 2: grid[1:], 3: grid}[axes], 1).int().contiguous()
        qk = [_place(_states(gen, h, n, FRAME, DTYPES[c["dtype"]], c["width"]), c["token_major"]) if h else None
              for h in (c["heads"], c["kv_heads"])]
        return dict(q=qk[0], k=qk[1], pos=pos)
    if kind == "decode":
        q = _states(gen, c["batch"] * c["heads"], 1, 1, torch.bfloat16).view(c["batch"], c["heads"], D)
        k, v = (_states(gen, c["batch"] * c["kv_heads"], c["capacity"], c["frame"], torch.bfloat16).view(
            c["batch"], c["kv_heads"], c["capacity"], D) for _ in range(2))
        lens = _lengths(c)[np.random.default_rng(seed).permutation(c["batch"])]
        return dict(q=q, k=k, v=v, lens=torch.from_numpy(lens.astype(np.int32)).cuda())
    tm = c["token_major"]
    s = dict(q=_place(_states(gen, c["heads"], c["n_q"], c["frame"], torch.bfloat16), tm),
             k=_place(_states(gen, c["kv_heads"], c["n_k"], c["frame"], torch.bfloat16), tm),
             v=_place(_states(gen, c["kv_heads"], c["n_k"], c["frame"], torch.bfloat16, amp=0.25), tm))
    if kind == "window_bwd":
        s["do"] = _place(torch.randn(c["heads"], c["n_q"], D, generator=gen, device="cuda").to(torch.bfloat16), tm)
        o, s["lse"] = _plain_window(c, s)
        s["o"] = _place(o, tm)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["c"] = dict(case)
    if own:  # outputs and workspaces that a program with a loop over layers keeps
        import paper_2609_35593_amd as ress

        s["ress"] = ress
        c, kind, dev = case, case["kind"], "cuda"
        if kind == "norm":
            s["out"] = torch.empty(s["x"].shape, dtype=DTYPES[c["y"]], device=dev)
            s["mean"], s["rstd"] = (torch.empty(c["rows"], device=dev) if c["stats"] else None for _ in range(2))
        elif kind == "norm_bwd":
            s["dx"] = torch.empty_like(s["x"])
            s["dgamma"], s["dbeta"] = (torch.empty(c["width"], device=dev) for _ in range(2))
            s["ws"] = torch.empty(ress.ress_layer_norm_bwd_workspace_size(c["rows"], c["width"]), dtype=torch.uint8,
                                  device=dev)
        elif kind == "rope":
            s["q_out"] = torch.empty_like(s["q"])
            s["k_out"] = None if s["k"] is None else torch.empty_like(s["k"])
        elif kind == "window":
            s["out"] = torch.empty_like(s["q"])
            s["lse"] = torch.empty(c["heads"], c["n_q"], device=dev) if c["lse"] else None
        elif kind == "window_bwd":
            s["dq"], s["dk"], s["dv"] = (torch.empty_like(s[n]) for n in "qkv")
            s["ws"] = torch.empty(ress.ress_window_attn_bwd_workspace_size(
                c["heads"], c["kv_heads"], c["n_q"], c["n_k"], q_offset=c["n_k"] - c["n_q"], frame=c["frame"],
                window=c["window"], n_sink=c["sinks"], causal=c["causal"]), dtype=torch.uint8, device=dev)
        else:
            s["out"] = torch.empty_like(s["q"])
            s["ws"] = torch.empty(ress.ress_window_attn_decode_workspace_size(
                c["batch"], c["heads"], c["kv_heads"], c["capacity"], frame=c["frame"], window=c["window"],
                n_sink=c["sinks"]), dtype=torch.uint8, device=dev)
    return s


# --------------------------------------------------------------------- run


def run(state):
    return (_own if own else _plain)(state["c"], state)


def _own(c, s):
    ress, kind = s["ress"], c["kind"]
    if kind == "norm":
        r = ress.ress_layer_norm(s["x"], s["gamma"], s["beta"], out=s["out"], mean=s["mean"], rstd=s["rstd"])
        return (r["y"], r["mean"], r["rstd"]) if c["stats"] else r["y"]
    if kind == "norm_bwd":
        r = ress.ress_layer_norm_bwd(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"], dx=s["dx"], dgamma=s["dgamma"],
                                     dbeta=s["dbeta"], workspace=s["ws"])
        return r["dx"], r["dgamma"], r["dbeta"]
    if kind == "rope":
        r = ress.ress_rope(s["q"], s["k"], s["pos"], dims=_dims(c), layout=c["layout"], base=c["base"],
                           inverse=c["inverse"], q_out=s["q_out"], k_out=s["k_out"])
        return r["q"] if s["k"] is None else (r["q"], r["k"])
    if kind == "decode":
        return ress.ress_window_attn_decode(s["q"], s["k"], s["v"], s["lens"], frame=c["frame"], window=c["window"],
                                            n_sink=c["sinks"], out=s["out"], workspace=s["ws"])
    kw = dict(q_offset=c["n_k"] - c["n_q"], frame=c["frame"], window=c["window"], n_sink=c["sinks"], causal=c["causal"])
    if kind == "window":
        r = ress.ress_window_attn(s["q"], s["k"], s["v"], out=s["out"], lse=s["lse"], **kw)
        return (r["o"], r["lse"]) if c["lse"] else r["o"]
    r = ress.ress_window_attn_bwd(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], dq=s["dq"], dk=s["dk"], dv=s["dv"],
                                  workspace=s["ws"], **kw)
    return r["dq"], r["dk"], r["dv"]


def _plain(c, s):
    kind = c["kind"]
    if kind == "norm":
        x = s["x"].float()
        mean = x.sum(1, keepdim=True) / c["width"]
        xc = x - mean
        rstd = ((xc * xc).sum(1, keepdim=True) / c["width"] + 1e-5).rsqrt()
        y = (xc * rstd * s["gamma"] + s["beta"]).to(DTYPES[c["y"]])
        return (y, mean[:, 0], rstd[:, 0]) if c["stats"] else y
    if kind == "norm_bwd":
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        xh = (s["x"].float() - s["mean"][:, None]) * rstd
        g = dy * s["gamma"]
        dx = rstd * (g - g.sum(1, keepdim=True) / c["width"] - xh * ((g * xh).sum(1, keepdim=True) / c["width"]))
        return dx.to(s["x"].dtype), (dy * xh).sum(0), dy.sum(0)
    if kind == "rope":
        cos, sin, a, b, rest = _plain_angles(c, s["pos"])
        q = _plain_turn(s["q"], cos, sin, a, b, rest)
        return q if s["k"] is None else (q, _plain_turn(s["k"], cos, sin, a, b, rest))
    if kind == "decode":
        g = c["heads"] // c["kv_heads"]
        q = s["q"].float().view(c["batch"], c["kv_heads"], g, D)
        n = s["lens"][:, None].long()
        at = torch.arange(c["capacity"], device=q.device)[None]
        lo = ((n - 1) // c["frame"] - c["window"] + 1) * c["frame"]
        seen = ((at < c["sinks"]) | (at >= lo)) & (at < n)
        x = torch.matmul(q, s["k"].float().transpose(2, 3).contiguous()) * D ** -0.5
        x = x.masked_fill(~seen[:, None, None], -math.inf)
        p = torch.exp(x - x.amax(3, keepdim=True))
        o = torch.matmul(p, s["v"].float()) / p.sum(3, keepdim=True)
        return o.view(c["batch"], c["heads"], D).to(torch.bfloat16)
    if kind == "window":
        o, lse = _plain_window(c, s)
        return (o, lse) if c["lse"] else o
    return _plain_window_bwd(c, s)


def _plain_angles(c, pos):
    """cos and sin [tokens][pairs], the channels a and b of each pair, and the channels left alone."""
    dims, total, at, pair = _dims(c), sum(_dims(c)), 0, 0
    axis, freq, a, b = [], [], [], []
    for ax, d in enumerate(dims):
        for i in range(d // 2):
            axis.append(ax)
            if c["layout"] == "sections":
                freq.append(c["base"] ** (-2.0 * pair / total))
                a.append(pair)
                b.append(pair + total // 2)
            else:
                freq.append(c["base"] ** (-2.0 * i / d))
                a.append(at + (2 * i if c["layout"] == "interleaved" else i))
                b.append(at + (2 * i + 1 if c["layout"] == "interleaved" else i + d // 2))
            pair += 1
        at += d
    t = pos[:, axis].double() * torch.tensor(freq, dtype=torch.float64).to(pos.device)
    if c["inverse"]:
        t = -t
    return torch.cos(t).float(), torch.sin(t).float(), a, b, list(range(total, c["width"]))


def _plain_turn(x, cos, sin, a, b, rest):
    y = torch.empty_like(x)
    xa, xb = x[..., a].float(), x[..., b].float()
    y[..., a] = (xa * cos - xb * sin).to(x.dtype)
    y[..., b] = (xa * sin + xb * cos).to(x.dtype)
    if rest:
        y[..., rest] = x[..., rest]
    return y


def _blocks(c):
    """Runs of queries with the keys any of them sees, cut so that their scores stay near 1 GB."""
    lo, hi, sk = _ranges(c)
    r0 = 0
    while r0 < c["n_q"]:
        rows = min(c["n_q"] - r0, 4096)
        while True:
            w0, w1, s1 = int(lo[r0]), int(hi[r0 + rows - 1]), int(sk[r0 + rows - 1])
            w0 = 0 if w0 <= s1 else w0
            w1 = max(w1, s1) if w0 == 0 else w1
            keys = max(0, w1 - w0) + (s1 if w0 else 0)
            if rows <= 64 or rows * keys * c["heads"] <= 1 << 28:
                break
            rows //= 2
        parts = ([(0, s1)] if w0 and s1 else []) + ([(w0, w1)] if w1 > w0 else [])
        yield r0, r0 + rows, parts
        r0 += rows


def _seen_block(c, r0, r1, parts, device):
    s = torch.cat([torch.arange(a, b, device=device) for a, b in parts])
    f = (torch.arange(r0, r1, device=device) + (c["n_k"] - c["n_q"])) // c["frame"]
    lo = ((f - c["window"] + 1) * c["frame"])[:, None]
    hi = ((f + (1 if c["causal"] else c["window"])) * c["frame"])[:, None]
    seen = (s >= lo) & (s < hi)
    return seen | ((s < c["sinks"]) & ((s < hi) if c["causal"] else True))


def _gather(x, parts):
    return torch.cat([x[:, a:b] for a, b in parts], 1)


def _shared(x, heads):
    return x.float().repeat_interleave(heads // x.shape[0], 0)


def _plain_window(c, s):
    H, n_q = c["heads"], c["n_q"]
    q, k, v = s["q"].float(), _shared(s["k"], H), _shared(s["v"], H)
    o = torch.zeros(H, n_q, D, dtype=torch.bfloat16, device=q.device)
    lse = torch.full((H, n_q), -math.inf, device=q.device)
    for r0, r1, parts in _blocks(c):
        if not parts:
            continue
        x = torch.matmul(q[:, r0:r1], _gather(k, parts).transpose(1, 2).contiguous()) * D ** -0.5
        x.masked_fill_(~_seen_block(c, r0, r1, parts, q.device), -math.inf)
        top = x.amax(2, keepdim=True)
        p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
        tot = p.sum(2, keepdim=True)
        o[:, r0:r1] = (torch.matmul(p, _gather(v, parts)) / torch.where(tot == 0, 1.0, tot)).to(torch.bfloat16)
        lse[:, r0:r1] = (top + torch.log(tot))[:, :, 0]
    return o, lse


def _plain_window_bwd(c, s):
    H, kv = c["heads"], c["kv_heads"]
    q, k, v, do = s["q"].float(), _shared(s["k"], H), _shared(s["v"], H), s["do"].float()
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for r0, r1, parts in _blocks(c):
        if not parts:
            continue
        kb, vb = _gather(k, parts), _gather(v, parts)
        x = torch.matmul(q[:, r0:r1], kb.transpose(1, 2).contiguous()) * D ** -0.5
        lse = s["lse"][:, r0:r1, None]
        p = torch.exp(x - torch.where(lse == -math.inf, 0.0, lse))
        p.masked_fill_(~_seen_block(c, r0, r1, parts, q.device), 0.0)
        ds = torch.matmul(do[:, r0:r1], vb.transpose(1, 2).contiguous())
        ds = p * (ds - (p * ds).sum(2, keepdim=True)) * D ** -0.5
        dq[:, r0:r1] = torch.matmul(ds, kb)
        gk = torch.matmul(ds.transpose(1, 2).contiguous(), q[:, r0:r1])
        gv = torch.matmul(p.transpose(1, 2).contiguous(), do[:, r0:r1])
        at = 0
        for a, b in parts:
            dk[:, a:b] += gk[:, at:at + b - a]
            dv[:, a:b] += gv[:, at:at + b - a]
            at += b - a
    dk, dv = (t.view(kv, H // kv, -1, D).sum(1) for t in (dk, dv))
    return dq.to(torch.bfloat16), dk.to(torch.bfloat16), dv.to(torch.bfloat16)


# ------------------------------------------------------------------- exact


def exact(case, seed):
    c, kind = case, case["kind"]
    s = _inputs(c, seed)
    if kind == "norm":
        x = s["x"].double()
        mean, var = x.mean(1), x.var(1, unbiased=False)
        rstd = 1.0 / torch.sqrt(var + 1e-5)
        y = (x - mean[:, None]) * rstd[:, None] * s["gamma"].double() + s["beta"].double()
        return (y, mean, rstd) if c["stats"] else y
    if kind == "norm_bwd":
        # The Jacobian of a row's normalised values, applied to gamma dy.
        x, dy, g = s["x"].double(), s["dy"].double(), s["gamma"].double()
        xc = x - x.mean(1, keepdim=True)
        sigma = torch.sqrt((xc ** 2).mean(1, keepdim=True) + 1e-5)
        w = dy * g / sigma
        dx = w - w.mean(1, keepdim=True) - xc * (w * xc).mean(1, keepdim=True) / sigma ** 2
        return dx, (dy * xc / sigma).sum(0), dy.sum(0)
    if kind == "rope":
        q = _exact_turn(c, s["q"], s["pos"])
        return q if s["k"] is None else (q, _exact_turn(c, s["k"], s["pos"]))
    if kind == "decode":
        g, out = c["heads"] // c["kv_heads"], []
        for i, n in enumerate(s["lens"].tolist()):
            at = torch.arange(n, device="cuda")
            at = at[(at < c["sinks"]) | ((n - 1) // c["frame"] - at // c["frame"] < c["window"])]
            k, v = (s[t][i][:, at].double().repeat_interleave(g, 0) for t in "kv")
            p = torch.softmax((k * s["q"][i].double()[:, None]).sum(2) / math.sqrt(D), 1)
            out.append((p[:, :, None] * v).sum(1))
        return torch.stack(out)
    return _exact_window(c, s)


def _exact_turn(c, x, pos):
    y, dims, at, pair = x.double(), _dims(c), 0, 0
    y = y.clone()
    n, half = sum(dims), sum(dims) // 2
    sign = -1.0 if c["inverse"] else 1.0
    for axis, d in enumerate(dims):
        p = pos[:, axis].double()
        for i in range(d // 2):
            if c["layout"] == "sections":
                angle, a, b = p / c["base"] ** (2.0 * pair / n), pair, pair + half
            else:
                angle = p / c["base"] ** (2.0 * i / d)
                a, b = (at + 2 * i, at + 2 * i + 1) if c["layout"] == "interleaved" else (at + i, at + i + d // 2)
            z = torch.complex(x[..., a].double(), x[..., b].double()) * torch.polar(torch.ones_like(angle), sign * angle)
            y[..., a], y[..., b] = z.real, z.imag
            pair += 1
        at += d
    return y


def _exact_window(c, s):
    """Head by head and query block by query block over all keys, by the definition of what a query sees."""
    H, g = c["heads"], c["heads"] // c["kv_heads"]
    n_q, n_k = c["n_q"], c["n_k"]
    fs = torch.arange(n_k, device="cuda") // c["frame"]
    sink = torch.arange(n_k, device="cuda") < c["sinks"]
    back = c["kind"] == "window_bwd"
    o = torch.zeros(H, n_q, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(H, n_q, dtype=torch.float64, device="cuda")
    dk, dv = (torch.zeros(c["kv_heads"], n_k, D, dtype=torch.float64, device="cuda") for _ in range(2))
    for h in range(H):
        k, v = s["k"][h // g].double().contiguous(), s["v"][h // g].double().contiguous()
        for r0 in range(0, n_q, 2048):
            r1 = min(n_q, r0 + 2048)
            f = ((torch.arange(r0, r1, device="cuda") + n_k - n_q) // c["frame"])[:, None]
            if c["causal"]:
                seen = (sink | (f - fs < c["window"])) & (fs <= f)
            else:
                seen = sink | ((f - fs).abs() < c["window"])
            q = s["q"][h, r0:r1].double()
            x = torch.where(seen, (q @ k.T) / math.sqrt(D), -math.inf)
            lse[h, r0:r1] = torch.logsumexp(x, 1)
            p = torch.where(seen, torch.exp(x - lse[h, r0:r1, None]), 0.0)
            if not back:
                o[h, r0:r1] = p @ v
                continue
            do = s["do"][h, r0:r1].double()
            dp = do @ v.T
            ds = p * (dp - (p * dp).sum(1, keepdim=True)) / math.sqrt(D)
            o[h, r0:r1] = ds @ k
            dk[h // g] += ds.T @ q
            dv[h // g] += p.T @ do
    if back:
        return o, dk, dv
    return (o, lse) if c["lse"] else o
