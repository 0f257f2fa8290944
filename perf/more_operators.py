"""What a stream of frames takes when its keys and values live in pages, for timing and for
comparing it with its definition: the norm of every head of Q and K with the position
rotation in the same pass (forward, backward, and with keys and values written into the
pages), the pages of a step (tables, slots and positions from request lengths, and pages
given back), and attention of a chunk of new tokens of several sequences over their pages.

With `own` set, run() makes the calls a program makes of this package; without it, the
same operators in elementary torch operations in 32 bits (rotary angles in 64). exact() is
each operator's definition in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

D = 64
FRAME = 37 * 37 + 5  # a 518 x 518 view in 14-pixel patches, and its special tokens
RANK = 8
EPS = 1e-5
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------- cases


def _heads(name, tokens, heads, kv_heads, dims=(32, 32), layout="split", norm="layer", dtype="bf16", width=D,
           base=100.0, first=0, token_major=False, kind="heads"):
    return dict(name=name, kind=kind, tokens=tokens, heads=heads, kv_heads=kv_heads, width=width,
                dims="/".join(str(d) for d in dims), layout=layout, norm=norm, dtype=dtype, base=base, first=first,
                token_major=token_major)


def _into_pages(name, streams, tokens, padding, page, heads, kv_heads, **kw):
    """`tokens` new tokens of each stream, and `padding` rows behind them that have no slot."""
    return dict(_heads(name, streams * tokens + padding, heads, kv_heads, kind="heads_pages", **kw), streams=streams,
                padding=padding, page=page)


def _tables(name, batch, page, ctx, new, padding=0):
    """Sequences of ctx[0] to ctx[1] cached tokens that get new[0] to new[1] more."""
    return dict(name=name, kind="tables", batch=batch, page=page, ctx_lo=ctx[0], ctx_hi=ctx[1], new_lo=new[0],
                new_hi=new[1], padding=padding)


def _release(name, batch, page, longest, kept):
    """Every sequence gives back its pages behind its first `kept`."""
    return dict(name=name, kind="release", batch=batch, page=page, longest=longest, kept=kept)


def _paged(name, batch, heads, kv_heads, page, ctx, new, frame, window, sinks, lse=False, token_major=False):
    return dict(name=name, kind="paged", batch=batch, heads=heads, kv_heads=kv_heads, page=page, ctx_lo=ctx[0],
                ctx_hi=ctx[1], new_lo=new[0], new_hi=new[1], frame=frame, window=window, sinks=sinks, lse=lse,
                token_major=token_major)


EVERY = 1 << 26  # a window that reaches every key


def listed():
    return [
        # One token of each of 24 streams: a decoding step's Q and K, all latency.
        _heads("heads_24_tokens", 24, 16, 4, (64,), norm="rms", base=1e4, first=20011),
        # Q and K of the 32-view layer, normed by head and turned by their patches' rows and columns.
        _heads("heads_32v", 32 * FRAME, 16, 16),
        # Training on a 16-view layer: the same step backward, with the gradients of its weights.
        _heads("heads_bwd_16v", 16 * FRAME, 16, 16, kind="heads_bwd"),
        # Training in float32 on one view, shared K heads, three axes in sections, token-major.
        _heads("heads_bwd_view_f32", FRAME, 12, 4, (16, 24, 24), "sections", norm="rms", dtype="f32", base=1e4,
               first=977, token_major=True, kind="heads_bwd"),
        # A new view of each of 8 streams on its way into the pages, in a padded batch.
        _into_pages("heads_pages_8_views", 8, FRAME, 272, 64, 16, 4, token_major=True),
        # A decoding step's tables: one token of each of 256 sequences.
        _tables("tables_256_steps", 256, 64, (1, 20000), (1, 1)),
        # Prompts of a view each for 47 streams, small pages, a padded batch.
        _tables("tables_47_views", 47, 16, (0, 30011), (FRAME, FRAME), padding=960),
        # Streams that leave, all but a shared first view's pages.
        _release("release_64", 64, 16, 20000, 85),
        # One token of one stream over everything that it has seen: the latency of a step.
        _paged("paged_1_token", 1, 16, 4, 64, (32 * FRAME - 8, 32 * FRAME - 8), (1, 1), 1, EVERY, 0),
        # Decoding streams and prompts in one batch, ragged, over a window of tokens and sinks.
        _paged("paged_mixed_24", 24, 16, 4, 16, (0, 20000), (1, 700), 1, 4096, 64, token_major=True),
        # A new view of one stream over the 31 before it.
        _paged("paged_view", 1, 16, 16, 64, (31 * FRAME, 31 * FRAME), (FRAME, FRAME), FRAME, EVERY, 0, lse=True),
        # Four views at once for 8 streams of up to 4 views: long chunks, a window of views and the first one.
        _paged("paged_8_prompts", 8, 16, 16, 128, (0, 4 * FRAME), (4 * FRAME, 4 * FRAME), FRAME, 3, FRAME),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_heads(rng, kind):
    layout = rng.choice(["split", "interleaved", "sections"])
    dims = rng.choice([(32, 32), (32, 32), (16, 24, 24), (64,), (20, 20, 24), (16, 16, 16), (10, 14)])
    kv = rng.choice([1, 4, 4, 16])
    heads = min(16, kv * rng.choice([1, 3, 4]))
    most = (16 if kind == "heads_bwd" else 32) * FRAME * 32
    dtype = rng.choice(["bf16", "bf16", "f32"])
    c = _heads("", _log(rng, 1, most // (heads + kv) // (2 if dtype == "f32" else 1)), heads, kv, dims, layout,
               norm=rng.choice(["layer", "rms"]), dtype=dtype, base=rng.choice([100.0, 1e4, 5e5]),
               first=rng.choice([0, rng.randint(0, 1 << 20)]), token_major=rng.random() < 0.4, kind=kind)
    if kind == "heads_pages":
        streams = min(c["tokens"], rng.choice([1, 3, 8, 24]))
        each = max(1, c["tokens"] // streams)
        padding = rng.choice([0, rng.randint(1, 300)])
        c.update(streams=streams, padding=padding, page=rng.choice([16, 32, 64, 128, 24]), tokens=streams * each + padding,
                 dtype="bf16")
    return c


def draw(rng):
    kind = rng.choice(["heads", "heads_bwd", "heads_pages", "tables", "release", "paged", "paged", "paged"])
    if kind.startswith("heads"):
        c = _draw_heads(rng, kind)
    elif kind == "tables":
        batch, page = _log(rng, 1, 256), rng.choice([16, 32, 64, 128, 24])
        each = _log(rng, 1, max(1, 47 * FRAME // batch))
        longest = _log(rng, 1, 30011)
        c = _tables("", batch, page, (0, longest), (rng.choice([1, each]), each), padding=rng.choice([0, rng.randint(1, 999)]))
    elif kind == "release":
        c = _release("", _log(rng, 1, 256), rng.choice([16, 32, 64, 128, 24]), _log(rng, 1, 20000),
                     rng.choice([0, 1, rng.randint(1, 100)]))
    else:
        while True:
            heads, kv = rng.choice([(1, 1), (8, 1), (6, 2), (12, 4), (16, 4), (32, 4), (16, 8), (16, 16)])
            batch, longest = _log(rng, 1, 48), _log(rng, 1, 32 * FRAME)
            new = rng.choice([1, 1, _log(rng, 1, 4 * FRAME)])
            frame = rng.choice([1, 1, rng.randint(2, 300), FRAME])
            c = _paged("", batch, heads, kv, rng.choice([16, 32, 64, 128, 24]), (rng.choice([0, longest]), longest),
                       (rng.choice([1, new]), new), frame, rng.choice([EVERY, _log(rng, 1, max(1, 16384 // frame) + 1)]),
                       rng.choice([0, rng.randint(1, 64), frame]), lse=rng.random() < 0.4, token_major=rng.random() < 0.4)
            ctx, n = _spread(c)
            if _pairs(c) * heads <= 2.2e9 and (ctx + n).sum() * kv <= 8 * 8 * FRAME * 16:
                break
    del c["name"]
    return c


def _spread(c):
    """Cached and new tokens of a case's sequences, paired at random but the same for every seed."""
    at = np.linspace(0.0, 1.0, c["batch"])
    ctx = np.rint(c["ctx_lo"] + at * (c["ctx_hi"] - c["ctx_lo"])).astype(np.int64)
    new = np.rint(c["new_lo"] * (c["new_hi"] / c["new_lo"]) ** at).astype(np.int64)
    return ctx, np.random.RandomState(5).permutation(new)


def _seen(c, ctx, new):
    """For each new token of a sequence: the keys [lo, hi) of its window and [0, sk) of its sinks."""
    f = np.arange(ctx, ctx + new, dtype=np.int64) // c["frame"]
    hi = np.minimum((f + 1) * c["frame"], ctx + new)
    lo = np.maximum(0, (f - c["window"] + 1) * c["frame"])
    return lo, hi, np.minimum(c["sinks"], lo)


def _pairs(c):
    total = 0
    for ctx, new in zip(*_spread(c)):
        lo, hi, sk = _seen(c, ctx, new)
        total += int((hi - lo + sk).sum())
    return total


def _reached(c):
    """Keys that some new token of their sequence sees, over all sequences."""
    total = 0
    for ctx, new in zip(*_spread(c)):
        lo, hi, sk = _seen(c, ctx, new)
        total += int(hi.max() - lo.min() + min(sk.max(), lo.min()))
    return total


def _released(c):
    """Pages of a release case's sequences (their order goes by the seed), and those given back."""
    lens = np.rint(np.linspace(0, c["longest"], c["batch"])).astype(np.int64)
    pages = -(-lens // c["page"])
    return pages, np.maximum(0, pages - c["kept"])


def work(case):
    c, kind = case, case["kind"]
    if kind.startswith("heads"):
        size = {"bf16": 2, "f32": 4}[c["dtype"]]
        n = c["tokens"] * (c["heads"] + c["kv_heads"]) * c["width"]
        pos = 4 * c["tokens"] * len(_dims(c))
        if kind == "heads_bwd":
            return {"bytes": 3 * n * size + pos + 24 * c["width"], "flops": 22 * n}
        more = 4 * c["tokens"] + 2 * size * (c["tokens"] - c["padding"]) * c["kv_heads"] * c["width"] if kind == "heads_pages" else 0
        return {"bytes": 2 * n * size + pos + 16 * c["width"] + more, "flops": 11 * n}
    if kind == "tables":
        ctx, new = _spread(c)
        pages = int((-(-(ctx + new) // c["page"]) - -(-ctx // c["page"])).sum())
        return {"bytes": 16 * c["batch"] + 8 * (int(new.sum()) + c["padding"]) + 8 * pages, "flops": 4 * int(new.sum())}
    if kind == "release":
        back = int(_released(c)[1].sum())
        return {"bytes": 8 * back + 8 * c["batch"], "flops": 2 * back}
    n = int(_spread(c)[1].sum()) * c["heads"]
    return {"bytes": 4 * n * D + _reached(c) * c["kv_heads"] * D * 4 + 4 * n * c["lse"], "flops": 4 * D * _pairs(c) * c["heads"]}


# ------------------------------------------------------------------ inputs


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _place(t, token_major):
    """[heads][tokens][width], with the tokens outermost in memory if token_major."""
    return t.transpose(0, 1).contiguous().transpose(0, 1) if token_major else t.contiguous()


def _states(gen, heads, tokens, fac, dtype, amp=0.5):
    """Activations [heads][tokens][width] with a low-rank part, so that attention is peaked."""
    z = torch.randn(heads, tokens, RANK, generator=gen, device="cuda")
    x = 0.5 * torch.randn(heads, tokens, fac.shape[2], generator=gen, device="cuda")
    return (amp * torch.matmul(z, fac) + x).to(dtype)


def _factors(gen, heads, width=D):
    return torch.randn(heads, RANK, width, generator=gen, device="cuda") * 1.5 * RANK ** -0.5


def _dims(c):
    return tuple(int(d) for d in c["dims"].split("/"))


def _ints(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def _page_rows(rng, counts, n_pages, spare):
    """A table of pages in no order, `spare` entries a row behind them that hold none."""
    order = rng.permutation(n_pages).astype(np.int32)
    table = np.full((len(counts), int(max(counts)) + spare), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(counts):
        table[b, :n] = order[at:at + n]
        at += n
    return table, order[at:]


def _inputs(c, seed):
    gen, kind, rng = _gen(seed), c["kind"], np.random.RandomState(seed % (1 << 31))
    if kind.startswith("heads"):
        n, w, dims, dt = c["tokens"], c["width"], _dims(c), DTYPES[c["dtype"]]
        t = torch.arange(n, device="cuda")
        grid = [c["first"] + t // FRAME, 1 + t % FRAME // 37, 1 + t % 37]  # time, patch row, patch column
        pos = torch.stack({1: [c["first"] + t], 2: grid[1:], 3: grid}[len(dims)], 1).int().contiguous()
        s = dict(pos=pos)
        for name, h in (("q", c["heads"]), ("k", c["kv_heads"])):
            x = _states(gen, h, n, _factors(gen, h, w), torch.float32, 1.0)
            if c["norm"] == "layer":
                x += 0.3 * torch.randn(w, generator=gen, device="cuda")
            s[name] = _place(x.to(dt), c["token_major"])
            s[name + "_gamma"] = 1 + 0.2 * torch.randn(w, generator=gen, device="cuda")
            s[name + "_beta"] = 0.1 * torch.randn(w, generator=gen, device="cuda") if c["norm"] == "layer" else None
            if kind == "heads_bwd":
                s["d" + name] = _place(torch.randn(h, n, w, generator=gen, device="cuda").to(dt), c["token_major"])
        if kind == "heads_pages":
            page, each = c["page"], (n - c["padding"]) // c["streams"]
            s["v"] = _place(_states(gen, c["kv_heads"], n, _factors(gen, c["kv_heads"], w), dt), c["token_major"])
            n_pages = c["streams"] * (-(-each // page) + 2) + 5
            table, _ = _page_rows(rng, [-(-each // page) + 2] * c["streams"], n_pages, 0)
            at = rng.randint(0, page, c["streams"])[:, None] + np.arange(each)  # (chunks begin inside a page)
            slots = np.take_along_axis(table, at // page, 1).astype(np.int64) * page + at % page
            s["slots"] = _ints(np.concatenate([slots.reshape(-1), np.full(c["padding"], -1)]))
            s["k_pages"], s["v_pages"] = (torch.zeros(n_pages, c["kv_heads"], page, w, dtype=dt, device="cuda") for _ in range(2))
        return s
    if kind == "release":
        pages, back = _released(c)
        order = rng.permutation(c["batch"])
        pages = pages[order]
        n_pages = int(pages.sum()) + 77
        table, free = _page_rows(rng, pages, n_pages, 3)
        stack = np.full(n_pages, -1, dtype=np.int32)
        stack[:len(free)] = free
        return dict(first=_ints(np.full(c["batch"], c["kept"])), last=_ints(pages), tables=_ints(table),
                    free_pages=_ints(stack), n_free=_ints([len(free)]))
    ctx, new = _spread(c)
    order = rng.permutation(c["batch"])
    ctx, new, page = ctx[order], new[order], c["page"]
    if kind == "tables":
        had, have = -(-ctx // page), -(-(ctx + new) // page)
        n_pages = int(have.sum()) + 77
        table, free = _page_rows(rng, had, n_pages, int((have - had).max()) + int(have.max() - had.max()) + 3)
        stack = np.full(n_pages, -1, dtype=np.int32)
        stack[:len(free)] = free
        return dict(lens=_ints(ctx), new_lens=_ints(new), tables=_ints(table), free_pages=_ints(stack),
                    n_free=_ints([len(free)]), n=int(new.sum()) + c["padding"])
    lens = ctx + new
    n_pages = int((-(-lens // page)).sum()) + 3
    table, _ = _page_rows(rng, -(-lens // page), n_pages, 2)
    kv = c["kv_heads"]
    fac = _factors(gen, kv)
    n = int(new.sum())
    q = _states(gen, c["heads"], n, fac.repeat_interleave(c["heads"] // kv, 0), torch.bfloat16, 0.7)
    k, v = (_states(gen, kv, n_pages * page, f, torch.bfloat16, a).view(kv, n_pages, page, D).transpose(0, 1).contiguous()
            for f, a in ((fac, 0.7), (_factors(gen, kv), 0.25)))
    return dict(q=_place(q, c["token_major"]), k=k, v=v, tables=_ints(table), lens=_ints(lens),
                cu_q=_ints(np.concatenate([[0], np.cumsum(new)])), host=[(int(a), int(b)) for a, b in zip(ctx, new)])


def prepare(case, seed):
    s = _inputs(case, seed)
    s["c"] = dict(case)
    if own:  # outputs and workspaces that a program with a loop over layers or steps keeps
        import paper_2609_35593_amd as ress

        s["ress"] = ress
        c, kind, dev = case, case["kind"], "cuda"
        if kind in ("heads", "heads_pages"):
            s["q_out"] = torch.empty_like(s["q"])
            s["k_out"] = torch.empty_like(s["k"]) if kind == "heads" else None
        elif kind == "heads_bwd":
            s["dq_in"], s["dk_in"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
            s["weights"] = {n: torch.empty(c["width"], device=dev) for n in ("q_dgamma", "q_dbeta", "k_dgamma", "k_dbeta")
                            if c["norm"] == "layer" or n.endswith("gamma")}
            s["ws"] = torch.empty(ress.ress_qk_norm_rope_bwd_workspace_size(c["heads"], c["kv_heads"], c["tokens"], c["width"]),
                                  dtype=torch.uint8, device=dev)
        elif kind == "tables":
            i32 = dict(dtype=torch.int32, device=dev)
            s["outs"] = dict(lens_out=torch.empty(c["batch"], **i32), n_free_out=torch.empty(1, **i32),
                             cu_q=torch.empty(c["batch"] + 1, **i32), slots=torch.empty(s["n"], **i32),
                             pos=torch.empty(s["n"], **i32), n_refused=torch.empty(1, **i32))
        elif kind == "release":
            s["n_free_out"] = torch.empty(1, dtype=torch.int32, device=dev)
            s["ws"] = torch.empty(ress.ress_pages_release_workspace_size(c["batch"]), dtype=torch.uint8, device=dev)
        else:
            s["out"] = torch.empty_like(s["q"])
            s["lse"] = torch.empty(c["heads"], s["q"].shape[1], device=dev) if c["lse"] else None
            s["ws"] = torch.empty(ress.ress_paged_attn_workspace_size(
                c["batch"], c["heads"], c["kv_heads"], s["q"].shape[1], page=c["page"], max_pages=s["tables"].shape[1],
                n_pages=s["k"].shape[0], frame=c["frame"], window=c["window"], n_sink=c["sinks"]), dtype=torch.uint8, device=dev)
    return s


# --------------------------------------------------------------------- run


def run(state):
    return (_own if own else _plain)(state["c"], state)


def _own(c, s):
    ress, kind = s["ress"], c["kind"]
    if kind.startswith("heads"):
        kw = dict(norm=c["norm"], q_gamma=s["q_gamma"], k_gamma=s["k_gamma"], eps=EPS, dims=_dims(c), layout=c["layout"],
                  base=c["base"])
        if kind == "heads_bwd":
            r = ress.ress_qk_norm_rope_bwd(s["dq"], s["dk"], s["q"], s["k"], s["pos"], dq=s["dq_in"], dk=s["dk_in"],
                                           workspace=s["ws"], **s["weights"], **kw)
            return r["dq"], r["dk"], *(r[n] for n in s["weights"])
        kw.update(q_beta=s["q_beta"], k_beta=s["k_beta"], q_out=s["q_out"])
        if kind == "heads":
            r = ress.ress_qk_norm_rope(s["q"], s["k"], s["pos"], k_out=s["k_out"], **kw)
            return r["q"], r["k"]
        r = ress.ress_qk_norm_rope_pages(s["q"], s["k"], s["v"], s["pos"], s["slots"], s["k_pages"], s["v_pages"], **kw)
        return r["q"], s["k_pages"], s["v_pages"]
    if kind == "tables":
        r = ress.ress_page_tables(s["lens"], s["new_lens"], s["tables"], s["free_pages"], s["n_free"], page=c["page"], **s["outs"])
        return s["tables"], r["lens"], r["n_free"], r["cu_q"], r["slots"], r["pos"], r["n_refused"]
    if kind == "release":
        n_free = ress.ress_pages_release(s["first"], s["last"], s["tables"], s["free_pages"], s["n_free"], clear=False,
                                         n_free_out=s["n_free_out"], workspace=s["ws"])
        return s["free_pages"], n_free
    r = ress.ress_paged_attn(s["q"], s["k"], s["v"], s["cu_q"], s["lens"], s["tables"], frame=c["frame"], window=c["window"],
                             n_sink=c["sinks"], out=s["out"], lse=s["lse"], workspace=s["ws"])
    return (r["o"], r["lse"]) if c["lse"] else r["o"]


def _plain(c, s):
    kind = c["kind"]
    if kind == "heads_bwd":
        angles = _plain_angles(c, s["pos"])
        q, k = (_plain_heads_bwd(c, s["d" + n], s[n], s[n + "_gamma"], angles) for n in "qk")
        sums = (q[1], q[2], k[1], k[2]) if c["norm"] == "layer" else (q[1], k[1])
        return q[0], k[0], *sums
    if kind.startswith("heads"):
        angles = _plain_angles(c, s["pos"])
        q, k = (_plain_heads(c, s[n], s[n + "_gamma"], s[n + "_beta"], angles) for n in "qk")
        if kind == "heads":
            return q, k
        n = c["tokens"] - c["padding"]
        page, at = s["slots"][:n].long() // c["page"], s["slots"][:n].long() % c["page"]
        s["k_pages"][page, :, at] = k[:, :n].transpose(0, 1)
        s["v_pages"][page, :, at] = s["v"][:, :n].transpose(0, 1)
        return q, s["k_pages"], s["v_pages"]
    if kind == "tables":
        return _plain_tables(c, s)
    if kind == "release":
        t = s["tables"]
        at = torch.arange(t.shape[1], device=t.device)
        back = t[(at >= s["first"][:, None]) & (at < s["last"][:, None])]
        s["free_pages"][s["n_free"].long() + torch.arange(back.numel(), device=t.device)] = back
        return s["free_pages"], (s["n_free"] + back.numel()).int()
    o, lse = _plain_paged(c, s)
    return (o, lse) if c["lse"] else o


def _plain_angles(c, pos):
    """cos and sin [tokens][pairs], the channels a and b of each pair."""
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
    return torch.cos(t).float(), torch.sin(t).float(), a, b


def _plain_norm(c, x):
    x = x.float()
    if c["norm"] == "layer":
        x = x - x.sum(2, keepdim=True) / c["width"]
    rstd = ((x * x).sum(2, keepdim=True) / c["width"] + EPS).rsqrt()
    return x * rstd, rstd


def _plain_turn(x, cos, sin, a, b):
    y = x.clone()
    xa, xb = x[..., a], x[..., b]
    y[..., a] = xa * cos - xb * sin
    y[..., b] = xa * sin + xb * cos
    return y


def _plain_heads(c, x, gamma, beta, angles):
    y = _plain_norm(c, x)[0] * gamma
    return _plain_turn(y if beta is None else y + beta, *angles).to(x.dtype)


def _plain_heads_bwd(c, dy, x, gamma, angles):
    cos, sin, a, b = angles
    dy = _plain_turn(dy.float(), cos, -sin, a, b)
    xh, rstd = _plain_norm(c, x)
    g = dy * gamma
    dx = g - xh * ((g * xh).sum(2, keepdim=True) / c["width"])
    if c["norm"] == "layer":
        dx = dx - g.sum(2, keepdim=True) / c["width"]
    return (dx * rstd).to(x.dtype), (dy * xh).sum((0, 1)), dy.sum((0, 1))


def _plain_tables(c, s):
    page, table = c["page"], s["tables"]
    lens, new = s["lens"].long(), s["new_lens"].long()
    had = (lens + page - 1) // page
    want = (lens + new + page - 1) // page - had
    fits = (torch.cumsum(want, 0) <= s["n_free"]) & (torch.cumsum(new, 0) <= s["n"]) & (lens + new <= table.shape[1] * page)
    new, want = new * fits, want * fits
    at = torch.arange(table.shape[1], device=table.device)
    fresh = (at >= had[:, None]) & (at < (had + want)[:, None])
    taken = (torch.cumsum(want, 0) - want)[:, None] + at - had[:, None]
    top = (s["n_free"] - 1 - taken).clamp(0, s["free_pages"].shape[0] - 1)
    table.copy_(torch.where(fresh, s["free_pages"][top], table))
    cu = torch.cat([torch.zeros_like(new[:1]), torch.cumsum(new, 0)])
    t = torch.arange(s["n"], device=table.device)
    b = torch.searchsorted(cu, t, right=True) - 1
    there = b < c["batch"]
    b = b.clamp(max=c["batch"] - 1)
    p = torch.where(there, lens[b] + t - cu[b], 0)
    slots = torch.where(there, table[b, p // page].long() * page + p % page, -1)
    refused = ((s["new_lens"] > 0) & ~fits).sum().view(1)
    return table, (lens + new).int(), (s["n_free"] - want.sum()).int(), cu.int(), slots.int(), p.int(), refused.int()


def _plain_paged(c, s):
    """Sequence by sequence, in runs of queries whose scores stay near 1 GB."""
    H, kv, page = c["heads"], c["kv_heads"], c["page"]
    g, n = H // kv, s["q"].shape[1]
    o = torch.zeros(H, n, D, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((H, n), -math.inf, device="cuda")
    t0 = 0
    for b, (ctx, new) in enumerate(s["host"]):
        lo, hi, sk = _seen(c, ctx, new)
        each = max(1, min(new, (1 << 28) // (H * (ctx + new))))
        for r0 in range(0, new, each):
            r1 = min(new, r0 + each)
            w0, w1 = int(lo[r0:r1].min()), int(hi[r0:r1].max())
            at = torch.arange(w0, w1, device="cuda")
            if sk[r0:r1].max() > 0:
                at = torch.cat([torch.arange(0, min(int(sk[r0:r1].max()), w0), device="cuda"), at])
            rows = s["tables"][b][at // page].long() * page + at % page
            k, v = (s[x].transpose(0, 1).reshape(kv, -1, D)[:, rows].float() for x in "kv")
            q = s["q"][:, t0 + r0:t0 + r1].float().reshape(kv, -1, D)
            x = torch.matmul(q, k.transpose(1, 2).contiguous()).view(H, r1 - r0, -1) * D ** -0.5
            fp, fs = (torch.arange(ctx + r0, ctx + r1, device="cuda") // c["frame"])[:, None], at // c["frame"]
            x.masked_fill_(~((fs <= fp) & ((fs > fp - c["window"]) | (at < c["sinks"]))), -math.inf)
            top = x.amax(2, keepdim=True)
            p = torch.exp(x - top)
            tot = p.sum(2, keepdim=True)
            y = torch.matmul(p.view(kv, g * (r1 - r0), -1), v).view(H, r1 - r0, D) / tot
            o[:, t0 + r0:t0 + r1] = y.to(torch.bfloat16)
            lse[:, t0 + r0:t0 + r1] = (top + torch.log(tot))[:, :, 0]
        t0 += new
    return o, lse


# ------------------------------------------------------------------- exact


def exact(case, seed):
    c, kind = case, case["kind"]
    s = _inputs(c, seed)
    if kind == "heads_bwd":
        q, k = (_exact_heads_bwd(c, s["d" + n], s[n], s[n + "_gamma"], s["pos"]) for n in "qk")
        sums = (q[1], q[2], k[1], k[2]) if c["norm"] == "layer" else (q[1], k[1])
        return q[0], k[0], *sums
    if kind.startswith("heads"):
        q, k = (_exact_heads(c, s[n], s[n + "_gamma"], s[n + "_beta"], s["pos"]) for n in "qk")
        if kind == "heads":
            return q, k
        kp, vp = s["k_pages"].double(), s["v_pages"].double()
        slots = s["slots"].cpu().numpy().astype(np.int64)
        t = torch.from_numpy(np.flatnonzero(slots >= 0)).cuda()
        at = torch.from_numpy(slots[slots >= 0]).cuda()
        for h in range(c["kv_heads"]):
            for pages, x in ((kp, k), (vp, s["v"].double())):
                rows = pages[:, h].reshape(-1, c["width"])
                rows[at] = x[h, t]
                pages[:, h] = rows.view(pages[:, h].shape)
        return q, kp, vp
    if kind == "tables":
        return _exact_tables(c, s)
    if kind == "release":
        first, last, table, free = (s[n].cpu().numpy() for n in ("first", "last", "tables", "free_pages"))
        n = int(s["n_free"][0])
        for b in range(c["batch"]):
            for i in range(first[b], last[b]):
                free[n] = table[b, i]
                n += 1
        return free, np.array([n], dtype=np.int32)
    return _exact_paged(c, s)


def _exact_turn(c, x, pos, sign):
    y, dims, at, pair = x.clone(), _dims(c), 0, 0
    n, half = sum(dims), sum(dims) // 2
    for axis, d in enumerate(dims):
        p = pos[:, axis].double()
        for i in range(d // 2):
            if c["layout"] == "sections":
                angle, a, b = p / c["base"] ** (2.0 * pair / n), pair, pair + half
            else:
                angle = p / c["base"] ** (2.0 * i / d)
                a, b = (at + 2 * i, at + 2 * i + 1) if c["layout"] == "interleaved" else (at + i, at + i + d // 2)
            z = torch.complex(x[..., a], x[..., b]) * torch.polar(torch.ones_like(angle), sign * angle)
            y[..., a], y[..., b] = z.real, z.imag
            pair += 1
        at += d
    return y


def _exact_heads(c, x, gamma, beta, pos):
    x = x.double()
    if c["norm"] == "layer":
        mean, var = x.mean(2, keepdim=True), x.var(2, unbiased=False, keepdim=True)
        y = (x - mean) / torch.sqrt(var + EPS) * gamma.double() + beta.double()
    else:
        y = x / torch.sqrt(x.square().mean(2, keepdim=True) + EPS) * gamma.double()
    return _exact_turn(c, y, pos, 1.0)


def _exact_heads_bwd(c, dy, x, gamma, pos):
    """The Jacobian of a row's normalised values, applied to gamma times the gradient turned back."""
    dy, x = _exact_turn(c, dy.double(), pos, -1.0), x.double()
    xc = x - x.mean(2, keepdim=True) if c["norm"] == "layer" else x
    sigma = torch.sqrt((xc ** 2).mean(2, keepdim=True) + EPS)
    w = dy * gamma.double() / sigma
    dx = w - xc * (w * xc).mean(2, keepdim=True) / sigma ** 2
    if c["norm"] == "layer":
        dx = dx - w.mean(2, keepdim=True)
    return dx, (dy * xc / sigma).sum((0, 1)), dy.sum((0, 1))


def _exact_tables(c, s):
    page = c["page"]
    lens, new, table, free = (s[n].cpu().numpy().copy() for n in ("lens", "new_lens", "tables", "free_pages"))
    n_free, cu, slots, pos = int(s["n_free"][0]), [0], [], []
    for b in range(c["batch"]):
        had, have = -(-int(lens[b]) // page), -(-int(lens[b] + new[b]) // page)
        assert have <= table.shape[1] and have - had <= n_free  # (the measured batches fit)
        for i in range(had, have):
            n_free -= 1
            table[b, i] = free[n_free]
        for p in range(int(lens[b]), int(lens[b] + new[b])):
            slots.append(int(table[b, p // page]) * page + p % page)
            pos.append(p)
        lens[b] += new[b]
        cu.append(len(slots))
    i32 = lambda x: np.array(x, dtype=np.int32)
    fill = s["n"] - len(slots)
    return table, lens, i32([n_free]), i32(cu), i32(slots + [-1] * fill), i32(pos + [0] * fill), i32([0])


def _exact_paged(c, s):
    """Head by head and query block by query block over all keys of a sequence, by the definition of what a query sees."""
    H, g, page = c["heads"], c["heads"] // c["kv_heads"], c["page"]
    n = s["q"].shape[1]
    o = torch.zeros(H, n, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(H, n, dtype=torch.float64, device="cuda")
    t0 = 0
    for b, (ctx, new) in enumerate(s["host"]):
        at = torch.arange(ctx + new, device="cuda")
        fs = at // c["frame"]
        page_of, row = s["tables"][b].long()[at // page], at % page
        for hk in range(c["kv_heads"]):
            k, v = s["k"][page_of, hk, row].double(), s["v"][page_of, hk, row].double()
            for r0 in range(0, new, 2048):
                r1 = min(new, r0 + 2048)
                f = ((torch.arange(r0, r1, device="cuda") + ctx) // c["frame"])[:, None]
                seen = ((at < c["sinks"]) | (f - fs < c["window"])) & (fs <= f)
                for h in range(hk * g, hk * g + g):
                    x = torch.where(seen, (s["q"][h, t0 + r0:t0 + r1].double() @ k.T) / math.sqrt(D), -math.inf)
                    l = torch.logsumexp(x, 1)
                    o[h, t0 + r0:t0 + r1] = torch.exp(x - l[:, None]) @ v
                    lse[h, t0 + r0:t0 + r1] = l
        t0 += new
    return (o, lse) if c["lse"] else o
