"""The steps of include/ress_layer.h as a layer runs them, with the library's projections between them: norm of the
residual stream, QKV projection, per-head norms and rotary positions of Q and K, windowed attention, output projection
into the stream, and the way back; eager, captured into a graph, on streams of their own, and token by token."""
import pytest
import torch

import layer_refs as R
from gpu_helpers import say

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
H, D, FRAME, FRAMES = 4, 64, 75, 6
N, DM = FRAME * FRAMES, 256
WIN = dict(frame=FRAME, window=2, n_sink=FRAME)
ROPE = dict(dims=(16, 24, 24), layout="split", base=100.0)


@pytest.fixture(scope="module")
def ress():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_35593_amd as r

    return r


@pytest.fixture(scope="module")
def state():
    g = torch.Generator(device="cuda").manual_seed(1)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    t = torch.arange(N, device="cuda")
    return dict(x=rn(N, DM), g1=1 + 0.1 * rn(DM), b1=0.1 * rn(DM), w=(rn(3 * DM, DM) * DM ** -0.5).to(BF),
                wo=(rn(DM, DM) * DM ** -0.5).to(BF), gq=1 + 0.1 * rn(D), gk=1 + 0.1 * rn(D),
                gram=torch.eye(D, device="cuda").expand(H, D, D).contiguous(),
                pos=torch.stack([t // FRAME, t % FRAME // 15, t % 15], 1).int().contiguous())


def _forward(ress, s, stream=None):
    n = ress.ress_layer_norm(s["x"], s["g1"], s["b1"], want_stats=True, stream=stream)
    p = ress.ress_qkv_proj_pool(n["y"], s["w"], s["gram"], bq=64, bk=64, stream=stream)
    nq = ress.ress_layer_norm(p["q"], s["gq"], want_stats=True, stream=stream)
    nk = ress.ress_layer_norm(p["k"], s["gk"], want_stats=True, stream=stream)
    r = ress.ress_rope(nq["y"], nk["y"], s["pos"], stream=stream, **ROPE)
    a = ress.ress_window_attn(r["q"], r["k"], p["v"], want_lse=True, stream=stream, **WIN)
    out = ress.ress_out_proj_residual_f32(a["o"], s["wo"], s["x"], stream=stream)
    return dict(n=n, p=p, nq=nq, nk=nk, r=r, a=a, out=out)


def _backward(ress, s, f, do, stream=None):
    """From the gradient of the attention output to those of the projected Q, K, V and of the norms' weights."""
    g = ress.ress_window_attn_bwd(do, f["r"]["q"], f["r"]["k"], f["p"]["v"], f["a"]["o"], f["a"]["lse"], stream=stream, **WIN)
    t = ress.ress_rope(g["dq"], g["dk"], s["pos"], inverse=True, stream=stream, **ROPE)
    q = ress.ress_layer_norm_bwd(t["q"], f["p"]["q"], s["gq"], f["nq"]["mean"], f["nq"]["rstd"], stream=stream)
    k = ress.ress_layer_norm_bwd(t["k"], f["p"]["k"], s["gk"], f["nk"]["mean"], f["nk"]["rstd"], stream=stream)
    return dict(g=g, t=t, q=q, k=k)


def _leaves(tree):
    for v in tree.values():
        if isinstance(v, dict):
            yield from _leaves(v)
        elif torch.is_tensor(v) and v.dtype != torch.uint8:
            yield v


def test_every_step_against_float64_of_what_it_was_given(ress, state):
    s = state
    f = _forward(ress, s)
    rel = lambda got, ref: float((got.double() - ref).norm() / ref.norm())
    # One rounding to bf16 is at most 2^-8 of each value, and 2^-9.8 rms of uniform ones; a product of 256 rounded
    # values adds nothing beyond float32. Twice the rms bounds a norm; attention adds its rounded probabilities.
    one = 2.0 ** -8
    assert rel(f["n"]["y"], R.norm(s["x"], s["g1"], s["b1"], 1e-5)[0]) < one
    qkv = (f["n"]["y"].double() @ s["w"].double().T).view(N, 3, H, D).permute(1, 2, 0, 3)
    for i, n in enumerate("qkv"):
        assert rel(f["p"][n], qkv[i]) < one, n
    assert rel(f["nq"]["y"], R.norm(f["p"]["q"], s["gq"], None, 1e-5)[0]) < one
    for n, src in (("q", f["nq"]["y"]), ("k", f["nk"]["y"])):
        assert rel(f["r"][n], R.rope(src, s["pos"], **ROPE)) < one, n
    vis = R.visible(N, N, 0, FRAME, 2, FRAME, True, device="cuda")
    o, lse, w, mag = R.window(f["r"]["q"], f["r"]["k"], f["p"]["v"], vis)
    R.within(f["a"]["o"], o, R.window_bound(o, w, mag), "o")
    res = s["x"].double() + f["a"]["o"].double().permute(1, 0, 2).reshape(N, DM) @ s["wo"].double().T
    assert rel(f["out"], res) < 2.0 ** -18
    do = torch.randn(H, N, D, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").to(BF)
    b = _backward(ress, s, f, do)
    dq, dk, dv, bq, bk, bv = R.window_bwd(do, f["r"]["q"], f["r"]["k"], f["p"]["v"], vis)
    for n, ref, bound in (("dq", dq, bq), ("dk", dk, bk), ("dv", dv, bv)):
        R.within(b["g"][n], ref, bound, n)
    for n, src in (("q", b["g"]["dq"]), ("k", b["g"]["dk"])):
        assert rel(b["t"][n], R.rope(src, s["pos"], inverse=True, **ROPE)) < one
        st = f["n" + n]
        dx, dg, db = R.norm_bwd(b["t"][n], f["p"][n], s["g" + n], st["mean"], st["rstd"])
        # (dgamma adds 1,800 terms of random sign: 2^-18 of its norm; dbeta's sum of turned gradients likewise)
        assert rel(b[n]["dx"], dx) < one and rel(b[n]["dgamma"], dg) < 2.0 ** -16 and rel(b[n]["dbeta"], db) < 2.0 ** -14


def test_whole_path_gradient_against_float64(ress, state):
    """The gradients at the end of the path back against float64 automatic differentiation of the path from the projected
    Q, K and V: three roundings on the way forward and three on the way back, 2^-8 each at most."""
    s = state
    f = _forward(ress, s)
    do = torch.randn(H, N, D, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(BF)
    b = _backward(ress, s, f, do)
    q, k, v = (f["p"][n].double().requires_grad_() for n in "qkv")
    vis = R.visible(N, N, 0, FRAME, 2, FRAME, True, device="cuda")

    def turn(x):
        cols = [None] * D
        for axis, fr, i, j in R.rope_pairs(ROPE["dims"], ROPE["layout"], ROPE["base"]):
            t = s["pos"][:, axis].double() * fr
            cols[i] = x[..., i] * torch.cos(t) - x[..., j] * torch.sin(t)
            cols[j] = x[..., i] * torch.sin(t) + x[..., j] * torch.cos(t)
        return torch.stack(cols, -1)

    ln = lambda x, g: torch.nn.functional.layer_norm(x, (D,), g.double(), None, 1e-5)
    x = torch.matmul(turn(ln(q, s["gq"])), turn(ln(k, s["gk"])).transpose(1, 2).contiguous()) / 8.0
    o = torch.matmul(torch.softmax(x.masked_fill(~vis, -float("inf")), 2), v)
    (o * do.double()).sum().backward()
    for got, ref in ((b["q"]["dx"], q.grad), (b["k"]["dx"], k.grad), (b["g"]["dv"], v.grad)):
        assert float((got.double() - ref).norm() / ref.norm()) < 6 * 2.0 ** -8


def test_captured_step_replays_like_the_eager_one(ress, state):
    """Forward and backward in one graph, replayed with eager work and synchronisations between the replays; an eager
    result of the same inputs lives on beside it."""
    s = {k: v.clone() for k, v in state.items()}
    do = torch.randn(H, N, D, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda").to(BF)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        f = _forward(ress, s)
        b = _backward(ress, s, f, do)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        cf = _forward(ress, s)
        cb = _backward(ress, s, cf, do)
    for rep in range(3):
        s["x"] += 0.01
        do.neg_()
        for t in list(_leaves(cf)) + list(_leaves(cb)):
            t.fill_(7)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        ef = _forward(ress, s)
        eb = _backward(ress, s, ef, do)
        for a, c in zip(list(_leaves(ef)) + list(_leaves(eb)), list(_leaves(cf)) + list(_leaves(cb))):
            assert torch.equal(a, c), rep
        say(f"[chain] replay {rep}: identical to the eager step")


def test_two_streams_at_once(ress, state):
    """Two steps on two streams given by argument, outputs and workspaces made inside: each as when run alone."""
    states = [state, {k: (v * 0.5 if k == "x" else v) for k, v in state.items()}]
    do = torch.randn(H, N, D, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda").to(BF)
    alone = []
    for s in states:
        f = _forward(ress, s)
        alone.append(list(_leaves(f)) + list(_leaves(_backward(ress, s, f, do))))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in states]
    for rep in range(3):
        got = []
        for s, st in zip(states, streams):
            f = _forward(ress, s, stream=st)
            got.append(list(_leaves(f)) + list(_leaves(_backward(ress, s, f, do, stream=st))))
        torch.cuda.synchronize()
        for a, b in zip(alone, got):
            assert all(torch.equal(x, y) for x, y in zip(a, b)), rep


def test_stream_by_address(ress, state):
    s = state
    st = torch.cuda.Stream()
    a = ress.ress_layer_norm(s["x"], s["g1"], s["b1"], stream=st.cuda_stream)["y"]
    torch.cuda.synchronize()
    assert torch.equal(a, ress.ress_layer_norm(s["x"], s["g1"], s["b1"])["y"])


def test_token_by_token_over_a_cache(ress, state):
    """The last frames' tokens one by one: keys turned straight into the cache, then attention over it; each row is what the
    whole call gives for a frame that ends there (within both bounds)."""
    s = state
    f = _forward(ress, s)
    q, k, v = f["r"]["q"], f["r"]["k"], f["p"]["v"]
    cap = N + 3
    kc, vc = (torch.full((1, H, cap, D), float("nan"), device="cuda").to(BF) for _ in range(2))
    t0 = N - 20
    kc[0, :, :t0], vc[0, :, :t0] = k[:, :t0], v[:, :t0]
    for t in range(t0, N):
        r = ress.ress_rope(f["nq"]["y"][:, t:t + 1], f["nk"]["y"][:, t:t + 1], s["pos"][t:t + 1], k_out=kc[0, :, t:t + 1], **ROPE)
        vc[0, :, t] = v[:, t]
        assert torch.equal(r["q"], q[:, t:t + 1]) and torch.equal(kc[0, :, t], k[:, t])
        lens = torch.tensor([t + 1], dtype=torch.int32, device="cuda")
        o = ress.ress_window_attn_decode(r["q"].transpose(0, 1), kc, vc, lens, **WIN)[0]
        vis = R.visible(1, t + 1, t, FRAME, 2, FRAME, True, device="cuda")
        ref, _, w, mag = R.window(r["q"], k[:, :t + 1], v[:, :t + 1], vis)
        R.within(o, ref[:, 0], R.window_bound(ref, w, mag)[:, 0], "o")
