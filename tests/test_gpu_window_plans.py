"""Windowed attention over the ways its kernels spread over the chip: keys cut over 6 to 32 workgroups, four key groups with a
cut, two groups for large frames, lists of queries cut into up to 64 slices, and the step of a stream: a view over a
cache of views. Against float64, with the bounds of layer_refs."""
import pytest
import torch

import layer_refs as R
from gpu_helpers import say
from test_gpu_window import _inputs, _kw

pytestmark = pytest.mark.gpu

# H, H_kv, n_q, n_k, q_offset, frame, window, n_sink, causal
CUTS = [
    (1, 1, 1, 9000, 8999, 1, 9000, 0, True),         # four key groups, keys cut over 17 workgroups
    (1, 1, 3, 40000, 39000, 1, 40000, 70, True),     # ... over 32
    (2, 2, 1, 20000, 19999, 1, 20000, 5, True),
    (3, 1, 70, 12000, 11000, 1, 12000, 5, False),    # ... over 23, all keys seen
    (1, 1, 40, 30000, 29960, 1374, 30, 1374, True),  # ... over 32, frames
    (5, 5, 100, 5000, 4900, 1, 5000, 0, True),       # ... over 9
    (8, 2, 130, 6000, 5870, 1, 6000, 0, True),       # two key groups, over 11
    (10, 2, 300, 12000, 11000, 1, 9000, 64, True),
    (24, 24, 100, 3100, 3000, 1, 3100, 0, True),
    (12, 4, 1374, 5496, 4122, 1374, 4, 1374, True),  # a view over three others, one key group, over 4
    (16, 16, 1374, 6870, 5496, 1374, 4, 1374, True),
]
# 512 to 1,199 blocks: two key groups where edges of large frames lie inside blocks, else one (frames of 768, all in reach).
FRAMES = [
    (64, 16, 1100, 1100, 0, 1000, 1, 0, True),
    (64, 64, 1100, 2500, 1100, 930, 2, 100, True),
    (32, 8, 2100, 2900, 500, 1010, 1, 5, False),
    (64, 64, 1100, 2500, 1024, 768, 2, 100, True),
    (64, 64, 1600, 1600, 0, 1600, 1, 5, False),
    (64, 8, 1000, 2000, 1000, 1000, 1, 700, True),
]
# Lists of queries in many slices: of sinks alone, of all.
SLICES = [
    (1, 1, 4000, 300, 0, 1, 5000, 300, False),
    (2, 2, 8000, 128, 0, 1, 1, 128, True),
    (1, 1, 3000, 3000, 0, 1, 700, 1, True),
    (4, 1, 2000, 200, 0, 1, 2000, 64, True),
    (2, 1, 5000, 600, 0, 1, 6000, 0, True),
]
# One key a query, by the sinks or the first position alone: dq and dk are what float32 leaves of 0.
ONE = [(2, 2, 100, 64, 500, 1, 3, 1, True), (4, 2, 1, 50, 0, 1, 7, 0, True)]


@pytest.fixture(scope="module")
def ress():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_35593_amd as r

    return r


@pytest.mark.parametrize("shape", CUTS + FRAMES + SLICES)
def test_forward(ress, shape):
    H, H_kv, n_q, n_k = shape[:4]
    say(f"[plans] {shape}")
    q, k, v, _ = _inputs(n_q + n_k, H, H_kv, n_q, n_k)
    kw = _kw(*shape[4:])
    o, lse, w, mag = R.window(q, k, v, R.visible(n_q, n_k, *shape[4:], device="cuda"))
    r = ress.ress_window_attn(q, k, v, want_lse=True, **kw)
    R.within(r["o"], o, R.window_bound(o, w, mag), "o")
    R.within(r["lse"], lse, 2.0 ** -18 * (mag + 1) + 2.0 ** -22 * lse.abs(), "lse")
    r2 = ress.ress_window_attn(q, k, v, **kw)["o"]
    R.within(r2, o, R.window_bound(o, w, mag), "o without lse")
    # A workspace of the caller's, of any contents, gives the same bits.
    size = ress.ress_window_attn_workspace_size(H, H_kv, n_q, n_k, **kw)
    assert (size > 0) == (shape in CUTS)
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(ress.ress_window_attn(q, k, v, workspace=ws, **kw)["o"], r2)


@pytest.mark.parametrize("shape", CUTS[-2:] + FRAMES + SLICES + ONE)
def test_backward(ress, shape):
    H, H_kv, n_q, n_k = shape[:4]
    say(f"[plans bwd] {shape}")
    q, k, v, do = _inputs(n_q * 3 + n_k, H, H_kv, n_q, n_k)
    kw = _kw(*shape[4:])
    f = ress.ress_window_attn(q, k, v, want_lse=True, **kw)
    ws = torch.full((ress.ress_window_attn_bwd_workspace_size(H, H_kv, n_q, n_k, **kw),), 255, dtype=torch.uint8, device="cuda")
    g = ress.ress_window_attn_bwd(do, q, k, v, f["o"], f["lse"], workspace=ws, **kw)
    dq, dk, dv, bq, bk, bv = R.window_bwd(do, q, k, v, R.visible(n_q, n_k, *shape[4:], device="cuda"))
    R.within(g["dv"], dv, bv, "dv")
    R.within(g["dk"], dk, bk, "dk")
    R.within(g["dq"], dq, bq, "dq")
    again = ress.ress_window_attn_bwd(do, q, k, v, f["o"], f["lse"], **kw)
    assert all(torch.equal(again[n], g[n]) for n in g)


@pytest.mark.parametrize("shape", [CUTS[1], CUTS[-1], FRAMES[0]])
def test_captured_replays(ress, shape):
    """Forward and backward in a graph, workspaces made inside the capture, replayed with eager calls of the same between: the
    eager call's bits on every replay."""
    H, H_kv, n_q, n_k = shape[:4]
    q, k, v, do = _inputs(5, H, H_kv, n_q, n_k)
    kw = _kw(*shape[4:])

    def step():
        f = ress.ress_window_attn(q, k, v, want_lse=True, **kw)
        return dict(f, **ress.ress_window_attn_bwd(do, q, k, v, f["o"], f["lse"], **kw))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        out = step()
    for rep in range(3):
        q.mul_(-1)
        for t in out.values():
            t.fill_(7)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[n], t) for n, t in step().items()), rep


@pytest.mark.parametrize("amp", [10.0, 60.0])
def test_backward_of_large_logits(ress, amp):
    """Logits of +-100 to +-1000: the probabilities that are formed again keep within the bound of their logits. Those below
    2^-126 lose digits to bf16's and float32's smallest steps, half of 2^-133 each: 300 terms of factors up to 300 are off by
    2^-134 2^17 at most, well below 2^-112."""
    q, k, v, do = _inputs(21, 4, 2, 300, 300, amp)
    kw = _kw(0, 1, 200, 4, True)
    f = ress.ress_window_attn(q, k, v, want_lse=True, **kw)
    g = ress.ress_window_attn_bwd(do, q, k, v, f["o"], f["lse"], **kw)
    dq, dk, dv, bq, bk, bv = R.window_bwd(do, q, k, v, R.visible(300, 300, 0, 1, 200, 4, True, device="cuda"))
    R.within(g["dv"], dv, bv + 2.0 ** -112, "dv")
    R.within(g["dk"], dk, bk + 2.0 ** -112, "dk")
    R.within(g["dq"], dq, bq + 2.0 ** -112, "dq")
