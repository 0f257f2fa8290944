"""One token over a cache against float64: lengths, sinks, frames, shared heads, layouts, captured calls."""
import math

import pytest
import torch

import layer_refs as R
from gpu_helpers import say

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


@pytest.fixture(scope="module")
def ress():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_35593_amd as r

    return r


def _inputs(seed, B, H, H_kv, cap, amp=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    mk = lambda *s: torch.randn(*s, 64, generator=g, device="cuda")
    return (mk(B, H) * amp).to(BF), mk(B, H_kv, cap).to(BF), (mk(B, H_kv, cap) + 0.3).to(BF)


def _reference(q, k, v, lens, frame, window, n_sink):
    """Per sequence, the windowed attention of its last position; the bound of the products and one rounding."""
    o, b = [], []
    for i, n in enumerate(lens):
        n = min(max(n, 0), k.shape[2])
        if n == 0:
            o.append(torch.zeros(q.shape[1], 64, dtype=torch.float64, device=q.device))
            b.append(torch.zeros_like(o[-1]))
            continue
        vis = R.visible(1, n, n - 1, frame, window, n_sink, True, device="cuda")
        x, _, w, mag = R.window(q[i][:, None], k[i, :, :n], v[i, :, :n], vis)
        o.append(x[:, 0])
        # float32 throughout: logits within 64 2^-24 mag, sums and weights within 2^-12, the output's rounding
        b.append((2.0 ** -8 * x.abs() + (2.0 ** -17 * mag[..., None] + 2.0 ** -12) * w)[:, 0])
    return torch.stack(o), torch.stack(b)


@pytest.mark.parametrize("H,H_kv", [(1, 1), (4, 4), (8, 4), (6, 2), (8, 1), (10, 2), (64, 4), (12, 1), (32, 2), (40, 1)])
@pytest.mark.parametrize("cap,frame,window,n_sink", [(1, 1, 1, 0), (63, 1, 1000, 0), (65, 1, 20, 3), (300, 10, 4, 17),
                                                     (1000, 1, 1, 0), (1500, 100, 3, 100), (2000, 1, 5000, 7)])
def test_lengths(ress, H, H_kv, cap, frame, window, n_sink):
    lens = sorted({0, 1, 2, cap // 3, cap // 2 + 1, cap - 1, cap, cap + 5, -3})
    say(f"[decode] H {H}/{H_kv} cap {cap} frame {frame} window {window} sinks {n_sink} lens {lens}")
    q, k, v = _inputs(cap + H, len(lens), H, H_kv, cap)
    t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    o = ress.ress_window_attn_decode(q, k, v, t, frame=frame, window=window, n_sink=n_sink)
    ref, b = _reference(q, k, v, lens, frame, window, n_sink)
    R.within(o, ref, b, "o")
    assert torch.equal(o, ress.ress_window_attn_decode(q, k, v, t, frame=frame, window=window, n_sink=n_sink))


@pytest.mark.parametrize("B,H,H_kv,cap", [(1, 16, 16, 30000), (1, 1, 1, 70000), (3, 16, 2, 9000), (40, 16, 4, 1500)])
def test_long_caches(ress, B, H, H_kv, cap):
    """Keys split over many workgroups."""
    q, k, v = _inputs(cap, B, H, H_kv, cap, 2.0)
    lens = [cap - 17 * i for i in range(B)]
    t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for frame, window, n_sink in ((1, cap, 0), (1374, 3, 1374), (1, 777, 5)):
        o = ress.ress_window_attn_decode(q, k, v, t, frame=frame, window=window, n_sink=n_sink)
        R.within(o, *_reference(q, k, v, lens, frame, window, n_sink), "o")


def test_large_logits(ress):
    q, k, v = _inputs(1, 2, 4, 2, 800, 60.0)
    t = torch.tensor([800, 333], dtype=torch.int32, device="cuda")
    o = ress.ress_window_attn_decode(q, k, v, t, window=10 ** 9)
    R.within(o, *_reference(q, k, v, [800, 333], 1, 10 ** 9, 0), "o")


@pytest.mark.parametrize("H_kv", [2, 8])
def test_unseen_keys_and_rows_around_the_output(ress, H_kv):
    """NaN behind the lengths and outside the windows has no part; an output inside a larger buffer leaves the rest."""
    q, k, v = _inputs(2, 3, 8, H_kv, 500)
    lens = [0, 140, 431]
    t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    kw = dict(window=60, n_sink=5)
    ref = ress.ress_window_attn_decode(q, k, v, t, **kw)
    for i, n in enumerate(lens):
        for x in (k, v):
            x[i, :, n:] = float("nan")
            x[i, :, min(5, n):max(0, n - 60)] = float("inf")
    buf = torch.full((5, 9, 80), 3.0, device="cuda").to(BF)
    out = buf[1:4, 1:, 8:72]
    got = ress.ress_window_attn_decode(q, k, v, t, out=out, **kw)
    assert torch.equal(got, ref) and not got[0].any()
    out.fill_(3.0)
    assert bool((buf == 3).all())


@pytest.mark.parametrize("H_kv", [2, 8])
def test_cache_layouts(ress, H_kv):
    """[B][capacity][heads][64] and slices of a buffer that holds keys and values."""
    q, k, v = _inputs(3, 4, 8, H_kv, 300)
    t = torch.tensor([300, 5, 77, 120], dtype=torch.int32, device="cuda")
    ref = ress.ress_window_attn_decode(q, k, v, t, window=100, n_sink=2)
    kv = torch.stack([k, v], 0).permute(1, 3, 0, 2, 4).contiguous()  # [B][capacity][2][heads][64]
    k2, v2 = (kv[:, :, i].transpose(1, 2) for i in range(2))
    q2 = q.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(ress.ress_window_attn_decode(q2, k2, v2, t, window=100, n_sink=2), ref)


def test_matches_the_prefill(ress):
    """The last row of ress_window_attn over the same keys, within both bounds."""
    q, k, v = _inputs(4, 1, 4, 2, 900)
    t = torch.tensor([900], dtype=torch.int32, device="cuda")
    kw = dict(frame=50, window=4, n_sink=60)
    a = ress.ress_window_attn_decode(q, k, v, t, **kw)[0]
    b = ress.ress_window_attn(q[0][:, None], k[0], v[0], q_offset=899, **kw)["o"][:, 0]
    vis = R.visible(1, 900, 899, 50, 4, 60, True, device="cuda")
    o, _, w, mag = R.window(q[0][:, None], k[0], v[0], vis)
    assert bool(((a.double() - b.double()).abs() <= 2 * R.window_bound(o, w, mag)[:, 0]).all())


@pytest.mark.parametrize("H,H_kv", [(8, 2), (4, 4)])
def test_captured_call_follows_the_lengths(ress, H, H_kv):
    """One graph, replayed while the cache grows: eager and replayed outputs are equal at every length."""
    B, cap = 3, 4000
    q, k, v = _inputs(5, B, H, H_kv, cap)
    lens = torch.tensor([3990, 1, 700], dtype=torch.int32, device="cuda")
    kw = dict(frame=1, window=3500, n_sink=8)
    ws = torch.empty(ress.ress_window_attn_decode_workspace_size(B, H, H_kv, cap, **kw), dtype=torch.uint8, device="cuda")
    assert ws.numel() > 0
    out = torch.empty_like(q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    ress.ress_window_attn_decode(q, k, v, lens, out=out, workspace=ws, stream=s, **kw)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        ress.ress_window_attn_decode(q, k, v, lens, out=out, workspace=ws, stream=s, **kw)
    for step in range(4):
        out.fill_(math.nan)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ress.ress_window_attn_decode(q, k, v, lens, **kw)), step
        lens += 3
        q.copy_(torch.randn(q.shape, device="cuda"))


def test_no_sequences(ress):
    q, k, v = _inputs(6, 0, 4, 2, 10)
    assert ress.ress_window_attn_decode(q, k, v, torch.empty(0, dtype=torch.int32, device="cuda"), window=3).shape == (0, 4, 64)
    q, k, v = _inputs(6, 2, 4, 2, 0)
    o = ress.ress_window_attn_decode(q, k, v, torch.zeros(2, dtype=torch.int32, device="cuda"), window=3)
    assert not o.any()
