"""The largest sizes that include/ress_layer.h allows, where they fit the card: grids, counters and offsets at their ends.
Compared on rows at the beginning, in the middle and at the end; what is computed alike for every row is compared whole."""
import pytest
import torch

import layer_refs as R
from gpu_helpers import say

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
N = 1 << 24


@pytest.fixture(scope="module")
def ress():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_35593_amd as r

    return r


@pytest.fixture(autouse=True)
def _free():
    yield
    torch.cuda.empty_cache()


def _rand(*shape, seed=0, dtype=BF):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda", dtype=dtype)


def test_norm_of_most_rows(ress):
    """2^31 - 1 rows of one channel: each its own mean, y is beta, gradients of x are zero."""
    rows = (1 << 31) - 1
    say(f"[largest] norm {rows} rows")
    x, beta = torch.empty(rows, 1, dtype=BF, device="cuda"), torch.tensor([3.0], device="cuda")
    x.view(-1).copy_(torch.arange(997, device="cuda").to(BF).repeat(rows // 997 + 1)[:rows])
    f = ress.ress_layer_norm(x, None, beta, want_stats=True)
    assert bool((f["y"] == 3).all())
    for part in (slice(0, 5000), slice(rows // 2, rows // 2 + 5000), slice(rows - 5000, rows)):
        assert torch.equal(f["mean"][part], x[part, 0].float())
    del f["y"]
    dy = torch.ones(rows, 1, dtype=BF, device="cuda")
    b = ress.ress_layer_norm_bwd(dy, x, None, f["mean"], f["rstd"])
    assert not b["dx"].any() and not b["dgamma"].any()
    # dbeta counts the rows: a lane's sum of ones, 2^31 / 2^17 lanes at most 2^14 each, is exact, and 2^31 - 1 rounds to 2^31
    assert abs(float(b["dbeta"]) - rows) <= 2.0 ** (31 - 20)


def test_far_rows_of_norm(ress):
    """Rows 2^30 elements apart."""
    buf = torch.empty(5 * (1 << 30), dtype=BF, device="cuda")
    x = buf.view(5, 1 << 30)[:, 7:1031]
    x.copy_(_rand(5, 1024))
    dense = x.contiguous()
    a, b = ress.ress_layer_norm(x, want_stats=True), ress.ress_layer_norm(dense, want_stats=True)
    R.within(a["y"], *(lambda y: (y, 2.0 ** -8 * y.abs() + 2.0 ** -16))(R.norm(dense, None, None, 1e-5)[0]), "y")
    ga = ress.ress_layer_norm_bwd(b["y"], x, None, a["mean"], a["rstd"], dx=x)
    gb = ress.ress_layer_norm_bwd(b["y"], dense, None, b["mean"], b["rstd"])
    R.within(ga["dgamma"], gb["dgamma"].double(), 2.0 ** -16 * (1 + gb["dgamma"].double().abs()), "dgamma")


@pytest.mark.parametrize("D,dims,layout", [(64, (32, 32), "split"), (256, (250,), "split"), (256, (256,), "interleaved")])
def test_rope_of_most_tokens(ress, D, dims, layout):
    say(f"[largest] rope {N} tokens of {D}")
    x = _rand(1, N, D)
    pos = torch.randint(-(1 << 31), (1 << 31) - 1, (N, len(dims)), device="cuda", dtype=torch.int64).to(torch.int32)
    y = ress.ress_rope(x, None, pos, dims=dims, layout=layout, base=1e4)["q"]
    for at in (0, N // 2 - 300, N - 600):
        part = slice(at, at + 600)
        ref = R.rope(x[:, part], pos[part], dims, layout, 1e4)
        # the angle of far positions, beside the bound's own: 2^-23 of a turn, and 2^-21 of a radian in the float64 form, whose
        # frequency and product are rounded to 2^-53 of 2^31 radians: below 2^-19 together
        mag = torch.zeros_like(ref)
        for _, _, a, b in R.rope_pairs(dims, layout, 1e4):
            mag[..., a] = mag[..., b] = x[:, part, a].double().abs() + x[:, part, b].double().abs()
        R.within(y[:, part], ref, R.rope_bound(x[:, part], ref, pos[part], dims, layout, 1e4) + 2.0 ** -19 * mag, "y")
    back = ress.ress_rope(y, None, pos, dims=dims, layout=layout, base=1e4, inverse=True)["q"]
    # two roundings of at most 2^-8 of a pair's length, below 8 sqrt(2)
    assert float((back.float() - x.float()).abs().max()) < 2.0 ** -3


def test_far_tokens_of_rope(ress):
    """Tokens 2^21 elements apart, 3,000 of them: 12.6 GB behind one pointer, in place."""
    buf = torch.empty(3000, 1 << 21, dtype=BF, device="cuda")
    k = buf[:, 64:128][None]
    k.copy_(_rand(1, 3000, 64))
    pos = torch.arange(3000, device="cuda", dtype=torch.int32)[:, None]
    ref = ress.ress_rope(None, k.contiguous(), pos, dims=(64,))["k"]
    assert torch.equal(ress.ress_rope(None, k, pos, dims=(64,), k_out=k)["k"], ref)


def test_window_of_most_tokens(ress):
    """2^24 queries behind position 2^24 over 2^24 keys, of which the window sees a part and the sinks the rest, and from
    position 0."""
    q, k, v, do = (_rand(1, N, 64, seed=s) for s in range(4))
    for off, window, n_sink in ((0, 100, 3), (N, 70, 5), (N, N + 50, 0)):
        say(f"[largest] window {N} tokens behind {off}")
        kw = dict(window=window, n_sink=n_sink, q_offset=off)
        if off and window > N:  # (all keys for the first queries, fewer later: few rows, long lists)
            rows = 128
            f = ress.ress_window_attn(q[:, :rows], k, v, want_lse=True, **kw)
            assert torch.isfinite(f["lse"]).all() and torch.isfinite(f["o"].float()).all()
            # means of 2^24 values of spread 1: weights are even to a factor of e^4, the mean within 2^-9
            assert float(f["o"].float().abs().max()) < 2.0 ** -4
            continue
        f = ress.ress_window_attn(q, k, v, want_lse=True, **kw)
        g = ress.ress_window_attn_bwd(do, q, k, v, f["o"], f["lse"], **kw)
        for at in (0, N // 2 - 100, N - 200):
            # the keys that these rows see, as a small problem: sinks, and those from the first window's start on
            rows = slice(at, at + 200)
            lo = min(max(off + at - window + 1, n_sink), N)
            keys = torch.cat([torch.arange(n_sink, device="cuda"), torch.arange(lo, min(off + at + 200, N), device="cuda")])
            p = torch.arange(at, at + 200, device="cuda")[:, None] + off
            vis = (keys <= p) & ((keys > p - window) | (keys < n_sink))
            o, lse, w, mag = R.window(q[:, rows], k[:, keys], v[:, keys], vis)
            R.within(f["o"][:, rows], o, R.window_bound(o, w, mag), "o")
            R.within(f["lse"][:, rows], lse, 2.0 ** -18 * (mag + 1) + 2.0 ** -22 * lse.abs(), "lse")
            dq, _, _, bq, _, _ = R.window_bwd(do[:, rows], q[:, rows], k[:, keys], v[:, keys], vis)
            R.within(g["dq"][:, rows], dq, bq, "dq")
        if off == 0:  # the last keys are seen by the last queries alone
            rows, keys = slice(N - 250, N), slice(N - 150, N)
            vis = R.visible(250, 250, 0, 1, window, 0, True, device="cuda")
            vis = torch.cat([torch.ones(250, n_sink, dtype=torch.bool, device="cuda"), vis], 1)
            kk, vv = torch.cat([k[:, :n_sink], k[:, rows]], 1), torch.cat([v[:, :n_sink], v[:, rows]], 1)
            _, dk, dv, _, bk, bv = R.window_bwd(do[:, rows], q[:, rows], kk, vv, vis)
            R.within(g["dk"][:, keys], dk[:, -150:], bk[:, -150:], "dk")
            R.within(g["dv"][:, keys], dv[:, -150:], bv[:, -150:], "dv")


@pytest.mark.parametrize("H", [1, 2])
def test_decode_of_the_longest_cache(ress, H):
    say(f"[largest] decode {N} tokens, {H} heads for 1")
    q, k, v = _rand(1, H, 64, seed=1), _rand(1, 1, N, 64, seed=2), _rand(1, 1, N, 64, seed=3)
    lens = torch.tensor([N], dtype=torch.int32, device="cuda")
    for window, n_sink in ((300, 7), (N, 0)):
        o = ress.ress_window_attn_decode(q, k, v, lens, window=window, n_sink=n_sink)
        x = (q[0].double() @ k[0, 0].double().T) / 8.0
        if window < N:
            x[:, n_sink:N - window] = -torch.inf
        p = torch.softmax(x, 1)
        ref, w = p @ v[0, 0].double(), p @ v[0, 0].double().abs()
        # a lane adds up to 2^16 weights, whose roundings have either sign: 2^8 2^-24 of their sum, with room
        R.within(o[0], ref, 2.0 ** -8 * ref.abs() + 2.0 ** -11 * w, "o")
        del x, p


@pytest.mark.parametrize("H,H_kv", [(1, 1), (2, 1)])
def test_decode_of_most_sequences(ress, H, H_kv):
    B = 65535
    q, k, v = _rand(B, H, 64, seed=1), _rand(B, H_kv, 3, 64, seed=2), _rand(B, H_kv, 3, 64, seed=3)
    lens = torch.arange(B, device="cuda", dtype=torch.int32) % 4
    o = ress.ress_window_attn_decode(q, k, v, lens, window=2, n_sink=0)
    x = (q.double()[:, :, None] * k.double()).sum(-1) / 8.0  # [B][H][3]
    t = torch.arange(3, device="cuda")[None]
    vis = (t < lens[:, None]) & (t >= lens[:, None] - 2)
    p = torch.where(vis[:, None], torch.exp(x - x.amax(-1, keepdim=True)), 0.0)
    p = p / p.sum(-1, keepdim=True).clamp_min(1e-300)
    ref = (p[..., None] * v.double()).sum(2)
    w = (p[..., None] * v.double().abs()).sum(2)
    R.within(o, ref, 2.0 ** -8 * ref.abs() + 2.0 ** -11 * w, "o")
    assert not o[lens == 0].any()
