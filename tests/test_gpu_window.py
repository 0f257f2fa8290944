"""Windowed attention, forward and backward, against float64: frames, windows, sinks, offsets, shared heads, strides,
empty rows, odd lengths."""
import pytest
import torch

import layer_refs as R
from gpu_helpers import say

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32

# H, H_kv, n_q, n_k, q_offset, frame, window, n_sink, causal
SHAPES = [
    (1, 1, 1, 1, 0, 1, 1, 0, True),
    (2, 1, 1, 700, 699, 1, 100, 0, True),
    (4, 2, 5, 300, 295, 7, 3, 9, True),
    (2, 2, 127, 127, 0, 1, 1000, 0, True),
    (2, 2, 129, 129, 0, 1, 33, 0, True),
    (3, 1, 200, 200, 0, 1, 64, 4, True),
    (2, 2, 500, 500, 0, 100, 2, 0, True),
    (2, 2, 500, 500, 0, 100, 2, 100, True),
    (2, 1, 500, 500, 0, 37, 1, 65, False),
    (2, 2, 333, 333, 0, 1, 20, 0, False),
    (2, 2, 333, 333, 0, 1, 1, 0, False),
    (2, 2, 260, 1000, 700, 64, 2, 130, True),
    (4, 4, 260, 900, 100, 50, 3, 5, False),
    (2, 2, 300, 200, 0, 10, 2, 0, True),       # queries behind the keys, some see nothing
    (2, 2, 300, 200, 150, 10, 2, 3, True),     # ... or the sinks only
    (2, 2, 100, 64, 500, 10, 3, 0, True),      # no query sees anything
    (2, 1, 50, 0, 0, 1, 5, 2, True),           # no keys
    (2, 2, 190, 190, 0, 1374, 4, 1374, True),  # one frame
    (2, 2, 400, 400, 0, 1, 2 ** 31 - 1, 2 ** 31 - 1, True),
    (2, 2, 300, 300, 0, 2 ** 31 - 1, 1, 0, False),
    (2, 1, 130, 130, 0, 2 ** 31 - 1, 2 ** 31 - 1, 0, False),
    (2, 1, 0, 150, 0, 1, 10, 3, True),         # no queries
    (6, 2, 1100, 1100, 0, 1, 30, 5, False),    # the sinks' queries cut into slices, the others' not
    (1, 1, 2500, 2500, 0, 1, 2500, 0, True),   # every block's queries cut, keys split over workgroups
    (8, 1, 150, 150, 0, 1, 50, 1, True),
    (2, 2, 1400, 1400, 0, 300, 2, 300, True),
    (2, 2, 700, 700, 0, 1, 90, 650, True),     # sinks beyond most windows
    (2, 2, 100, 100, 300, 1, 10, 80, True),    # the sinks only, keys behind them in their last tile
    (2, 2, 2500, 2500, 0, 1, 100, 5, True),    # the sinks' queries alone cut
    (8, 4, 1100, 4800, 3700, 1, 3650, 10, True),  # long lists, cut over workgroups
    (16, 4, 1100, 4800, 3700, 1, 3650, 10, True),
    (3, 3, 1000, 3900, 2900, 1, 3000, 5, True),
    (64, 16, 2050, 2050, 0, 1, 300, 70, True),  # workgroups for several fillings: one key group a workgroup
    (64, 64, 2050, 2050, 0, 100, 3, 100, True),
    (64, 8, 2050, 2050, 0, 1, 90, 3, False),
]


@pytest.fixture(scope="module")
def ress():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_35593_amd as r

    return r


def _inputs(seed, H, H_kv, n_q, n_k, amp=1.0):
    """A mean that keys and values share, as real ones have."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    mk = lambda h, n, a, m: (torch.randn(h, n, 64, generator=g, device="cuda") * a
                             + m * torch.randn(h, 1, 64, generator=g, device="cuda")).to(BF)
    return mk(H, n_q, amp, 0.0), mk(H_kv, n_k, 1.0, 0.7), mk(H_kv, n_k, 0.7, 0.3), mk(H, n_q, 1.0, 0.0)


def _kw(q_offset, frame, window, n_sink, causal):
    return dict(q_offset=q_offset, frame=frame, window=window, n_sink=n_sink, causal=causal)


@pytest.mark.parametrize("shape", SHAPES)
def test_forward(ress, shape):
    H, H_kv, n_q, n_k = shape[:4]
    say(f"[window] {shape}")
    q, k, v, _ = _inputs(n_q + n_k, H, H_kv, n_q, n_k)
    vis = R.visible(n_q, n_k, *shape[4:], device="cuda")
    r = ress.ress_window_attn(q, k, v, want_lse=True, **_kw(*shape[4:]))
    o, lse, w, mag = R.window(q, k, v, vis)
    R.within(r["o"], o, R.window_bound(o, w, mag), "o")
    R.within(r["lse"], lse, 2.0 ** -18 * (mag + 1) + 2.0 ** -22 * lse.abs(), "lse")
    assert not r["o"][:, ~vis.any(1)].any()  # zeros, exactly
    r2 = ress.ress_window_attn(q, k, v, **_kw(*shape[4:]))
    R.within(r2["o"], o, R.window_bound(o, w, mag), "o without lse")
    assert torch.equal(ress.ress_window_attn(q, k, v, **_kw(*shape[4:]))["o"], r2["o"])


@pytest.mark.parametrize("amp", [10.0, 60.0])
def test_large_logits(ress, amp):
    """Logits of +-100 to +-1000: the references move, and nothing overflows."""
    q, k, v, _ = _inputs(3, 2, 2, 400, 400, amp)
    kw = _kw(0, 1, 300, 4, True)
    vis = R.visible(400, 400, 0, 1, 300, 4, True, device="cuda")
    o, lse, w, mag = R.window(q, k, v, vis)
    r = ress.ress_window_attn(q, k, v, want_lse=True, **kw)
    R.within(r["o"], o, R.window_bound(o, w, mag), "o")
    R.within(r["lse"], lse, 2.0 ** -18 * (mag + 1) + 2.0 ** -22 * lse.abs(), "lse")


def test_rising_logits_move_the_reference(ress):
    """Every later tile outweighs all before it by far more than float32's range allows against one reference."""
    q, k, v, _ = _inputs(4, 1, 1, 128, 640)
    k *= (torch.arange(640, device="cuda") // 64 * 30.0 + 1.0)[None, :, None].to(BF)
    vis = R.visible(128, 640, 512, 1, 640, 0, True, device="cuda")
    o, lse, w, mag = R.window(q, k, v, vis)
    r = ress.ress_window_attn(q, k, v, want_lse=True, **_kw(512, 1, 640, 0, True))
    R.within(r["o"], o, R.window_bound(o, w, mag), "o")
    R.within(r["lse"], lse, 2.0 ** -18 * (mag + 1) + 2.0 ** -22 * lse.abs(), "lse")


def test_scale(ress):
    q, k, v, _ = _inputs(5, 2, 2, 100, 100)
    vis = R.visible(100, 100, 0, 1, 30, 0, True, device="cuda")
    o, _, w, mag = R.window(q, k, v, vis, scale=0.3)
    R.within(ress.ress_window_attn(q, k, v, scale=0.3, **_kw(0, 1, 30, 0, True))["o"], o, R.window_bound(o, w, mag))


def test_unseen_keys_may_hold_anything(ress):
    """NaN and infinities in keys that no query of a 128-query block sees have no part in it: behind the window, between
    sinks and window, and, in a cache, behind the last key."""
    q, k, v, _ = _inputs(6, 2, 2, 100, 1000)
    kw = _kw(800, 1, 128, 5, True)  # the block sees [0, 5) and [673, 900)
    ref = ress.ress_window_attn(q, k, v, **kw)["o"]
    for t in (k, v):
        t[:, 5:673] = float("nan")
        t[:, 900:950] = float("inf")
        t[:, 950:] = float("nan")
    assert torch.equal(ress.ress_window_attn(q, k, v, **kw)["o"], ref)
    # ... also where sinks and window share a tile of 64 keys: the block sees [0, 5) and [40, 199).
    q, k, v, do = _inputs(6, 2, 2, 60, 300)
    kw = _kw(139, 1, 100, 5, True)
    ref = ress.ress_window_attn(q, k, v, want_lse=True, **kw)
    gref = ress.ress_window_attn_bwd(do, q, k, v, ref["o"], ref["lse"], **kw)
    for t in (k, v):
        t[:, 5:40] = float("nan")
        t[:, 199:] = float("inf")
    got = ress.ress_window_attn(q, k, v, want_lse=True, **kw)
    grad = ress.ress_window_attn_bwd(do, q, k, v, got["o"], got["lse"], **kw)
    assert torch.equal(got["o"], ref["o"]) and torch.equal(got["lse"], ref["lse"]) and torch.equal(grad["dq"], gref["dq"])
    # ... and where every window lies behind the keys, and the sinks end inside the last tile.
    q, k, v, do = _inputs(6, 2, 2, 60, 100)
    kw = _kw(300, 1, 10, 80, True)
    ref = ress.ress_window_attn(q, k, v, want_lse=True, **kw)
    gref = ress.ress_window_attn_bwd(do, q, k, v, ref["o"], ref["lse"], **kw)
    for t in (k, v):
        t[:, 80:] = float("nan")
    got = ress.ress_window_attn(q, k, v, want_lse=True, **kw)
    grad = ress.ress_window_attn_bwd(do, q, k, v, got["o"], got["lse"], **kw)
    assert torch.equal(got["o"], ref["o"]) and torch.equal(got["lse"], ref["lse"]) and torch.equal(grad["dq"], gref["dq"])
    # A NaN key inside only spoils the queries that see it.
    q, k, v, _ = _inputs(6, 1, 1, 300, 300)
    kw = _kw(0, 100, 1, 0, True)
    ref = ress.ress_window_attn(q, k, v, **kw)["o"]
    k[:, 150] = float("nan")
    o = ress.ress_window_attn(q, k, v, **kw)["o"]
    assert torch.equal(o[:, :100], ref[:, :100]) and torch.equal(o[:, 200:], ref[:, 200:]) and bool(o[:, 100:200].isnan().all())


def test_unseen_queries_may_hold_anything(ress):
    """Queries that see none of a block of 128 keys have no part in the block's gradients, whatever they and their
    gradients hold: keys 0 .. 127 are seen by queries 0 .. 146 alone."""
    q, k, v, do = _inputs(13, 2, 1, 500, 500)
    kw = _kw(0, 1, 20, 0, True)
    f = ress.ress_window_attn(q, k, v, want_lse=True, **kw)
    ref = ress.ress_window_attn_bwd(do, q, k, v, f["o"], f["lse"], **kw)
    q[:, 147:] = float("nan")
    do[:, 147:] = float("inf")
    f = ress.ress_window_attn(q, k, v, want_lse=True, **kw)
    got = ress.ress_window_attn_bwd(do, q, k, v, f["o"], f["lse"], **kw)
    assert torch.equal(got["dk"][:, :128], ref["dk"][:, :128]) and torch.equal(got["dv"][:, :128], ref["dv"][:, :128])
    assert torch.equal(got["dq"][:, :128], ref["dq"][:, :128])


def test_dense_window_matches_dense_attention(ress):
    """A window over everything is the library's dense attention: both within their bounds of the same values."""
    q, k, v, _ = _inputs(7, 4, 4, 700, 700)
    vis = torch.ones(700, 700, dtype=torch.bool, device="cuda")
    o, _, w, mag = R.window(q, k, v, vis)
    a = ress.ress_window_attn(q, k, v, window=1, frame=700, causal=False)["o"]
    b = ress.ress_dense_attn(q, k, v, bq=128, bk=128)
    R.within(a, o, R.window_bound(o, w, mag))
    # The dense kernel also rounds Q times the scale to bf16: 2^-8 of a logit's magnitude, both sides of the quotient.
    R.within(b, o, R.window_bound(o, w, mag) + 2.0 ** -7 * mag[..., None] * w)


@pytest.mark.parametrize("shape", [(4, 2, 300, 300, 0, 1, 70, 5, True), (4, 4, 130, 500, 370, 60, 2, 60, True),
                                   (2, 2, 260, 260, 0, 30, 2, 0, False)])
def test_strides(ress, shape):
    """Token-major tensors, slices of a packed projection, outputs inside larger buffers, broadcast K/V heads: the bits of
    the contiguous call, forward and backward; what lies around the outputs stays."""
    H, H_kv, n_q, n_k = shape[:4]
    q, k, v, do = _inputs(8, H, H_kv, n_q, n_k)
    kw = _kw(*shape[4:])
    ref = ress.ress_window_attn(q, k, v, want_lse=True, **kw)
    gref = ress.ress_window_attn_bwd(do, q, k, v, ref["o"], ref["lse"], **kw)

    def inside(t, value=3.0):  # [tokens + 8][heads + 1][72], token-major
        buf = torch.full((t.shape[1] + 8, t.shape[0] + 1, 72), value, device="cuda", dtype=t.dtype)
        view = buf[3:3 + t.shape[1], 1:, :64].transpose(0, 1)
        view.copy_(t)
        return buf, view

    (_, q2), (_, k2), (_, v2), (_, do2) = (inside(t) for t in (q, k, v, do))
    ob, o2 = inside(torch.zeros_like(q))
    r = ress.ress_window_attn(q2, k2, v2, out=o2, want_lse=True, **kw)
    assert torch.equal(o2, ref["o"]) and torch.equal(r["lse"], ref["lse"])
    bufs = {n: inside(torch.zeros_like(t)) for n, t in (("dq", q), ("dk", k), ("dv", v))}
    g = ress.ress_window_attn_bwd(do2, q2, k2, v2, o2, r["lse"], **{n: b[1] for n, b in bufs.items()}, **kw)
    for n in ("dq", "dk", "dv"):
        assert torch.equal(g[n], gref[n]), n
        bufs[n][1].fill_(3.0)
        assert bool((bufs[n][0] == 3).all()), n
    o2.fill_(3.0)
    assert bool((ob == 3).all())
    one = k[:1].expand(H_kv, -1, -1)  # a head stride of 0
    assert torch.equal(ress.ress_window_attn(q, one, one, **kw)["o"],
                       ress.ress_window_attn(q, one.contiguous(), one.contiguous(), **kw)["o"])


def test_offsets_beyond_32_bits(ress):
    """Rows 2^16 elements apart, 40,000 of them: 5.2 GB of key and value each behind one pointer."""
    q, k, v, _ = _inputs(9, 2, 1, 200, 40000)
    kw = _kw(39800, 1, 500, 70, True)
    ref = ress.ress_window_attn(q, k, v, **kw)["o"]
    far = []
    for t in (k, v):
        buf = torch.empty(40000, 1 << 16, dtype=BF, device="cuda")
        view = buf[:, :64][None]
        view.copy_(t)
        far.append(view)
    assert torch.equal(ress.ress_window_attn(q, *far, **kw)["o"], ref)
    lens = torch.tensor([40000], dtype=torch.int32, device="cuda")
    for heads in (2, 1):
        a = ress.ress_window_attn_decode(q[:heads, -1][None], k[None], v[None], lens, window=500, n_sink=70)
        b = ress.ress_window_attn_decode(q[:heads, -1][None], far[0][None], far[1][None], lens, window=500, n_sink=70)
        assert torch.equal(a, b)


@pytest.mark.parametrize("shape", SHAPES)
def test_backward(ress, shape):
    H, H_kv, n_q, n_k = shape[:4]
    say(f"[window bwd] {shape}")
    q, k, v, do = _inputs(n_q * 3 + n_k, H, H_kv, n_q, n_k)
    kw = _kw(*shape[4:])
    vis = R.visible(n_q, n_k, *shape[4:], device="cuda")
    f = ress.ress_window_attn(q, k, v, want_lse=True, **kw)
    nan = {n: torch.full_like(t, float("nan")) for n, t in (("dq", q), ("dk", k), ("dv", v))}
    g = ress.ress_window_attn_bwd(do, q, k, v, f["o"], f["lse"], **nan, **kw)
    dq, dk, dv, bq, bk, bv = R.window_bwd(do, q, k, v, vis)
    R.within(g["dv"], dv, bv, "dv")
    R.within(g["dk"], dk, bk, "dk")
    R.within(g["dq"], dq, bq, "dq")
    assert not g["dq"][:, ~vis.any(1)].any() and not g["dk"][:, ~vis.any(0)].any() and not g["dv"][:, ~vis.any(0)].any()
    again = ress.ress_window_attn_bwd(do, q, k, v, f["o"], f["lse"], **kw)
    assert all(torch.equal(again[n], g[n]) for n in g)


@pytest.mark.parametrize("shape", [(4, 2, 1, 1, 0, 1, 7, 1, False), (3, 1, 200, 200, 0, 1, 1, 0, True),
                                   (2, 2, 150, 150, 0, 1, 1, 0, False), (4, 4, 90, 1, 0, 50, 1, 0, True)])
def test_one_key_has_no_gradient_of_its_logit(ress, shape):
    """A softmax over one key is 1: dq and dk are zero exactly, dv is d_o of the queries that see the key."""
    H, H_kv, n_q, n_k = shape[:4]
    q, k, v, do = _inputs(77, H, H_kv, n_q, n_k)
    kw = _kw(*shape[4:])
    f = ress.ress_window_attn(q, k, v, want_lse=True, **kw)
    g = ress.ress_window_attn_bwd(do, q, k, v, f["o"], f["lse"], **kw)
    vis = R.visible(n_q, n_k, *shape[4:], device="cuda")
    assert not g["dq"].any() and not g["dk"].any()
    _, _, dv, _, _, bv = R.window_bwd(do, q, k, v, vis)
    R.within(g["dv"], dv, bv, "dv")


def test_backward_keeps_small_gradients_beside_a_common_key(ress):
    """Keys with a mean far above their spread: dq is what is left of sums that nearly cancel, and stays within its bound
    (delta taken from the rounded o alone would leave that mean times the rounding in it)."""
    g = torch.Generator(device="cuda").manual_seed(12)
    q, v, do = (torch.randn(2, 400, 64, generator=g, device="cuda").to(BF) for _ in range(3))
    k = (torch.randn(2, 400, 64, generator=g, device="cuda") * 0.25 + 4.0).to(BF)
    kw = _kw(0, 1, 200, 0, False)
    vis = R.visible(400, 400, 0, 1, 200, 0, False, device="cuda")
    f = ress.ress_window_attn(q, k, v, want_lse=True, **kw)
    r = ress.ress_window_attn_bwd(do, q, k, v, f["o"], f["lse"], **kw)
    dq, _, _, bq, _, _ = R.window_bwd(do, q, k, v, vis)
    R.within(r["dq"], dq, bq, "dq")
    # ds is rounded to bf16 (2^-8 at most, uniform: 2^-9.8 rms), 400 terms of random sign with keys of size 4 against
    # gradients of spread 0.25: 16 times 2^-9.8, less than 3%.
    assert float((r["dq"].double() - dq).norm() / dq.norm()) < 0.03
