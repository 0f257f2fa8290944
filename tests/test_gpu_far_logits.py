"""Windowed attention of logits far beyond what a float32 softmax resolves: products that float32 holds exactly, so that the
largest logit is known, and every weight is that of the definition."""
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


def _whole(seed, power, *shape):
    """Integers from -3 to 3 times 2^power: sums of 64 products of two of them have at most 10 bits."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randint(-3, 4, (*shape, 64), generator=g, device="cuda") * 2.0 ** power).to(BF)


def _values(seed, *shape):
    return torch.randn(*shape, 64, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(BF)


def _reference(q, k, v, vis, scale=0.125):
    """o, lse, sum p |v| of one K/V head per query head's group, from logits relative to the row's largest: the float64 log-sum
    itself does not resolve them."""
    o, lse, w = [], [], []
    for h in range(q.shape[0]):
        hk = h * k.shape[0] // q.shape[0]
        x = torch.where(vis, q[h].double() @ k[hk].double().T, -torch.inf)
        m = x.amax(1, keepdim=True)
        p = torch.where(vis, torch.exp((x - torch.where(vis.any(1, keepdim=True), m, 0.0)) * scale), 0.0)
        total = p.sum(1, keepdim=True)
        p = p / torch.where(total == 0, 1.0, total)
        o.append(p @ v[hk].double())
        w.append(p @ v[hk].double().abs())
        lse.append((m * scale + torch.log(total))[:, 0])
    return torch.stack(o), torch.stack(lse), torch.stack(w)


# H, H_kv, n_q, n_k, q_offset, frame, window, n_sink, causal: one, two and four key groups, keys split over workgroups
SHAPES = [
    (2, 2, 500, 500, 0, 100, 2, 100, True),
    (3, 1, 200, 200, 0, 1, 64, 4, False),
    (1, 1, 33, 700, 667, 1, 700, 0, True),
    (1, 1, 1, 5000, 4999, 1, 5000, 0, True),
    (8, 4, 1100, 4800, 3700, 1, 3650, 10, True),
    (64, 16, 2050, 2050, 0, 1, 300, 70, True),
]


@pytest.mark.parametrize("power", [8, 20, 28, 32, 40, 64, 110])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(ress, shape, power):
    """Logits 2^(power - 3) apart at least: a row is the mean of the values of its largest ones. From 2^28 on (2^25 a unit in
    base 2) their weights are 1 exactly, so only sums (2^-18 of sum p |v|) and the output (2^-8) round; below, where the
    scaled reference is rounded, a weight is 2^e with e of up to half a unit, and its own rounding to bf16 shows: 2^-8 of
    each term and of the sum. lse: the reference in base 2, its scale and ln 2 are rounded to float32, five times 2^-24 at most."""
    H, H_kv, n_q, n_k = shape[:4]
    say(f"[far] {shape} 2^{power}")
    q, k, v = _whole(1, power // 2, H, n_q), _whole(2, power - power // 2, H_kv, n_k), _values(3, H_kv, n_k)
    kw = dict(zip(("q_offset", "frame", "window", "n_sink", "causal"), shape[4:]))
    o, lse, w = _reference(q, k, v, R.visible(n_q, n_k, *shape[4:], device="cuda"))
    bound = 2.0 ** -8 * o.abs() + 2.0 ** -18 * w if power >= 28 else 2.0 ** -8 * (w + 2 * o.abs()) + 2.0 ** -12 * w
    R.within(ress.ress_window_attn(q, k, v, **kw)["o"], o, bound, "o")
    r = ress.ress_window_attn(q, k, v, want_lse=True, **kw)
    R.within(r["o"], o, bound, "o beside lse")
    R.within(r["lse"], lse, 2.0 ** -21 * lse.abs() + 2.0 ** -18, "lse")


@pytest.mark.parametrize("shape", SHAPES)
def test_forward_about_the_turn(ress, shape):
    """Logits that lie a few units (natural) about 2^24 in base 2, where references begin to be kept unscaled: products are
    whole multiples of 8 below 2^27, which float32 holds, a unit of the logit each. Parts of a row on both sides are joined.
    Weights are of ordinary sizes: probabilities rounded to bf16 for their product, sums, the output."""
    H, H_kv, n_q, n_k = shape[:4]
    at = int(2.0 ** 24 / (0.125 * 1.4426950408889634)) // 8 * 8 - 104  # the largest of a tile is some 13 units above
    q, k = torch.zeros(H, n_q, 64, device="cuda"), torch.zeros(H_kv, n_k, 64, device="cuda")
    bits = [b for b in range(27) if at >> b & 1]
    assert len(bits) <= 24 and min(bits) >= 3
    for c, b in enumerate(bits):
        q[..., c], k[..., c] = 2.0 ** (b // 2), 2.0 ** (b - b // 2)
    g = torch.Generator(device="cuda").manual_seed(5)
    q[..., 24:] = torch.randint(0, 2, (H, n_q, 40), generator=g, device="cuda") * 16.0 - 8.0
    k[..., 24:] = torch.randint(-1, 2, (H_kv, n_k, 40), generator=g, device="cuda")
    q, k, v = q.to(BF), k.to(BF), _values(6, H_kv, n_k)
    kw = dict(zip(("q_offset", "frame", "window", "n_sink", "causal"), shape[4:]))
    o, lse, w = _reference(q, k, v, R.visible(n_q, n_k, *shape[4:], device="cuda"))
    bound = 2.0 ** -8 * (w + 2 * o.abs()) + 2.0 ** -12 * w
    R.within(ress.ress_window_attn(q, k, v, **kw)["o"], o, bound, "o")
    r = ress.ress_window_attn(q, k, v, want_lse=True, **kw)
    R.within(r["o"], o, bound, "o beside lse")
    R.within(r["lse"], lse, 2.0 ** -21 * lse.abs() + 2.0 ** -18, "lse")


@pytest.mark.parametrize("scale", [1e35, 2e30, 2.0 ** 27, 1e-38, 1e-44])
def test_forward_scales(ress, scale):
    """The largest scales leave the largest logits, the smallest the mean of the visible values."""
    q, k, v = _whole(7, 0, 2, 300), _whole(8, 0, 2, 300), _values(9, 2, 300)
    vis = R.visible(300, 300, 0, 1, 200, 5, True, device="cuda")
    o, _, w = _reference(q, k, v, vis, scale)
    R.within(ress.ress_window_attn(q, k, v, window=200, n_sink=5, scale=scale)["o"], o,
             2.0 ** -8 * (w + 2 * o.abs()) + 2.0 ** -12 * w, "o")


def _decode(ress, q, k, v, lens, kw, scale=None):
    """The output, and o and sum p |v| of every sequence's last position."""
    t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    got = ress.ress_window_attn_decode(q, k, v, t, scale=scale, **kw)
    ref = []
    for i, n in enumerate(lens):
        vis = R.visible(1, n, n - 1, 1, kw["window"], kw["n_sink"], True, device="cuda")
        o, _, w = _reference(q[i][:, None], k[i, :, :n], v[i, :, :n], vis, 0.125 if scale is None else scale)
        ref.append((o[:, 0], w[:, 0]))
    return got, torch.stack([o for o, _ in ref]), torch.stack([w for _, w in ref])


# B, H, H_kv, capacity, window, n_sink: a head a K/V head and shared ones, in one workgroup and cut over several
CACHES = [(3, 2, 2, 400, 300, 5), (1, 4, 4, 9000, 9000, 0), (3, 8, 2, 400, 300, 5), (1, 40, 1, 9000, 5000, 64)]


@pytest.mark.parametrize("power", [8, 20, 28, 32, 40, 64, 110])
@pytest.mark.parametrize("cache", CACHES)
def test_decode(ress, cache, power):
    """As in the forward pass; references are taken from the scores, so weights are 1 at any size, and no weight is rounded
    to bf16 (2^-16 of it at most is lost)."""
    B, H, H_kv, cap, window, n_sink = cache
    say(f"[far decode] {cache} 2^{power}")
    q, k, v = _whole(11, power // 2, B, H), _whole(12, power - power // 2, B, H_kv, cap), _values(13, B, H_kv, cap)
    got, o, w = _decode(ress, q, k, v, [cap - 7 * i for i in range(B)], dict(window=window, n_sink=n_sink))
    R.within(got, o, 2.0 ** -8 * o.abs() + 2.0 ** -16 * w, "o")
    # All logits far below zero: the least of them are the largest.
    got, o, w = _decode(ress, -q.abs(), k.abs() + k.abs().amax(), v, [cap - 7 * i for i in range(B)],
                        dict(window=window, n_sink=n_sink))
    R.within(got, o, 2.0 ** -8 * o.abs() + 2.0 ** -16 * w, "o, all far below zero")


@pytest.mark.parametrize("scale", [1e35, 2e30, 2.0 ** 27, 1e-38, 1e-44])
@pytest.mark.parametrize("cache", CACHES)
def test_decode_scales(ress, cache, scale):
    B, H, H_kv, cap, window, n_sink = cache
    q, k, v = _whole(14, 0, B, H), _whole(15, 0, B, H_kv, cap), _values(16, B, H_kv, cap)
    got, o, w = _decode(ress, q, k, v, [cap - 7 * i for i in range(B)], dict(window=window, n_sink=n_sink), scale)
    R.within(got, o, 2.0 ** -8 * o.abs() + 2.0 ** -12 * w, "o")
