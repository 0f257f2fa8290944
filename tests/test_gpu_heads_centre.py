"""The norm of heads subtracts the mean from the values, not from their products: rows far from zero, whose means float32 holds
exactly, keep every digit of what is left."""
import pytest
import torch

import pages_refs as PR
from gpu_helpers import say
from layer_refs import HALF, rope, within

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
# Widths whose inverse, and with these rows whose sums, float32 holds exactly; the last ones by pairs of channels.
WIDTHS = [(64, (32, 32)), (64, (8, 8)), (128, (32, 48, 32)), (256, (64, 64, 64, 64)), (64, (4, 4)), (64, (20, 20, 24)), (256, (62, 64))]


@pytest.fixture(scope="module")
def ress():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_35593_amd as r

    return r


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(kind, H, N, D, dtype, seed):
    """Whole numbers, rows of one value or of values near one: sums below 2^24, so means and what is left of the values are exact."""
    at = torch.tensor([1000.0, -4096.0, 3.0, 60000.0 if D == 64 else 30000.0, 0.0, 7168.0], device="cuda")
    x = at[torch.arange(N, device="cuda") % len(at)][None, :, None].repeat(H, 1, D)
    x = x.to(dtype).float()
    if kind == "near":
        step = 1.0 if dtype is F32 else 512.0  # (of bf16 at 60,000 and less: whole numbers too)
        x = (x + step * torch.randint(-3, 4, (H, N, D), generator=_gen(seed), device="cuda")).to(dtype).float()
    assert x.sum(-1).abs().max() < 2 ** 24 and torch.equal(x, x.round())
    return x.to(dtype)


def _check(y, x, pos, gamma, beta, dims, layout, what):
    """Half a step of the output, and of each term 2^-19 as in pages_refs.heads (rstd 12 2^-24 of itself, products, weights and
    coefficients 6 2^-24, a cosine or sine 2^-22); nothing for the mean, which is exact."""
    g, b = gamma.double(), beta.double()
    xh, _ = PR._norm(x, "layer", 1e-5)
    ref = rope(xh * g + b, pos, dims, layout, 1e4)
    within(y, ref, HALF[x.dtype] * ref.abs() + 2.0 ** -19 * PR._meet(xh.abs() * g.abs() + b.abs(), dims, layout), what)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("layout", ["split", "interleaved", "sections"])
@pytest.mark.parametrize("D,dims", WIDTHS)
def test_rows_far_from_zero(ress, D, dims, layout, dtype):
    say(f"[heads far from zero] D {D} {dims} {layout} {dtype}")
    H, H_kv, N, page = 6, 1, 130, 16
    pos = torch.randint(-1000, 1001, (N, len(dims)), generator=_gen(1), device="cuda", dtype=torch.int32)
    rn = lambda s: torch.randn(D, generator=_gen(s), device="cuda")
    w = dict(q_gamma=1 + 0.3 * rn(2), q_beta=0.2 * rn(3), k_gamma=1 + 0.3 * rn(4), k_beta=0.2 * rn(5))
    kw = dict(dims=dims, layout=layout, base=1e4, **w)
    for kind in ("one value", "near"):
        q, k = _rows(kind, H, N, D, dtype, 6), _rows(kind, H_kv, N, D, dtype, 7)
        odd = torch.empty(H, N, D + 3, dtype=dtype, device="cuda")[..., 1:D + 1]  # (pairs of channels, whatever the axes)
        odd.copy_(q)
        for name, x in (("chunks", q), ("odd strides", odd)):
            r = ress.ress_qk_norm_rope(x, k, pos, **kw)
            _check(r["q"], q, pos, w["q_gamma"], w["q_beta"], dims, layout, f"q {name} {kind}")
            _check(r["k"], k, pos, w["k_gamma"], w["k_beta"], dims, layout, f"k {name} {kind}")
        slots = torch.randperm(160, generator=_gen(8), device="cuda")[:N].int()
        kp, vp = (torch.zeros(10, H_kv, page, D, dtype=dtype, device="cuda") for _ in range(2))
        r = ress.ress_qk_norm_rope_pages(q, k, k, pos, slots, kp, vp, **kw)
        at = slots.long()
        _check(r["q"], q, pos, w["q_gamma"], w["q_beta"], dims, layout, f"q of pages {kind}")
        _check(kp[at // page, :, at % page].transpose(0, 1), k, pos, w["k_gamma"], w["k_beta"], dims, layout, f"k into pages {kind}")
