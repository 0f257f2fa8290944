"""Rotary positions against float64: layouts, types, strides, far positions, in place."""
import pytest
import torch

import layer_refs as R
from gpu_helpers import say

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ress():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_35593_amd as r

    return r


def _inputs(seed, H, H_kv, N, D, axes, dtype, far=1000):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, k = (torch.randn(h, N, D, generator=g, device="cuda").to(dtype) for h in (H, H_kv))
    pos = torch.randint(-far, far + 1, (N, axes), generator=g, device="cuda", dtype=torch.int32)
    return q, k, pos


def _check(got, x, pos, dims, layout, base, inverse=False):
    ref = R.rope(x, pos, dims, layout, base, inverse)
    R.within(got, ref, R.rope_bound(x, ref, pos, dims, layout, base), layout)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("layout", ["split", "interleaved", "sections"])
@pytest.mark.parametrize("D,dims", [(64, (32, 32)), (64, (64,)), (64, (16, 24, 24)), (64, (16, 16)), (64, (20, 20, 24)),
                                    (64, (8, 8)), (128, (32, 48, 32)), (256, (64, 64, 64, 64)), (2, (2,)), (6, (2, 2)),
                                    (48, (16, 16, 16)), (64, (0, 32)), (64, (0,)), (80, (48, 16))])
def test_layouts(ress, D, dims, layout, dtype):
    say(f"[rope] D {D} {dims} {layout} {dtype}")
    for H, H_kv, N in ((3, 1, 77), (1, 5, 1), (9, 2, 300), (2, 7, 20000), (2, 1, 130)):
        q, k, pos = _inputs(D + N, H, H_kv, N, D, len(dims), dtype)
        for inverse in (False, True):
            r = ress.ress_rope(q, k, pos, dims=dims, layout=layout, base=1e4, inverse=inverse)
            _check(r["q"], q, pos, dims, layout, 1e4, inverse)
            _check(r["k"], k, pos, dims, layout, 1e4, inverse)
            if sum(dims) < D:  # copied bit for bit
                assert torch.equal(r["q"][..., sum(dims):], q[..., sum(dims):])


@pytest.mark.parametrize("layout", ["split", "sections"])
def test_far_positions_keep_their_phase(ress, layout):
    q, k, pos = _inputs(1, 2, 2, 500, 64, 2, F32, far=1 << 24)
    r = ress.ress_rope(q, k, pos, dims=(32, 32), layout=layout, base=100.0)
    _check(r["q"], q, pos, (32, 32), layout, 100.0)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("dims", [(32, 32), (20, 24)])
def test_strides_and_in_place(ress, dims, dtype):
    """Token-major inputs, an output inside a cache, odd strides, in place: the values of the contiguous call; what lies
    around an output stays."""
    H, N, D = 4, 150, 64
    q, k, pos = _inputs(2, H, H, N, D, 2, dtype)
    ref = ress.ress_rope(q, k, pos, dims=dims, base=100.0)
    tm = torch.stack([q, k], 1).permute(2, 1, 0, 3).contiguous()  # [N][2][H][D]
    cache = torch.full((H, N + 40, D), 7.0, device="cuda").to(dtype)
    r = ress.ress_rope(tm[:, 0].transpose(0, 1), tm[:, 1].transpose(0, 1), pos, dims=dims, base=100.0,
                       k_out=cache[:, 13:13 + N])
    assert torch.equal(r["q"], ref["q"]) and torch.equal(cache[:, 13:13 + N], ref["k"])
    assert bool((cache[:, :13] == 7).all()) and bool((cache[:, 13 + N:] == 7).all())
    odd = torch.zeros(H, N, D + 3, device="cuda").to(dtype)[..., 1:D + 1]
    odd.copy_(q)
    assert torch.equal(ress.ress_rope(odd, None, pos, dims=dims, base=100.0)["q"], ref["q"])
    z = tm.clone()
    v = z[:, 0].transpose(0, 1)
    ress.ress_rope(v, None, pos, dims=dims, base=100.0, q_out=v)
    assert torch.equal(v, ref["q"]) and torch.equal(z[:, 1], tm[:, 1])


@pytest.mark.parametrize("layout", ["split", "interleaved", "sections"])
def test_copied_channels_keep_nan_and_infinity(ress, layout):
    q, _, pos = _inputs(3, 2, 1, 30, 64, 2, BF)
    q[..., 32:] = float("inf")
    q[..., 50] = float("nan")
    y = ress.ress_rope(q, None, pos, dims=(16, 16), layout=layout)["q"]
    assert torch.equal(y[..., 32:].view(torch.int16), q[..., 32:].view(torch.int16))
    assert bool(torch.isfinite(y[..., :32]).all())


def test_inverse_is_the_gradient(ress):
    """<turn(x), y> = <x, turn back(y)>: float32, 64 products of magnitude 1 a token, each within 2^-20."""
    x, y, pos = _inputs(4, 3, 3, 100, 64, 2, F32)
    a = ress.ress_rope(x, None, pos, dims=(32, 32))["q"].double() * y.double()
    b = x.double() * ress.ress_rope(y, None, pos, dims=(32, 32), inverse=True)["q"].double()
    mag = (x.double().abs().sum(2) * y.double().abs().amax(2))
    assert bool(((a.sum(2) - b.sum(2)).abs() <= 2.0 ** -19 * mag).all())


def test_no_tokens(ress):
    q, k, pos = _inputs(5, 2, 2, 0, 64, 2, BF)
    r = ress.ress_rope(q, k, pos, dims=(32, 32))
    assert r["q"].shape == (2, 0, 64)
