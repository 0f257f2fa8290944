"""Layer norm of values near the ends of what include/ress_layer.h allows: squares up to 2^112, their sums below 2^127."""
import pytest
import torch

import layer_refs as R

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ress():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_35593_amd as r

    return r


@pytest.mark.parametrize("xt", [F32, BF])
@pytest.mark.parametrize("width", [64, 16384])
def test_large_values(ress, width, xt):
    """As ordinary rows, which a power of two does not change: mean and sums within 81 steps of 2^-24 of sums of magnitudes
    (means near 0 here), 2^-17 of everything that has size 1; the output's half step."""
    g = torch.Generator(device="cuda").manual_seed(width)
    u = torch.rand(9, width, generator=g, device="cuda") * 2 - 1
    x = (u * 2.0 ** 56).to(xt)
    dy = torch.randn(9, width, generator=g, device="cuda")
    f = ress.ress_layer_norm(x, out_dtype=F32, want_stats=True)
    y, mean, rstd = R.norm(x, None, None, 1e-5)
    R.within(f["y"], y, 2.0 ** -17, "y")
    R.within(f["mean"], mean, 2.0 ** (56 - 17), "mean")
    R.within(f["rstd"], rstd, 2.0 ** -17 * rstd, "rstd")
    b = ress.ress_layer_norm_bwd(dy, x, None, f["mean"], f["rstd"])
    dx, dg, db = R.norm_bwd(dy, x, None, f["mean"], f["rstd"])
    # rstd is at most 2^-54; |dy| < 6: dx is a sum of terms below 2^-50, each within 2^-17, rounded once
    R.within(b["dx"], dx, R.HALF[xt] * dx.abs() + 2.0 ** -67, "dx")
    R.within(b["dgamma"], dg, 2.0 ** -17 * (dy.abs().sum(0).double() * 2), "dgamma")
    R.within(b["dbeta"], db, 2.0 ** -17 * dy.abs().sum(0).double(), "dbeta")
