"""The weights of attention over pages sum to one as they enter the product with the values, with and without the logarithm of
their sum: values that are all alike come out as they are."""
import pytest
import torch

import pages_refs as PR
from gpu_helpers import say
from layer_refs import within

pytestmark = pytest.mark.gpu

BF, I32 = torch.bfloat16, torch.int32


@pytest.fixture(scope="module")
def ress():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_35593_amd as r

    return r


def _t(x):
    return torch.tensor(x, dtype=I32, device="cuda")


@pytest.mark.parametrize("page", [13, 16])
@pytest.mark.parametrize("H,H_kv,lens,new", [(2, 1, [700], [1]), (1, 1, [9000], [3]), (4, 2, [300, 64, 500], [300, 50, 130]),
                                             (1, 1, [6000], [200]), (8, 2, [9000, 40, 3000], [150, 40, 70])])
def test_values_that_are_all_alike(ress, H, H_kv, lens, new, page):
    """Every 64th key's probability is 1 of the row's reference and the others' 0.50193, which bf16 rounds down by 2^-8 of itself:
    by a sum of unrounded ones the output would be off by nearly that, where 2^-9 reaches the next bf16 number. Float32 leaves
    2^-11 (sums of 9,000 terms at worst), so the outputs are the values, bit for bit."""
    say(f"[paged weights] H {H}/{H_kv} lens {lens} new {new} page {page}")
    counts = [-(-n // page) for n in lens]
    n_pages, most = sum(counts) + 1, max(counts) + 1
    g = torch.Generator(device="cuda").manual_seed(page)
    order = torch.randperm(n_pages, generator=g, device="cuda").int()
    tables, at = torch.full((len(lens), most), -1, dtype=I32, device="cuda"), 0
    k = torch.zeros(n_pages, H_kv, page, 64, dtype=BF, device="cuda")
    for b, n in enumerate(counts):
        tables[b, :n] = order[at:at + n]
        s = torch.arange(0, lens[b], 64, device="cuda")
        k[tables[b, s // page].long(), :, s % page, 0] = 1.0
        at += n
    c = (1 + (127 - 3 * torch.arange(64, device="cuda") % 128) / 128.0).to(BF)  # from the top of a power of two down
    assert c[0] == 255 / 128
    v = c.expand(k.shape).contiguous()
    cu = [sum(new[:i]) for i in range(len(new) + 1)]
    q = torch.zeros(H, cu[-1], 64, dtype=BF, device="cuda")
    q[..., 0] = 1.0
    args = (q, k, v, _t(cu), _t(lens), tables)
    scale = 0.6893  # exp(-scale) = 0.50193
    _, lse, _, bl, _ = PR.paged(q, k, v, cu, lens, tables, 1, 10 ** 9, 0, scale)
    for want in (False, True):
        r = ress.ress_paged_attn(*args, window=10 ** 9, scale=scale, want_lse=want)
        assert torch.equal(r["o"], c.expand(r["o"].shape)), f"logarithm wanted: {want}"
        if want:
            within(r["lse"], lse, bl, "lse")


def test_outputs_are_the_same_with_the_logarithm(ress):
    """Where keys are not cut, bit for bit."""
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(60, 2, 16, 64, generator=g, device="cuda").to(BF) for _ in range(2))
    q = (2 * torch.randn(4, 400, 64, generator=g, device="cuda")).to(BF)
    tables = torch.randperm(60, generator=g, device="cuda").int().view(2, 30)
    args = (q, k, v, _t([0, 250, 400]), _t([450, 400]), tables)
    a = ress.ress_paged_attn(*args, window=300, n_sink=5)
    b = ress.ress_paged_attn(*args, window=300, n_sink=5, want_lse=True)
    assert torch.equal(a["o"], b["o"])
