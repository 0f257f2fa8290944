"""Slots between 2^24 and 2^31 - 2, the last that a cache can have: keys and values of few channels, in pages of 2^20 tokens."""
import pytest
import torch

from gpu_helpers import say

pytestmark = pytest.mark.gpu

I32 = torch.int32


@pytest.mark.parametrize("D,layout", [(2, "split"), (4, "interleaved")])
@pytest.mark.parametrize("page", [1 << 20, (1 << 20) - 3])
def test_far_slots(D, layout, page):
    """By pairs of channels and by chunks; pages of a power of two tokens and others. 2,047 pages take 8.6 GB for K and for V with two
    channels. What is written is found in its row, and nothing else is."""
    import paper_2609_35593_amd as ress

    say(f"[far slots] D {D} page {page}")
    n_pages = (2 ** 31 - 1) // page
    top = n_pages * page
    where = [top - 1, top - 2, top - page, top - page - 1, 1 << 30, (1 << 30) + 1, (1 << 30) - 1, (1 << 29) + page // 2, 1 << 24, 0]
    none = [top, 2 ** 31 - 1, -1]  # (the first behind the end, the largest number, no slot)
    assert top <= 2 ** 31 - 1 and where[0] > 2 ** 31 - 2 ** 21 and len(set(where)) == len(where)
    none = [s for s in none if not 0 <= s < top]
    N = len(where) + len(none)
    g = torch.Generator(device="cuda").manual_seed(page)
    k, v = (torch.randn(1, N, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    assert k.count_nonzero() == v.count_nonzero() == N * D
    pos = torch.arange(N, device="cuda", dtype=I32)[:, None]
    kp, vp = (torch.zeros(n_pages, 1, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ress.ress_qk_norm_rope_pages(None, k, v, pos, torch.tensor(none + where, dtype=I32, device="cuda"), kp, vp, dims=(D,), layout=layout)
    want = ress.ress_qk_norm_rope(None, k, pos, dims=(D,), layout=layout)["k"]
    at = torch.tensor(where, device="cuda")
    n = len(none)
    for pages, rows in ((kp, want), (vp, v)):
        assert torch.equal(pages[at // page, 0, at % page], rows[0, n:])
        pages[at // page, 0, at % page] = 0.0
        assert not any(bool(part.any()) for part in pages.split(64))
