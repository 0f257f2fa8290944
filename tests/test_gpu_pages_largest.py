"""The largest sizes of include/ress_pages.h: 2^24 tokens, 65,535 sequences, caches of 2^24 tokens."""
import math

import pytest
import torch

import layer_refs as R
import pages_refs as PR
from gpu_helpers import say
from layer_refs import within

pytestmark = pytest.mark.gpu

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32
MOST = 65535


@pytest.fixture(scope="module")
def ress():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_35593_amd as r

    return r


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def test_heads_of_the_most_tokens(ress):
    """Sampled rows against float64; the weights' gradients of a gradient that is zero but for some rows."""
    N = 1 << 24
    say("[largest] heads")
    q = torch.randn(1, N, 64, generator=_gen(1), device="cuda").to(BF)
    pos = torch.arange(N, device="cuda", dtype=I32)[:, None]
    at = torch.cat([torch.arange(50, device="cuda"), torch.randint(0, N, (500,), generator=_gen(2), device="cuda"),
                    torch.arange(N - 50, N, device="cuda")])
    r = ress.ress_qk_norm_rope(q, None, pos, dims=(32,))
    y, b = PR.heads(q[:, at], pos[at], None, None, "layer", 1e-5, (32,), "split", 100.0)
    within(r["q"][:, at], y, b, "q")
    del r
    at = at.unique()
    dq = torch.zeros_like(q)
    dq[:, at] = torch.randn(1, len(at), 64, generator=_gen(3), device="cuda").to(BF)
    g = ress.ress_qk_norm_rope_bwd(dq, None, q, None, pos, dims=(32,))
    ref, bounds = PR.heads_bwd(dq[:, at], q[:, at], pos[at], None, "layer", 1e-5, (32,), "split", 100.0)
    within(g["dq"][:, at], ref[0], bounds[0], "dq")
    for n, want, bound in zip(("q_dgamma", "q_dbeta"), ref[1:], bounds[1:]):
        within(g[n], want, bound, n)
    assert g["dq"].count_nonzero() == g["dq"][:, at].count_nonzero()


def test_tables_of_the_most_sequences(ress):
    say("[largest] tables")
    page, max_pages = 4, 9
    g = torch.Generator().manual_seed(4)
    lens = torch.randint(0, 30, (MOST,), generator=g)
    new = torch.randint(0, 4, (MOST,), generator=g)
    had, have = -(-lens // page), -(-(lens + new) // page)
    n_pages = int(have.sum()) + 9
    order = torch.randperm(n_pages, generator=g)
    first = had.cumsum(0) - had
    at = torch.arange(max_pages)
    table = torch.where(at < had[:, None], order[(first[:, None] + at).clamp(max=n_pages - 1)], -1)
    n_free = n_pages - int(had.sum())
    free = torch.cat([order[int(had.sum()):], torch.full((int(had.sum()),), -1)])
    for cut in (0, 1000):  # (all of them, and all but those behind a stack that ends)
        rows = table.tolist()
        N = int(new.sum()) + 5
        want = PR.tables(lens.tolist(), new.tolist(), rows, free.tolist(), n_free - 9 - cut, page, N)
        t = table.int().cuda()
        r = ress.ress_page_tables(lens.int().cuda(), new.int().cuda(), t, free.int().cuda(),
                                  torch.tensor([n_free - 9 - cut], dtype=I32, device="cuda"), page=page, tokens=N)
        for n, x in want.items():
            assert torch.equal(r[n].cpu(), torch.tensor(x, dtype=I32)), (n, cut)
        assert torch.equal(t.cpu(), torch.tensor(rows, dtype=I32))
        assert (want["n_refused"][0] > 0) == (cut > 0)
    d_free, n = free.int().cuda(), torch.tensor([want["n_free"][0]], dtype=I32, device="cuda")
    stack = free.tolist()
    height = PR.release([1] * MOST, [max_pages] * MOST, rows, stack, want["n_free"][0], True)
    zero = torch.zeros(MOST, dtype=I32, device="cuda")
    out = ress.ress_pages_release(zero + 1, zero + max_pages, t, d_free, n)
    assert out.tolist() == [height] and torch.equal(d_free.cpu(), torch.tensor(stack, dtype=I32))
    assert torch.equal(t.cpu(), torch.tensor(rows, dtype=I32))


def test_lists_of_the_most_tokens(ress):
    """One sequence of 2^24 tokens in pages of one token, from nothing."""
    N = 1 << 24
    say("[largest] lists")
    free = torch.randperm(N, generator=_gen(5), device="cuda").int()
    t = torch.full((1, N), -1, dtype=I32, device="cuda")
    z = torch.zeros(1, dtype=I32, device="cuda")
    r = ress.ress_page_tables(z, z + N, t, free, z + N, page=1, tokens=N)
    assert r["lens"].item() == N and r["n_free"].item() == 0 and r["n_refused"].item() == 0 and r["cu_q"].tolist() == [0, N]
    assert torch.equal(t[0], free.flip(0)) and torch.equal(r["slots"], t[0])
    assert torch.equal(r["pos"], torch.arange(N, device="cuda", dtype=I32))
    stack = torch.zeros(N, dtype=I32, device="cuda")
    assert ress.ress_pages_release(z, z + N, t, stack, z).item() == N and torch.equal(stack, free.flip(0)) and (t == -1).all()


@pytest.mark.parametrize("H,H_kv", [(2, 1), (64, 1)])
def test_attention_of_the_most_sequences(ress, H, H_kv):
    """One new token of each of 65,535 sequences of up to 7 tokens; as blocks of 32 rows and of 128."""
    say(f"[largest] sequences, {H} heads")
    page, width = 4, 2
    g = _gen(6)
    lens = torch.randint(1, 8, (MOST,), generator=g, device="cuda")
    n_pages = 1000
    k, v = (torch.randn(n_pages, H_kv, page, 64, generator=g, device="cuda").to(BF) for _ in range(2))
    tables = torch.randint(0, n_pages, (MOST, width), generator=g, device="cuda", dtype=I32)
    q = torch.randn(H, MOST, 64, generator=g, device="cuda").to(BF)
    cu = torch.arange(MOST + 1, device="cuda", dtype=I32)
    o = ress.ress_paged_attn(q, k, v, cu, lens.int(), tables, window=5)["o"]
    s = torch.arange(page * width, device="cuda")
    rows = tables[:, s // page].long() * page + s % page
    kk, vv = (x[:, 0].reshape(-1, 64)[rows].double() for x in (k, v))
    vis = (s < lens[:, None]) & (s >= lens[:, None] - 5)
    for h in range(0, H, max(1, H // 2)):
        qd = q[h].double()
        x = torch.where(vis, (kk * qd[:, None]).sum(2) / 8.0, -math.inf)
        p = torch.softmax(x, 1)[:, :, None]
        ref, w = (p * vv).sum(1), (p * vv.abs()).sum(1)
        mag = torch.where(vis, (kk.abs() * qd.abs()[:, None]).sum(2) / 8.0, 0.0).amax(1)
        within(o[h], ref, R.window_bound(ref, w, mag), "o")


@pytest.mark.parametrize("H", [1, 64])
def test_the_longest_cache(ress, H):
    """2^24 tokens in pages of 64, one new token: the last pages far behind 2^31 bytes; every key seen. Keys are few
    different rows, so that the float64 form has them counted."""
    n, page, kinds = 1 << 24, 64, 256
    say(f"[largest] cache, {H} heads")
    g = _gen(7)
    kk, vv = (torch.randn(kinds, 64, generator=g, device="cuda").to(BF) for _ in range(2))
    kind = torch.randint(0, kinds, (n,), generator=g, device="cuda")
    n_pages = n // page
    tables = torch.randperm(n_pages, generator=g, device="cuda").int()[None]
    back = torch.empty(n_pages, dtype=torch.long, device="cuda")
    back[tables[0].long()] = torch.arange(n_pages, device="cuda")
    k, v = (x[kind.view(n_pages, page)[back]][:, None].contiguous() for x in (kk, vv))
    q = torch.randn(H, 1, 64, generator=g, device="cuda").to(BF)
    cu, lens = (torch.tensor(x, dtype=I32, device="cuda") for x in ([0, 1], [n]))
    r = ress.ress_paged_attn(q, k, v, cu, lens, tables, window=1 << 30, want_lse=True)
    count = torch.bincount(kind, minlength=kinds).double()
    x = q[:, 0].double() @ kk.double().T / 8.0 + count.log()
    p = torch.softmax(x, 1)
    ref, w = p @ vv.double(), p @ vv.double().abs()
    mag = (q[:, 0].double().abs() @ kk.double().abs().T / 8.0).amax(1)
    # (2^18 tiles of a row, in parts of 2^11 at most: sums of 2^24 weights in float32 add 2^-12 of w)
    within(r["o"][:, 0], ref, R.window_bound(ref, w, mag) + 2.0 ** -12 * w, "o")
    lse = torch.logsumexp(x, 1)
    within(r["lse"][:, 0], lse, 2.0 ** -18 * (mag + 1) + 2.0 ** -22 * lse.abs() + 2.0 ** -12, "lse")


def test_the_last_slots(ress):
    """Slots up to 2^31 - 2, of a cache with more tokens than it has memory for: pages that share their rows."""
    page = 1 << 20
    n_pages = 2047
    k = torch.randn(1, 3, 64, generator=_gen(8), device="cuda").to(BF)
    pages = torch.zeros(page, 64, dtype=BF, device="cuda")
    pos = torch.zeros(3, 1, dtype=I32, device="cuda")
    shared = pages.expand(n_pages, 1, page, 64)
    slots = torch.tensor([n_pages * page - 1, 5, n_pages * page], dtype=I32, device="cuda")
    with pytest.raises(ress.RessError):  # (an output that overlaps itself)
        ress.ress_qk_norm_rope_pages(None, k, k, pos, slots, shared, shared, dims=(64,))
    big = torch.zeros(1, 1, (1 << 24), 64, dtype=BF, device="cuda")
    out = torch.zeros_like(big)
    slots = torch.tensor([(1 << 24) - 1, 1 << 24, 0], dtype=I32, device="cuda")
    ress.ress_qk_norm_rope_pages(None, k, k, pos, slots, big, out, dims=(64,))
    assert torch.equal(out[0, 0, -1], k[0, 0]) and torch.equal(out[0, 0, 0], k[0, 2]) and out.count_nonzero() == 128


@pytest.mark.parametrize("B", [3, 1500])
def test_a_stack_of_more_than_2_28_pages(ress, B):
    """Pages given back to, and taken from, heights beyond 2^28, and a stack that is full before the last entry."""
    say("[largest] stack", B)
    n_pages = (1 << 28) + 5 * B
    height = n_pages - 4 * B
    free = torch.zeros(n_pages, dtype=I32, device="cuda")
    want = torch.arange(5 * B, dtype=I32, device="cuda") * 7 + n_pages - 40 * B
    tables = torch.full((B, 8), -1, dtype=I32, device="cuda")
    tables[:, 1:6] = want.view(B, 5)
    first, last = (torch.full((B,), i, dtype=I32, device="cuda") for i in (0, 8))
    n_free = torch.full((1,), height, dtype=I32, device="cuda")
    out = ress.ress_pages_release(first, last, tables, free, n_free)
    assert out.tolist() == [n_pages]  # a fifth of the entries has no room
    assert torch.equal(free[height:], want[:4 * B]) and not free[:1000].any() and free[height - 1000:height].count_nonzero() == 0
    assert (tables == -1).all()
    # Two tokens of each sequence, on pages of one: from the top of the stack down.
    r = ress.ress_page_tables(torch.zeros_like(first), torch.full_like(first, 2), tables, free, out, page=1, tokens=2 * B)
    assert r["n_free"].tolist() == [n_pages - 2 * B] and r["n_refused"].tolist() == [0]
    taken = want[:4 * B].flip(0)[:2 * B]
    assert torch.equal(tables[:, :2].reshape(-1), taken) and torch.equal(r["slots"], taken)
    # The first of each goes back.
    out = ress.ress_pages_release(torch.zeros_like(first), torch.full_like(first, 1), tables, free, r["n_free"])
    assert out.tolist() == [n_pages - B] and torch.equal(free[n_pages - 2 * B:n_pages - B], taken.view(B, 2)[:, 0])
