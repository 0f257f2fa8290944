"""Tables, slots and positions of a step, and pages given back, against lists on the host (whole numbers, equal)."""
import pytest
import torch

import pages_refs as PR
from gpu_helpers import say

pytestmark = pytest.mark.gpu

I32 = torch.int32


@pytest.fixture(scope="module")
def ress():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_35593_amd as r

    return r


def _t(x):
    return torch.tensor(x, dtype=I32, device="cuda")


def _state(seed, B, page, max_pages, longest, spare, stride=None):
    """Lengths, tables of random pages that hold them, and a stack of the other pages."""
    g = torch.Generator().manual_seed(seed)
    lens = torch.randint(0, min(longest, page * max_pages) + 1, (B,), generator=g).tolist() if B else []
    n_pages = sum(-(-n // page) for n in lens) + spare
    order = torch.randperm(n_pages, generator=g).tolist()
    rows, at = [], 0
    for n in lens:
        m = -(-n // page)
        rows.append(order[at:at + m] + [-1] * (max_pages - m))
        at += m
    free = order[at:] + [-5] * at
    t = torch.full((B, stride or max_pages), -77, dtype=I32, device="cuda")
    if B:
        t[:, :max_pages] = _t(rows)
    return lens, rows, t, t[:, :max_pages], free, spare, g


def _check(ress, lens, new, rows, buf, tables, free, n_free, page, N, **kw):
    stride = buf.shape[1]
    want = PR.tables(lens, new, rows, free, n_free, page, N)
    r = ress.ress_page_tables(_t(lens), _t(new), tables, _t(free), _t([n_free]), page=page, tokens=N, **kw)
    for n, x in want.items():
        assert r[n].tolist() == x, n
    assert tables.tolist() == rows
    assert (buf[:, tables.shape[1]:] == -77).all() and buf.shape[1] == stride
    return r


@pytest.mark.parametrize("B,page,max_pages,longest,most,padding", [
    (1, 16, 4, 0, 1, 0), (1, 1, 300, 100, 200, 3), (3, 16, 40, 300, 50, 7), (256, 64, 20, 1000, 1, 0), (64, 7, 60, 300, 90, 11),
    (1023, 16, 8, 100, 3, 5), (1024, 16, 8, 100, 3, 0), (1025, 16, 8, 100, 3, 1), (5000, 4, 6, 20, 4, 1000),
    (2, 4096, 3, 5000, 3000, 0), (5, 64, 200, 9000, 3000, 100), (1, 128, 600, 10, 70000, 999)])
def test_steps(ress, B, page, max_pages, longest, most, padding):
    """Lists in one launch and in two, tables with rows further apart, sequences with no new tokens among them."""
    say(f"[tables] B {B} page {page} x {max_pages} longest {longest} new {most}")
    for seed in (0, 1):
        state = _state(seed + B, B, page, max_pages, longest, B * (most // page + 2) + 5, max_pages + 3 * seed)
        lens, rows, buf, tables, free, n_free, g = state
        new = [min(int(torch.randint(0, most + 1, (1,), generator=g)), page * max_pages - n) for n in lens]
        if B == 1:
            new = [min(most, page * max_pages - lens[0])]
        _check(ress, lens, new, rows, buf, tables, free, n_free, page, sum(new) + padding)


def test_no_room(ress):
    """A table that is too short, a list of tokens or a stack that ends, at the first, a middle and the last sequence."""
    for seed, (spare, short_n, huge) in enumerate(((0, 0, None), (3, 0, None), (9, 0, 2), (500, 7, None), (500, 100000, 0),
                                                   (1, 0, 39), (500, 0, 5))):
        lens, rows, buf, tables, free, n_free, g = _state(seed, 40, 4, 12, 30, spare)
        new = torch.randint(0, 9, (40,), generator=g).tolist()
        new[3], new[7] = -4, 0
        if huge is not None:
            new[huge] = 2 ** 31 - 1
        N = max(sum(n for n in new if 0 < n < 100) - short_n, 0)
        _check(ress, lens, new, rows, buf, tables, free, n_free, 4, N)
    # More than a turn of sequences behind the one that stops them, in both launches.
    for N in (50, 5000):
        lens, rows, buf, tables, free, n_free, g = _state(9, 2500, 4, 6, 20, 2000)
        _check(ress, lens, [2] * 2500, rows, buf, tables, free, n_free, 4, N)


def test_lengths_and_pages_that_are_not_there(ress):
    """Lengths outside a table, stacks that are too high or low, entries and free pages outside the cache."""
    lens, rows, buf, tables, free, n_free, g = _state(3, 6, 4, 12, 30, 50)
    lens[0], lens[1] = -9, 10 ** 9
    tables[2, :] = -1
    rows[2] = [-1] * 12
    tables[3, 0] = 10 ** 6
    rows[3][0] = 10 ** 6
    free[n_free - 2] = -3
    _check(ress, lens, [3, 2, 5, 1, 9, 0], rows, buf, tables, free, n_free, 4, 30)
    for height in (-4, 0, len(free), len(free) + 9, 2 ** 31 - 1):
        lens, rows, buf, tables, free, n_free, g = _state(4, 3, 4, 12, 30, 40)
        free = [f if f >= 0 else 1 for f in free]
        _check(ress, lens, [2, 5, 1], rows, buf, tables, free, height, 4, 8)


def test_nothing_to_do(ress):
    e = torch.empty(0, dtype=I32, device="cuda")
    r = ress.ress_page_tables(e, e, torch.empty(0, 5, dtype=I32, device="cuda"), _t([1, 2]), _t([2]), page=4, tokens=3)
    assert r["cu_q"].tolist() == [0] and r["slots"].tolist() == [-1] * 3 and r["n_free"].tolist() == [2] and r["pos"].tolist() == [0] * 3
    r = ress.ress_page_tables(_t([3, 0]), _t([1, 1]), torch.empty(2, 0, dtype=I32, device="cuda"), e, _t([0]), page=4, tokens=5000)
    assert r["lens"].tolist() == [0, 0] and r["n_refused"].tolist() == [2] and (r["slots"] == -1).all()
    r = ress.ress_page_tables(_t([3]), _t([1]), torch.zeros(1, 2, dtype=I32, device="cuda"), _t([0]), _t([1]), page=4, tokens=0)
    assert r["lens"].tolist() == [3] and r["n_refused"].tolist() == [1]
    n = ress.ress_pages_release(e, e, torch.empty(0, 5, dtype=I32, device="cuda"), _t([1, 2]), _t([9]))
    assert n.tolist() == [2]


@pytest.mark.parametrize("N", [64, 6000])
def test_in_place_steps_of_a_captured_call(ress, N):
    """Lengths and the stack's height updated in place, step after step, by a captured call beside eager work."""
    page, B, max_pages = 4, 20, 2000
    lens, rows, buf, tables, free, n_free, g = _state(5, B, page, max_pages, 40, 5000)
    d_lens, d_free, d_n = _t(lens), _t(free), _t([n_free])
    new = torch.zeros(B, dtype=I32, device="cuda")
    cu, slots, pos, ref = (torch.empty(n, dtype=I32, device="cuda") for n in (B + 1, N, N, 1))
    call = lambda: ress.ress_page_tables(d_lens, new, tables, d_free, d_n, page=page, lens_out=d_lens, n_free_out=d_n, cu_q=cu,
                                         slots=slots, pos=pos, n_refused=ref)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(5):
        n = torch.randint(0, N // B + 1, (B,), generator=g).tolist()
        new.copy_(_t(n))
        graph.replay()
        torch.cuda.synchronize()
        w = PR.tables(lens, n, rows, free, n_free, page, N)
        lens, n_free = w["lens"], w["n_free"][0]
        assert d_lens.tolist() == lens and d_n.tolist() == [n_free] and cu.tolist() == w["cu_q"] and slots.tolist() == w["slots"]
        assert pos.tolist() == w["pos"] and tables.tolist() == rows


@pytest.mark.parametrize("B,max_pages,clear", [(1, 1, True), (1, 5000, False), (3, 300, True), (64, 257, False), (1024, 9, True),
                                               (1025, 9, True), (3000, 5, False)])
def test_release(ress, B, max_pages, clear):
    say(f"[release] B {B} x {max_pages}")
    for seed in (0, 1):
        lens, rows, buf, tables, free, n_free, g = _state(seed + B, B, 1, max_pages, max_pages, 7, max_pages + 5 * seed)
        first = torch.randint(-2, max_pages + 1, (B,), generator=g).tolist()
        last = torch.randint(-2, max_pages + 3, (B,), generator=g).tolist()
        if seed == 0:
            first, last = [0] * B, [2 ** 31 - 1] * B
        if max_pages > 2:  # (entries that are no page of the cache)
            rows[0][1] = -1
            rows[-1][2] = 10 ** 8
            tables.copy_(_t(rows))
        d_free, stack = _t(free), list(free)
        n = ress.ress_pages_release(_t(first), _t(last), tables, d_free, _t([n_free]), clear=clear)
        height = PR.release(first, last, rows, stack, n_free, clear)
        assert n.tolist() == [height] and d_free.tolist() == stack and tables.tolist() == rows
        assert (buf[:, max_pages:] == -77).all()
        if clear:  # a second release finds nothing
            again = ress.ress_pages_release(_t(first), _t(last), tables, d_free, n, n_free_out=n)
            assert again.tolist() == [height] and d_free.tolist() == stack


def test_release_onto_a_full_stack(ress):
    """Entries that some sequence gives back twice: the stack never passes its end."""
    tables = _t([[0, 1, 2], [2, 1, 0], [0, 0, 0]])
    free, n = _t([5, 5, 5, 5, 5]), _t([1])
    out = ress.ress_pages_release(_t([0, 0, 0]), _t([3, 3, 3]), tables, free, n, clear=False)
    assert out.tolist() == [5] and free.tolist() == [5, 0, 1, 2, 2]
    for height in (5, 9, -3):
        free = _t([5, 5, 5, 5, 5])
        out = ress.ress_pages_release(_t([0, 0, 0]), _t([3, 0, 0]), tables, free, _t([height]), clear=False)
        assert out.tolist() == [5 if height > 0 else 3] and free.tolist() == ([5] * 5 if height > 0 else [0, 1, 2, 5, 5])


def test_what_is_released_is_taken_again(ress):
    """Steps and releases in turn: no page is ever in two tables, or in a table and on the stack."""
    page, B, max_pages, n_pages = 4, 12, 30, 150
    g = torch.Generator().manual_seed(8)
    tables, lens = torch.full((B, max_pages), -1, dtype=I32, device="cuda"), torch.zeros(B, dtype=I32, device="cuda")
    free, n = torch.arange(n_pages, dtype=I32, device="cuda"), _t([n_pages])
    for _ in range(30):
        new = _t(torch.randint(0, 20, (B,), generator=g).tolist())
        ress.ress_page_tables(lens, new, tables, free, n, page=page, tokens=160, lens_out=lens, n_free_out=n)
        held = tables[tables >= 0].tolist()
        stack = free[:n.item()].tolist()
        assert sorted(held + stack) == list(range(n_pages))
        ends = torch.rand(B, generator=g) < 0.2
        ress.ress_pages_release(torch.zeros_like(lens), _t([max_pages if e else 0 for e in ends]), tables, free, n, n_free_out=n)
        lens.masked_fill_(ends.cuda(), 0)
