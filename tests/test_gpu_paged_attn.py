"""Attention of new tokens over pages against float64: ragged batches, pages of any size, windows, sinks, frames, shared heads, strides,
pages that are not there, far offsets, captured calls."""
import math

import pytest
import torch

import pages_refs as PR
from gpu_helpers import say
from layer_refs import within

pytestmark = pytest.mark.gpu

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


@pytest.fixture(scope="module")
def ress():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_35593_amd as r

    return r


def _t(x):
    return torch.tensor(x, dtype=I32, device="cuda")


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _state(seed, H, H_kv, page, lens, new, padding=0, amp=1.0, spare=2):
    """q, pages, tables and lengths; pages in no order, NaN wherever no token is."""
    g = _gen(seed)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    counts = [-(-max(n, 0) // page) for n in lens]
    n_pages, most = sum(counts) + spare, max(counts + [0]) + 1
    order = torch.randperm(n_pages, generator=g, device="cuda").int()
    tables, at = torch.full((len(lens), most), -1, dtype=I32, device="cuda"), 0
    k, v = ((rn(n_pages, H_kv, page, 64) * a + m * rn(H_kv, 1, 64)).to(BF) for a, m in ((1.0, 0.7), (0.7, 0.3)))
    live = torch.zeros(n_pages, page, dtype=torch.bool, device="cuda")
    for b, n in enumerate(counts):
        tables[b, :n] = order[at:at + n]
        if n:
            live[order[at:at + n].long()] = (torch.arange(n * page, device="cuda") < lens[b]).view(n, page)
        at += n
    for x in (k, v):
        x.masked_fill_(~live[:, None, :, None], float("nan"))
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    q = (rn(H, cu[-1] + padding, 64) * amp).to(BF)
    return q, k, v, cu, tables


def _check(ress, q, k, v, cu, lens, tables, frame=1, window=10 ** 9, n_sink=0, scale=None, **kw):
    ref, lse, bo, bl, rows = PR.paged(q, k, v, cu, lens, tables, frame, window, n_sink, scale)
    args = (q, k, v, _t(cu), _t(lens), tables)
    opt = dict(frame=frame, window=window, n_sink=n_sink, scale=scale, **kw)
    out, lse_out = torch.full(q.shape, 7.0, dtype=BF, device="cuda"), torch.full(q.shape[:2], 7.0, device="cuda")
    r = ress.ress_paged_attn(*args, out=out, lse=lse_out, **opt)
    within(r["o"][:, rows], ref[:, rows], bo[:, rows], "o")
    within(r["lse"][:, rows], lse[:, rows], bl[:, rows], "lse")
    blind = torch.isinf(lse) & rows
    assert not r["o"][blind].any()  # zeros, exactly
    assert (out[:, ~rows] == 7.0).all() and (lse_out[:, ~rows] == 7.0).all()  # left as they were
    plain = ress.ress_paged_attn(*args, **opt)
    assert plain["lse"] is None
    within(plain["o"][:, rows], ref[:, rows], bo[:, rows], "o without lse")
    assert torch.equal(ress.ress_paged_attn(*args, **opt)["o"][:, rows], plain["o"][:, rows])
    return r


HEADS = [(1, 1), (4, 4), (8, 2), (6, 2), (8, 1), (40, 1)]
BATCHES = [  # lengths, new tokens
    ([1], [1]), ([700], [1]), ([5, 0, 64, 65, 130], [1, 0, 1, 1, 2]), ([300], [300]), ([40, 333, 7, 200], [40, 33, 7, 1]),
    ([1000, 3, 500], [130, 3, 257]), ([129, 128, 127], [129, 128, 127]), ([20, 20], [33, 20])]


@pytest.mark.parametrize("H,H_kv", HEADS)
@pytest.mark.parametrize("page", [1, 7, 16, 64, 128])
def test_batches(ress, H, H_kv, page):
    for i, (lens, new) in enumerate(BATCHES):
        say(f"[paged] H {H}/{H_kv} page {page} lens {lens} new {new}")
        q, k, v, cu, tables = _state(i + page, H, H_kv, page, lens, new, padding=i % 3)
        _check(ress, q, k, v, cu, lens, tables)


@pytest.mark.parametrize("page", [5, 16, 256])
@pytest.mark.parametrize("frame,window,n_sink", [(1, 1, 0), (1, 20, 3), (1, 100, 70), (10, 4, 17), (100, 2, 100), (37, 1, 65),
                                                 (1374, 4, 1374), (2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1), (1, 64, 64), (64, 1, 0)])
def test_windows(ress, page, frame, window, n_sink):
    say(f"[paged] page {page} frame {frame} window {window} sinks {n_sink}")
    for H, H_kv, lens, new in ((4, 2, [700, 64, 1, 333], [1, 1, 1, 1]), (4, 1, [900, 130, 400], [200, 130, 77]),
                               (2, 2, [1500, 800], [500, 3])):
        q, k, v, cu, tables = _state(page + frame % 97, H, H_kv, page, lens, new)
        _check(ress, q, k, v, cu, lens, tables, frame, window, n_sink)


@pytest.mark.parametrize("H,H_kv,lens,new,window", [
    (4, 4, [30000], [1], 10 ** 9), (16, 4, [9000, 20, 4000], [1, 1, 1], 10 ** 9), (16, 2, [12000], [5], 3000),
    (8, 8, [5000, 3000], [700, 20], 10 ** 9), (16, 16, [6000], [300], 10 ** 9), (2, 1, [9000, 1, 8000], [40, 1, 900], 5000)])
def test_long_caches(ress, H, H_kv, lens, new, window):
    """Keys split over workgroups, some sequences' over more than others'."""
    say(f"[paged] H {H}/{H_kv} lens {lens} new {new} window {window}")
    for page in (16, 24):
        q, k, v, cu, tables = _state(page, H, H_kv, page, lens, new, padding=3)
        _check(ress, q, k, v, cu, lens, tables, 1, window, 9)


@pytest.mark.parametrize("new", [[1, 4], [150, 90]])
@pytest.mark.parametrize("page", [8, 13, 64])
def test_pages_that_are_not_there(ress, page, new):
    """Entries outside the cache hide their keys: some, those of whole tiles, all."""
    lens = [700, 300]
    for seed, share in enumerate((0.1, 0.5, 0.95, 1.0)):
        q, k, v, cu, tables = _state(seed, 4, 2, page, lens, new)
        gone = torch.rand(tables.shape, generator=_gen(seed), device="cuda") < share
        bad = torch.randint(0, 2, tables.shape, generator=_gen(seed + 9), device="cuda") * (2 ** 31 - 1 - k.shape[0]) + k.shape[0]
        bad = torch.where(torch.rand(tables.shape, generator=_gen(seed + 5), device="cuda") < 0.5, bad, -bad).int()
        tables = torch.where(gone, bad, tables)
        _check(ress, q, k, v, cu, lens, tables, 1, 500, 20)
    q, k, v, cu, tables = _state(9, 4, 2, page, lens, new)
    none = torch.empty(0, 2, page, 64, dtype=BF, device="cuda")
    r = ress.ress_paged_attn(q, none, none, _t(cu), _t(lens), tables, window=10, want_lse=True)
    assert not r["o"].any() and (r["lse"] == -math.inf).all()
    r = ress.ress_paged_attn(q, k, v, _t(cu), _t(lens), tables[:, :0], window=10, want_lse=True)
    assert not r["o"].any() and (r["lse"] == -math.inf).all()


def test_lengths_outside_a_table(ress):
    """Negative and too long ones are clamped; new tokens before position 0 see nothing."""
    lens, new = [200, 0, 77], [5, 3, 90]
    q, k, v, cu, tables = _state(1, 4, 2, 16, lens, new)
    tables = tables[:, :13].contiguous()
    for got in ([10 ** 9, -5, 77], [2 ** 31 - 1, -2 ** 31, 60]):
        k2, v2 = k.nan_to_num(0.5), v.nan_to_num(0.5)  # (tokens up to the table's end are seen)
        _check(ress, q, k2, v2, cu, got, tables, 1, 10 ** 9, 2)


def test_offsets_that_descend_or_pass_the_rows(ress):
    """Nothing behind the rows is written, whatever the offsets are."""
    lens, new = [200, 50, 77], [5, 3, 9]
    q, k, v, cu, tables = _state(2, 4, 2, 16, lens, new)
    k, v = k.nan_to_num(0.5), v.nan_to_num(0.5)
    buf = torch.full((4, 40, 64), 7.0, dtype=BF, device="cuda")
    for bad in ([0, 10 ** 9, 10 ** 9, 10 ** 9], [-5, 3, 1, 99], [9, 5, 2, 0], [2 ** 31 - 1, -2 ** 31, 5, 6]):
        ress.ress_paged_attn(q, k, v, _t(bad), _t(lens), tables, window=30, out=buf[:, 3:20])
        torch.cuda.synchronize()
        assert (buf[:, :3] == 7.0).all() and (buf[:, 20:] == 7.0).all()


@pytest.mark.parametrize("N", [12, 700])
def test_offsets_in_no_order_where_keys_are_cut(ress, N):
    """The same with keys that are cut over workgroups, whose parts stay in their workspace."""
    B, g = 5, torch.Generator().manual_seed(N)
    q, k, v, cu, tables = _state(4, 4, 2, 16, [9000, 7000, 3, 4000, 6000], [N // 5] * B, padding=N - N // 5 * 5)
    k, v = k.nan_to_num(0.5), v.nan_to_num(0.5)
    n = ress.ress_paged_attn_workspace_size(B, 4, 2, N, page=16, max_pages=tables.shape[1], n_pages=k.shape[0], window=8000)
    assert n > 0
    ws, buf = torch.full((n + 4096,), 77, dtype=torch.uint8, device="cuda"), torch.full((4, N + 20, 64), 7.0, dtype=BF, device="cuda")
    bad = [[0] + [10 ** 9] * B, [N, N // 2, 0, N, 0, N], [0, N, 0, N, 0, N], list(range(N, N - 6, -1))]
    bad += [torch.randint(-20, N + 20, (B + 1,), generator=g).tolist() for _ in range(20)]
    for cu in bad:
        ress.ress_paged_attn(q, k, v, _t(cu), _t([9000, 7000, 3, 4000, 6000]), tables, window=8000, out=buf[:, 10:N + 10], workspace=ws[:n])
        torch.cuda.synchronize()
        assert (buf[:, :10] == 7.0).all() and (buf[:, N + 10:] == 7.0).all() and (ws[n:] == 77).all()


def test_thousands_of_offsets_in_no_order(ress):
    """The same with a list of where blocks begin."""
    g = torch.Generator().manual_seed(3)
    q, k, v, cu, tables = _state(2, 2, 1, 16, [40] * 700, [1] * 700)
    k, v = k.nan_to_num(0.5), v.nan_to_num(0.5)
    buf = torch.full((2, 720, 64), 7.0, dtype=BF, device="cuda")
    for lo, hi in ((0, 700), (-10, 900), (-2 ** 31, 2 ** 31 - 1)):
        bad = torch.randint(lo, hi, (701,), generator=g).tolist()
        ress.ress_paged_attn(q, k, v, _t(bad), _t([40] * 700), tables, window=30, out=buf[:, 3:703])
        torch.cuda.synchronize()
        assert (buf[:, :3] == 7.0).all() and (buf[:, 703:] == 7.0).all()


def test_offsets_that_begin_behind_the_first_row(ress):
    lens, new = [9000, 70], [1, 2]
    q, k, v, cu, tables = _state(3, 8, 2, 16, lens, new, padding=6)
    _check(ress, q, k, v, [c + 2 for c in cu], lens, tables)


@pytest.mark.parametrize("amp", [10.0, 60.0])
def test_large_logits(ress, amp):
    lens, new = [700, 300, 2000], [1, 200, 3]
    q, k, v, cu, tables = _state(4, 4, 2, 16, lens, new, amp=amp)
    _check(ress, q, k, v, cu, lens, tables, 1, 1500, 4)
    q, k, v, cu, tables = _state(5, 2, 2, 16, [640, 640], [128, 1])
    _check(ress, q, k * (1 + torch.arange(k.shape[0], device="cuda") * 3.0)[:, None, None, None].to(BF), v, cu, [640, 640], tables)


def test_far_logits(ress):
    """Products that float32 holds exactly, up to 2^119: a row's weights are those of its largest ones."""
    for new in (1, 100):
        lens = [500]
        q, k, v, cu, tables = _state(6, 2, 1, 16, lens, [new])
        q.fill_(0.0)
        q[..., 0] = 2.0 ** 60
        k.nan_to_num_(0.0)
        k[..., 0] = torch.randint(-3, 4, k.shape[:3], generator=_gen(3), device="cuda").to(BF) * 2.0 ** 56
        r = ress.ress_paged_attn(q, k, v, _t(cu), _t(lens), tables, window=10 ** 9, scale=1.0, want_lse=True)
        flat = tables[0, :-1].long()
        kk, vv = k[flat, 0].reshape(-1, 64)[:500], v[flat, 0].reshape(-1, 64)[:500].double()
        for t in range(new):
            n = 500 - new + t + 1
            top = kk[:n, 0] == kk[:n, 0].max()
            want = vv[:n][top].mean(0)
            # weights rounded to bf16 (2^-8 of each), the output (2^-8), sums in float32
            lim = 2.0 ** -8 * (vv[:n][top].abs().mean(0) + 2 * want.abs()) + 2.0 ** -12
            assert ((r["o"][:, t].double() - want).abs() <= lim).all(), (new, t)


@pytest.mark.parametrize("new", [[1, 3], [200, 77]])
def test_strides(ress, new):
    """Token-major queries and outputs, pages with tokens first, heads first, K and V interleaved, tables inside a larger one:
    the contiguous call's results."""
    lens = [800, 300]
    q, k, v, cu, tables = _state(7, 4, 2, 16, lens, new)
    args = _t(cu), _t(lens)
    want = ress.ress_paged_attn(q, k, v, *args, tables, window=600, n_sink=5, want_lse=True)
    token_major = lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)
    both = torch.stack([k, v], 3)  # [n_pages][H_kv][page][2][64]
    wide = torch.full((2, tables.shape[1] + 9), -1, dtype=I32, device="cuda")
    wide[:, 4:4 + tables.shape[1]] = tables
    forms = {"tokens first": (k.transpose(1, 2).contiguous().transpose(1, 2), v.transpose(1, 2).contiguous().transpose(1, 2)),
             "heads first": (k.transpose(0, 1).contiguous().transpose(0, 1), v), "interleaved": (both[..., 0, :], both[..., 1, :])}
    for name, (a, b) in forms.items():
        buf = torch.full((q.shape[1], 9, 64), 7.0, dtype=BF, device="cuda")
        out = buf.transpose(0, 1)[2:6]
        r = ress.ress_paged_attn(token_major(q), a, b, *args, wide[:, 4:4 + tables.shape[1]], window=600, n_sink=5, out=out, want_lse=True)
        assert torch.equal(r["o"], want["o"]) and torch.equal(r["lse"], want["lse"]), name
        assert (buf[:, :2] == 7.0).all() and (buf[:, 6:] == 7.0).all()


def test_pages_beyond_32_bits(ress):
    """Keys and values whose rows lie behind 2^31 elements."""
    page, n_pages = 16, 200
    k = torch.zeros(n_pages, 1, page, 1 << 20, dtype=BF, device="cuda")[..., :64]  # 2^31.6 elements
    v = torch.zeros(n_pages, 1, page, 64, dtype=BF, device="cuda")
    g = _gen(8)
    k.copy_(torch.randn(k.shape, generator=g, device="cuda"))
    v.copy_(torch.randn(v.shape, generator=g, device="cuda"))
    tables = torch.arange(n_pages - 1, n_pages - 31, -1, device="cuda", dtype=I32)[None]
    for new in (1, 200):
        q = torch.randn(2, new, 64, generator=g, device="cuda").to(BF)
        _check(ress, q, k, v, [0, new], [470], tables)


def test_many_sequences(ress):
    """More sequences than a workgroup looks at in one turn, most of them of one new token, some of none or many."""
    g = torch.Generator().manual_seed(9)
    for B in (255, 256, 257, 1200):
        lens = torch.randint(1, 90, (B,), generator=g).tolist()
        new = [0 if i % 7 == 3 else min(n, 40 if i % 100 == 50 else 1) for i, n in enumerate(lens)]
        q, k, v, cu, tables = _state(B, 2, 1, 16, lens, new)
        _check(ress, q, k, v, cu, lens, tables, 1, 50, 3)


@pytest.mark.parametrize("B,H,H_kv,top,new", [(60, 8, 4, 6000, 1), (60, 8, 4, 6000, 30), (130, 2, 1, 5000, 1), (130, 2, 1, 5000, 90),
                                              (256, 2, 2, 700, 1), (257, 2, 2, 700, 1), (40, 16, 16, 900, 1), (12, 8, 8, 8000, 150),
                                              (256, 2, 1, 2000, 100), (257, 2, 1, 2000, 100)])
def test_uneven_lengths(ress, B, H, H_kv, top, new):
    """Keys cut by sequences' lengths, from one to `top` on a log scale: single tokens and chunks, some sequences without any."""
    lens = [round(top ** (i / (B - 1))) for i in range(B)]
    q, k, v, cu, tables = _state(B + new, H, H_kv, 16, lens, [0 if i % 9 == 4 else min(n, new) for i, n in enumerate(lens)])
    _check(ress, q, k, v, cu, lens, tables)
    _check(ress, q, k, v, cu, lens, tables, 5, 60, 30)


@pytest.mark.parametrize("B", [512, 513, 4097])
@pytest.mark.parametrize("many", [0, 130])
def test_thousands_of_sequences(ress, B, many):
    """Around the number from which a list tells where sequences' blocks begin, and beyond; blocks of 32 rows and of 128, empty
    sequences first, last and between, and rows behind the last."""
    g = torch.Generator().manual_seed(B + many)
    lens = torch.randint(many, 60 + many, (B,), generator=g).tolist()
    new = [0 if i % 5 == 0 or i == B - 1 else min(n, many or 1 + i % 3) for i, n in enumerate(lens)]
    q, k, v, cu, tables = _state(B, 1, 1, 32, lens, new, padding=5)
    _check(ress, q, k, v, cu, lens, tables, 1, 40, 2)


def test_captured_call_follows_its_lengths(ress):
    """One graph over steps whose lengths, offsets and tables change, beside eager work; a second one with a workspace of its own."""
    H, H_kv, page, B, N = 8, 2, 16, 3, 60
    q, k, v, cu, tables = _state(10, H, H_kv, page, [3000, 2500, 1000], [20, 20, 20])
    k, v = k.nan_to_num(0.5), v.nan_to_num(0.5)
    d_cu, d_lens, d_tab = _t(cu), _t([3000, 2500, 1000]), tables.clone()
    kw = dict(window=2000, n_sink=7)
    graphs, outs = [], []
    for _ in range(2):
        ws = torch.empty(max(1, ress.ress_paged_attn_workspace_size(B, H, H_kv, N, page=page, max_pages=tables.shape[1],
                                                                    n_pages=k.shape[0], **kw)), dtype=torch.uint8, device="cuda")
        call = lambda: ress.ress_paged_attn(q, k, v, d_cu, d_lens, d_tab, workspace=ws, want_lse=True, **kw)
        call()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append((call(), ws))
    for lens, cu2 in (([3000, 2500, 1000], [0, 20, 40, 60]), ([1, 2500, 999], [0, 1, 2, 60]), ([2999, 5, 640], [0, 50, 55, 60])):
        d_lens.copy_(_t(lens))
        d_cu.copy_(_t(cu2))
        d_tab.copy_(tables.flip(0) if lens[0] == 1 else tables)
        q.copy_(torch.randn(q.shape, generator=_gen(lens[2]), device="cuda"))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        ref, lse, bo, bl, rows = PR.paged(q, k, v, cu2, lens, d_tab, 1, 2000, 7)
        for r, _ in outs:
            within(r["o"], ref, bo, "o")
            within(r["lse"], lse, bl, "lse")
