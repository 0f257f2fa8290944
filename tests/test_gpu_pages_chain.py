"""The steps of ress_pages.h together, as a program that serves streams of frames uses them: tables, norm and rotation into pages,
attention, projection; against the same streams by the contiguous steps, and beside work on other streams."""
import pytest
import torch

from gpu_helpers import say

pytestmark = pytest.mark.gpu

BF, I32 = torch.bfloat16, torch.int32


@pytest.fixture(scope="module")
def ress():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_35593_amd as r

    return r


def _steps(B, turns, most, g):
    """New tokens of every sequence, turn by turn: prompts, single tokens, pauses."""
    return [[0 if int(torch.randint(0, 4, (1,), generator=g)) == 0 else int(torch.randint(1, most if t % 3 == 0 else 2, (1,), generator=g))
             for _ in range(B)] for t in range(turns)]


@pytest.mark.parametrize("H,H_kv,page,frame,window,n_sink", [(8, 2, 16, 1, 10 ** 9, 0), (4, 4, 24, 10, 3, 10), (6, 2, 64, 1, 40, 5)])
def test_streams_over_pages_are_the_contiguous_steps(ress, H, H_kv, page, frame, window, n_sink):
    """Every step's outputs against windowed attention over the sequence's whole normed and turned keys. Both round alike but for the
    weights' bf16 rounding and the order of sums: 2^-7 of the values' size."""
    g = torch.Generator().manual_seed(page)
    B, n_pages, max_pages, N = 4, 400, 100, 360
    gd = torch.Generator(device="cuda").manual_seed(page)
    rn = lambda *s: torch.randn(*s, generator=gd, device="cuda")
    w = dict(q_gamma=1 + 0.2 * rn(64), q_beta=0.1 * rn(64), k_gamma=1 + 0.2 * rn(64), k_beta=0.1 * rn(64))
    kw = dict(dims=(64,), base=1e4, **w)
    i32 = dict(dtype=I32, device="cuda")
    tables, lens = torch.full((B, max_pages), -1, **i32), torch.zeros(B, **i32)
    free, n_free = torch.randperm(n_pages, generator=gd, device="cuda").int(), torch.tensor([n_pages], **i32)
    kp, vp = (torch.full((n_pages, H_kv, page, 64), float("nan"), dtype=BF, device="cuda") for _ in range(2))
    seen = [([], []) for _ in range(B)]
    for turn, new in enumerate(_steps(B, 9, 90, g)):
        q, k, v = rn(H, N, 64).to(BF), rn(H_kv, N, 64).to(BF), rn(H_kv, N, 64).to(BF)
        before = lens.tolist()
        t = ress.ress_page_tables(lens, torch.tensor(new, **i32), tables, free, n_free, page=page, tokens=N, lens_out=lens,
                                  n_free_out=n_free)
        assert t["n_refused"].item() == 0
        r = ress.ress_qk_norm_rope_pages(q, k, v, t["pos"][:, None], t["slots"], kp, vp, **kw)
        o = ress.ress_paged_attn(r["q"], kp, vp, t["cu_q"], lens, tables, frame=frame, window=window, n_sink=n_sink, want_lse=True)
        cu = t["cu_q"].tolist()
        for b in range(B):
            if new[b] == 0:
                continue
            rows = slice(cu[b], cu[b + 1])
            pos = torch.arange(before[b], before[b] + new[b], device="cuda", dtype=I32)[:, None]
            c = ress.ress_qk_norm_rope(q[:, rows], k[:, rows], pos, **kw)
            assert torch.equal(c["q"], r["q"][:, rows])
            seen[b][0].append(c["k"])
            seen[b][1].append(v[:, rows])
            kk, vv = (torch.cat(x, 1) for x in seen[b])
            ref = ress.ress_window_attn(c["q"], kk, vv, window=window, frame=frame, n_sink=n_sink, q_offset=before[b], want_lse=True)
            err = (ref["o"].float() - o["o"][:, rows].float()).abs()
            size = vv.float().abs().amax()
            assert err.max() <= 2.0 ** -7 * size and err.mean() <= 2.0 ** -9 * size, (turn, b)
            assert (ref["lse"] - o["lse"][:, rows]).abs().max() <= 1e-4
        if turn == 4:  # a sequence ends, another takes its place
            ress.ress_pages_release(torch.zeros_like(lens), torch.tensor([0, max_pages, 0, 0], **i32), tables, free, n_free,
                                    n_free_out=n_free)
            lens[1] = 0
            seen[1] = ([], [])
    say(f"[chain] pages left {n_free.item()}, lengths {lens.tolist()}")


def _calls(ress):
    """Calls that make outputs and workspaces; inputs are ready before."""
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn(h, 6000, 64, generator=g, device="cuda").to(BF) for h in (8, 2, 2))
    pos = torch.arange(6000, device="cuda", dtype=I32)[:, None]
    kp, vp = (torch.zeros(400, 2, 16, 64, dtype=BF, device="cuda") for _ in range(2))
    tab = torch.randperm(400, generator=g, device="cuda").int()[None]
    t = lambda *x: torch.tensor(x, dtype=I32, device="cuda")
    ress.ress_qk_norm_rope_pages(q, k, v, pos, (tab[0, (pos[:, 0] // 16).long()] * 16 + pos[:, 0] % 16).int(), kp, vp, dims=(64,))
    fresh, lens, new, stack, height = tab.clone(), t(100), t(5000), tab[0].clone(), t(400)
    return {
        "heads": lambda **s: ress.ress_qk_norm_rope(q, k, pos, dims=(64,), **s),
        "heads_bwd": lambda **s: ress.ress_qk_norm_rope_bwd(q, k, q, k, pos, dims=(64,), **s),
        "tables": lambda **s: ress.ress_page_tables(lens, new, fresh, stack, height, page=16, tokens=6000, **s),
        "release": lambda **s: {"n": ress.ress_pages_release(t(0), t(0), fresh, stack, height, **s)},
        "chunk": lambda **s: ress.ress_paged_attn(q, kp, vp, t(0, 6000), t(6000), tab, window=6000, want_lse=True, **s),
        "token": lambda **s: ress.ress_paged_attn(q[:, :1], kp, vp, t(0, 1), t(6000), tab, window=6000, want_lse=True, **s),
    }


@pytest.mark.parametrize("name", ["heads", "heads_bwd", "tables", "release", "chunk", "token"])
def test_calls_on_another_stream_beside_pending_work(ress, name):
    """The caller's stream, torch's current one full of work whose memory is freed meanwhile."""
    call = _calls(ress)[name]
    want = {n: t.clone() for n, t in call().items()}
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        scratch = [torch.randn(1 << 22, device="cuda") for _ in range(4)]
        for x in scratch:
            for _ in range(10):
                x.mul_(1.0001)
        del scratch, x
        got = call(stream=side)
        side.synchronize()
        assert all(torch.equal(got[n], want[n]) for n in want), name
    torch.cuda.synchronize()


def test_two_calls_at_once(ress):
    """The same calls on two streams, each with memory of its own."""
    for name, call in _calls(ress).items():
        if name == "tables":
            continue  # (writes its tables)
        want = {n: t.clone() for n, t in call().items()}
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(2)]
        got = [call(stream=s) for _ in range(3) for s in streams]
        torch.cuda.synchronize()
        assert all(torch.equal(r[n], want[n]) for r in got for n in want), name
