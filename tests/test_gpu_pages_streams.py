"""The calls of include/ress_pages.h on other streams, their inputs made beforehand, so that nothing in a call waits: beside work that
is still queued on torch's current stream when the call has returned, and two at once."""
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


@pytest.fixture(scope="module")
def calls(ress):
    """Calls that make outputs and workspaces of their own, over inputs that nothing changes but the tables' rows, which every
    call writes alike."""
    g = torch.Generator(device="cuda").manual_seed(1)
    t = lambda *x: torch.tensor(x, dtype=I32, device="cuda")
    q, k, v = (torch.randn(h, 6000, 64, generator=g, device="cuda").to(BF) for h in (8, 2, 2))
    pos = torch.arange(6000, device="cuda", dtype=I32)[:, None]
    kp, vp = (torch.zeros(400, 2, 16, 64, dtype=BF, device="cuda") for _ in range(2))
    tab = torch.randperm(400, generator=g, device="cuda").int()[None]
    slots = (tab[0, (pos[:, 0] // 16).long()] * 16 + pos[:, 0] % 16).int()
    ress.ress_qk_norm_rope_pages(q, k, v, pos, slots, kp, vp, dims=(64,))
    kp2, vp2 = torch.zeros_like(kp), torch.zeros_like(vp)
    lens, new, stack, height, fresh = t(100), t(5000), tab[0].clone(), t(400), tab.clone()
    first, last, empty, given = t(0), t(30), t(0), torch.full((400,), -1, dtype=I32, device="cuda")
    all_q, one_q, many, whole = t(0, 6000), t(0, 1), torch.arange(601, device="cuda", dtype=I32), t(6000)
    token, each = q[:, :1].contiguous(), torch.full((600,), 50, dtype=I32, device="cuda")
    tables = tab.expand(600, 400).contiguous()
    torch.cuda.synchronize()
    return {
        "heads": lambda **s: ress.ress_qk_norm_rope(q, k, pos, dims=(64,), **s),
        "heads_pages": lambda **s: ress.ress_qk_norm_rope_pages(q, k, v, pos, slots, kp2, vp2, dims=(64,), **s),
        "heads_bwd": lambda **s: ress.ress_qk_norm_rope_bwd(q, k, q, k, pos, dims=(64,), **s),
        "tables": lambda **s: dict(ress.ress_page_tables(lens, new, fresh, stack, height, page=16, tokens=6000, **s), tables=fresh),
        "release": lambda **s: dict(n=ress.ress_pages_release(first, last, tab, given, empty, clear=False, **s), stack=given),
        "chunk": lambda **s: ress.ress_paged_attn(q, kp, vp, all_q, whole, tab, window=6000, want_lse=True, **s),
        "token": lambda **s: ress.ress_paged_attn(token, kp, vp, one_q, whole, tab, window=6000, want_lse=True, **s),
        "many": lambda **s: ress.ress_paged_attn(q[:, :600], kp, vp, many, each, tables, window=6000, want_lse=True, **s),
    }


NAMES = ["heads", "heads_pages", "heads_bwd", "tables", "release", "chunk", "token", "many"]


@pytest.mark.parametrize("name", NAMES)
def test_beside_work_that_is_pending(calls, name):
    """Blocks of any size that queued work still writes, over and over, are free again for the current stream: on another one no
    call may take them, for its outputs or for its workspace."""
    call, side = calls[name], torch.cuda.Stream()
    want = {n: t.clone() for n, t in call().items()}
    call(stream=side)  # (that stream has memory from here on: no call waits for an allocation)
    done = torch.cuda.Event()
    for turn in range(3):
        scratch = [torch.zeros(1 << n, dtype=torch.uint8, device="cuda") for n in range(9, 29, 2) for _ in range(4)]
        scratch += [torch.zeros(1 << 28, dtype=torch.uint8, device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        for _ in range(40):  # (some 30 ms, queued in a third of that)
            for x in scratch:
                x.add_(1)
        del scratch, x
        done.record()
        got = call(stream=side)
        assert not done.query(), "the queued work ended before the call was made"
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[n]) for n in want), (name, turn)
        say(f"[streams] {name} {turn}")


def test_two_at_once(calls):
    """The same calls on two streams, over inputs that outlive them, each with memory of its own."""
    for name in NAMES:
        call = calls[name]
        want = {n: t.clone() for n, t in call().items()}
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(2)]
        got = [call(stream=s) for _ in range(3) for s in streams]
        torch.cuda.synchronize()
        assert all(torch.equal(r[n], want[n]) for r in got for n in want), name
