"""Calls on a stream of the caller's: where their memory comes from, and results beside work pending on the current one."""
import pytest
import torch

from gpu_helpers import say

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ress():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_35593_amd as r

    return r


def _mk(*shape, dtype=BF, seed=0):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


def _cases(ress):
    """Calls that make outputs of 8 MB and more, and workspaces; inputs are ready before."""
    x, w = _mk(4096, 1024, dtype=F32), torch.ones(1024, device="cuda")
    st = ress.ress_layer_norm(x, w, want_stats=True)
    q, k, v, do = _mk(8, 9000, 64, seed=1), _mk(8, 9000, 64, seed=2), _mk(8, 9000, 64, seed=3), _mk(8, 9000, 64, seed=4)
    pos = torch.arange(9000, device="cuda", dtype=torch.int32)[:, None]
    kw = dict(window=9000, n_sink=3)
    f = ress.ress_window_attn(q, k, v, want_lse=True, **kw)
    lens, q1 = torch.full((8,), 9000, device="cuda", dtype=torch.int32), q[:, :8].contiguous()
    return {
        "norm": lambda **s: ress.ress_layer_norm(x, w, want_stats=True, out_dtype=F32, **s),
        "norm_bwd": lambda **s: ress.ress_layer_norm_bwd(st["y"], x, w, st["mean"], st["rstd"], **s),
        "rope": lambda **s: ress.ress_rope(q, k, pos, dims=(64,), **s),
        "window": lambda **s: ress.ress_window_attn(q, k, v, want_lse=True, **kw, **s),
        "window_bwd": lambda **s: ress.ress_window_attn_bwd(do, q, k, v, f["o"], f["lse"], **kw, **s),
        "decode": lambda **s: {"o": ress.ress_window_attn_decode(q1, k[:, None], v[:, None], lens, **kw, **s)},
    }


def _base_cases(ress):
    """The same of the attention path's functions (include/ress.h)."""
    H, N, kw = 16, 8192, dict(bq=128, bk=128)
    q, k, v = (_mk(H, N, 64, seed=s) for s in (5, 6, 7))
    gram = torch.eye(64, device="cuda").expand(H, 64, 64).contiguous()
    x, wq, wo = _mk(N, H * 64, seed=8), _mk(3 * H * 64, H * 64, seed=9), _mk(H * 64, H * 64, seed=10)
    xf, a, b = x.float(), q.float(), k.float()
    sel = ress.ress_select(q, k, v, gram, [20] * H, **kw)
    kept = sel["kept_count"], sel["kept_idx"]
    return {
        "select": lambda **s: ress.ress_select(q, k, v, gram, [20] * H, want_debug=True, **kw, **s),
        "sparse": lambda **s: {"o": ress.ress_sparse_attn(q, k, v, *kept, **kw, **s)},
        "sparse_f32": lambda **s: {"o": ress.ress_sparse_attn_out_f32(q, k, v, *kept, **kw, **s)},
        "dense": lambda **s: {"o": ress.ress_dense_attn(q, k, v, **kw, **s)},
        "qkv": lambda **s: {n: t for n, t in ress.ress_qkv_proj_pool(x, wq, gram, **kw, **s).items() if n != "workspace"},
        "out": lambda **s: {"r": ress.ress_out_proj_residual(q, wo, x, **s)},
        "out_f32": lambda **s: {"r": ress.ress_out_proj_residual_f32(q, wo, xf, **s)},
        "drift": lambda **s: {"d": ress.ress_block_drift_sq(a, b, gram, bq=128, **s)},
    }


@pytest.mark.parametrize("path", [_cases, _base_cases], ids=["layer", "attention"])
def test_results_beside_pending_work(ress, path):
    """Blocks just returned by the current stream, whose queue still writes them, are not given to a call on another stream:
    their addresses are others, and results are those of a call alone. (The queue is kept busy by products of known length.)"""
    cases = path(ress)
    alone = {n: {k: t.clone() for k, t in f().items() if t is not None} for n, f in cases.items()}
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    m = torch.randn(4096, 4096, device="cuda")
    for n, f in cases.items():
        torch.cuda.synchronize()
        blocks = {}
        for size in (1 << 14, 1 << 16, 9 << 20, 10 << 20, 17 << 20, 34 << 20, 80 << 20):
            blocks[size] = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(3)]
        for _ in range(3):
            m @ m
        for ts in blocks.values():
            for t in ts:
                t.fill_(255)
        taken = [(t.data_ptr(), t.data_ptr() + t.numel()) for ts in blocks.values() for t in ts]
        del blocks, ts, t  # back in the current stream's pool, their fills still queued
        got = f(stream=side)
        for k, t in got.items():
            if t is not None:
                assert not any(a <= t.data_ptr() < b for a, b in taken), (n, k)
        torch.cuda.synchronize()
        for k, t in alone[n].items():
            assert torch.equal(got[k], t), (n, k)
        say(f"[streams] {n}")


def test_captured_on_a_forked_stream(ress):
    """Calls on a second stream inside a capture, outputs and workspaces made inside: replays, with eager calls of the same
    between them, give the eager bits."""
    cases = _cases(ress)
    main, side = torch.cuda.Stream(), torch.cuda.Stream()

    def step(**s):
        return [(n, k, t) for n, f in cases.items() for k, t in f(**s).items() if t is not None]

    for s in (main, side):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=main):
        side.wait_stream(main)
        out = step(stream=side)
        main.wait_stream(side)
    for rep in range(3):
        for _, _, t in out:
            t.fill_(7)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for (n, k, t), (_, _, e) in zip(out, step()):
            assert torch.equal(t, e), (n, k, rep)
