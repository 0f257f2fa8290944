"""What the binding of include/ress_pages.h does with memory, on the CPU, as tests/test_layer_binding.py does it for ress_layer.h:
its calls are followed up to the C entry point, which is replaced, with host tensors in the place of the device's."""
import pytest
import torch

from test_layer_binding import _Stream, _Torch, _z

F32, I32 = torch.float32, torch.int32


@pytest.fixture
def pages():
    from paper_2609_35593_amd import pages

    return pages


@pytest.fixture
def traced(pages, monkeypatch):
    """(torch's stand-in, list that each call's address arguments are appended to)."""
    from paper_2609_35593_amd import memory

    fake, calls = _Torch(), []

    def call(fn, device, stream, *args):
        calls.append((fn.__name__, [a for a in args if isinstance(a, int)], [(p, r() is not None) for r, p, _ in fake.made]))

    monkeypatch.setattr(memory, "torch", fake)
    monkeypatch.setattr(memory, "raw_stream", lambda index: fake.cuda.current)
    monkeypatch.setattr(pages, "_device", lambda name, t: t.device)
    monkeypatch.setattr(pages, "_call", call)
    return fake, calls


def _i(*shape):
    return torch.zeros(shape, dtype=I32)


# Calls that need a workspace and are given none.
CALLS = {
    "ress_qk_norm_rope_bwd": lambda b, **kw: b.ress_qk_norm_rope_bwd(_z(2, 9, 64), _z(1, 9, 64), _z(2, 9, 64), _z(1, 9, 64), _i(9, 1),
                                                                     dims=(64,), **kw),
    "ress_pages_release": lambda b, **kw: b.ress_pages_release(_i(2), _i(2), _i(2, 5), _i(9), _i(1), **kw),
    "ress_paged_attn": lambda b, **kw: b.ress_paged_attn(_z(4, 1, 64), _z(700, 4, 16, 64), _z(700, 4, 16, 64), _i(2), _i(1), _i(1, 700),
                                                         window=10000, **kw),
}


@pytest.mark.parametrize("name", CALLS)
def test_workspace_lives_until_its_kernels_are_enqueued(pages, traced, name):
    fake, calls = traced
    CALLS[name](pages)
    (called, addresses, made), = calls
    assert called == name
    workspaces = [m for m, (_, _, dtype) in zip(made, fake.made) if dtype == torch.uint8]
    assert len(workspaces) == 1
    (address, alive), = workspaces
    assert address in addresses and alive


CALLS_ALL = dict(
    CALLS,
    ress_qk_norm_rope=lambda b, **kw: b.ress_qk_norm_rope(_z(2, 9, 64), _z(1, 9, 64), _i(9, 2), dims=(32, 32), **kw),
    ress_qk_norm_rope_pages=lambda b, **kw: b.ress_qk_norm_rope_pages(_z(2, 9, 64), _z(1, 9, 64), _z(1, 9, 64), _i(9, 1), _i(9),
                                                                      _z(3, 1, 4, 64), _z(3, 1, 4, 64), dims=(64,), **kw),
    ress_page_tables=lambda b, **kw: b.ress_page_tables(_i(2), _i(2), _i(2, 5), _i(9), _i(1), page=4, tokens=7, **kw),
    lse=lambda b, **kw: b.ress_paged_attn(_z(4, 1, 64), _z(3, 4, 16, 64), _z(3, 4, 16, 64), _i(2), _i(1), _i(1, 2), window=10,
                                          want_lse=True, **kw))


@pytest.mark.parametrize("name", CALLS_ALL)
@pytest.mark.parametrize("stream", [_Stream(9), 9], ids=["object", "address"])
def test_memory_for_another_stream_is_that_streams(pages, traced, name, stream):
    """Outputs and workspaces of a call on a stream that is not the current one are allocated with that stream current; outputs are
    marked as in use on the current stream."""
    fake, _ = traced
    CALLS_ALL[name](pages, stream=stream)
    assert fake.made and fake.on == [9] * len(fake.made) and fake.cuda.current == 7
    for (_, _, dtype), used in zip(fake.made, fake.used):
        assert used == ([] if dtype == torch.uint8 else [7])


@pytest.mark.parametrize("name", CALLS_ALL)
@pytest.mark.parametrize("stream", [None, _Stream(7), 7], ids=["none", "object", "address"])
def test_memory_on_the_current_stream(pages, traced, name, stream):
    fake, _ = traced
    CALLS_ALL[name](pages, stream=stream)
    assert fake.made and fake.on == [7] * len(fake.made) and not any(fake.used)


def test_metadata_is_checked(pages, traced):
    """Wrong types, shapes, strides: refused before the entry point is called."""
    _, calls = traced
    q, k, pos = _z(2, 9, 64), _z(1, 9, 64), _i(9, 1)
    kp, t = _z(3, 1, 4, 64), _i(2, 5)
    heads = lambda **kw: pages.ress_qk_norm_rope(**dict(dict(q=q, k=k, pos=pos, dims=(64,)), **kw))
    into = lambda **kw: pages.ress_qk_norm_rope_pages(**dict(dict(q=q, k=k, v=k, pos=pos, slots=_i(9), k_pages=kp, v_pages=kp, dims=(64,)), **kw))
    tables = lambda **kw: pages.ress_page_tables(**dict(dict(lens=_i(2), new_lens=_i(2), tables=t, free_pages=_i(9), n_free=_i(1), page=4,
                                                             tokens=7), **kw))
    attn = lambda **kw: pages.ress_paged_attn(**dict(dict(q=q, k_pages=kp, v_pages=kp, cu_q=_i(3), lens=_i(2), tables=t, window=5), **kw))
    bwd = lambda **kw: pages.ress_qk_norm_rope_bwd(**dict(dict(dq_out=q, dk_out=k, q=q, k=k, pos=pos, dims=(64,)), **kw))
    wide = torch.zeros(2, 9, 128, dtype=torch.bfloat16)[..., ::2]
    f32 = lambda *s: torch.zeros(s, dtype=F32)
    for call, bad in ((heads, dict(q=wide)), (heads, dict(k=k.float())), (heads, dict(k=_z(1, 8, 64))), (heads, dict(pos=None)),
                      (heads, dict(pos=_i(9, 2))), (heads, dict(pos=pos.long())), (heads, dict(q_gamma=f32(63))),
                      (heads, dict(k_beta=_z(64))), (heads, dict(q_out=_z(2, 9, 32))), (heads, dict(norm="batch")),
                      (heads, dict(layout="spiral")), (heads, dict(dims=())), (heads, dict(dims=(2,) * 5)), (heads, dict(q=None, k=None)),
                      (heads, dict(q=_z(9, 64))), (into, dict(v=None)), (into, dict(k=None)), (into, dict(slots=None)),
                      (into, dict(slots=_i(8))), (into, dict(k_pages=_z(3, 2, 4, 64))), (into, dict(v_pages=_z(3, 1, 5, 64))),
                      (into, dict(v_pages=kp.float())), (into, dict(v=_z(1, 9, 32))), (tables, dict(lens=_i(3))), (tables, dict(lens=None)),
                      (tables, dict(tables=t[:, ::2])), (tables, dict(tables=t.long())), (tables, dict(n_free=_i(2))),
                      (tables, dict(tokens=None)), (tables, dict(free_pages=None)), (tables, dict(slots=_i(6))), (tables, dict(cu_q=_i(2))),
                      (attn, dict(q=q.float())), (attn, dict(k_pages=_z(3, 1, 4, 32))), (attn, dict(v_pages=_z(2, 1, 4, 64))),
                      (attn, dict(cu_q=_i(2))), (attn, dict(cu_q=None)), (attn, dict(lens=_i(3))), (attn, dict(tables=None)),
                      (attn, dict(lse=f32(2, 8))), (attn, dict(out=_z(2, 8, 64))), (attn, dict(q=wide)), (bwd, dict(dq_out=_z(2, 8, 64))),
                      (bwd, dict(dk=k.float())), (bwd, dict(k_dbeta=f32(32))), (bwd, dict(q_gamma=_z(64)))):
        with pytest.raises(ValueError):
            call(**bad)
    for call in (heads, into, tables, attn, bwd):
        with pytest.raises(ValueError):
            call(**({"page": 2 ** 40} if call is tables else {"window": 2.5} if call is attn else {"eps": "x"}))
    assert not calls
