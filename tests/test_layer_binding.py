"""What the binding of include/ress_layer.h does with memory, on the CPU: its calls are followed up to the C entry point,
which is replaced, with host tensors in the place of the device's."""
import contextlib
import weakref

import pytest
import torch

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture
def layer():
    from paper_2609_35593_amd import layer

    return layer


@pytest.fixture
def memory():
    from paper_2609_35593_amd import memory

    return memory


class _Stream:
    def __init__(self, address):
        self.cuda_stream = address

    def __eq__(self, other):
        return self.cuda_stream == other.cuda_stream


class _Cuda:
    """Streams by address, 7 the current one outside every context."""

    def __init__(self):
        self.current = 7

    @contextlib.contextmanager
    def stream(self, s):
        before, self.current = self.current, s.cuda_stream
        yield
        self.current = before

    def current_stream(self, device=None):
        return _Stream(self.current)

    def ExternalStream(self, address, device=None):
        return _Stream(address)


class _Torch:
    """The binding's torch: `made` notes what it allocates, `on` the stream that was current then, `used` what the tensors
    are marked as in use on."""

    def __init__(self):
        self.made, self.on, self.used, self.cuda = [], [], [], _Cuda()

    def __getattr__(self, name):
        return getattr(torch, name)

    def _note(self, t):
        self.made.append((weakref.ref(t), t.data_ptr(), t.dtype))
        self.on.append(self.cuda.current)
        used = []
        self.used.append(used)
        t.record_stream = lambda s: used.append(s.cuda_stream)
        return t

    def empty(self, *a, **kw):
        return self._note(torch.empty(*a, **kw))

    def empty_strided(self, *a, **kw):
        return self._note(torch.empty_strided(*a, **kw))


@pytest.fixture
def traced(layer, memory, monkeypatch):
    """(torch's stand-in, list that each call's address arguments are appended to)."""
    fake, calls = _Torch(), []

    def call(fn, device, stream, *args):
        calls.append((fn.__name__, [a for a in args if isinstance(a, int)], [(p, r() is not None) for r, p, _ in fake.made]))

    monkeypatch.setattr(memory, "torch", fake)
    monkeypatch.setattr(layer, "_device", lambda name, t: t.device)
    monkeypatch.setattr(layer, "_call", call)
    monkeypatch.setattr(memory, "raw_stream", lambda index: fake.cuda.current)
    return fake, calls


def _z(*shape, dtype=BF):
    return torch.zeros(shape, dtype=dtype)


# Calls that need a workspace and are given none.
CALLS = {
    "ress_layer_norm_bwd": lambda b, **kw: b.ress_layer_norm_bwd(_z(40, 64), _z(40, 64, dtype=F32), None, _z(40, dtype=F32),
                                                                 _z(40, dtype=F32), **kw),
    "ress_window_attn": lambda b, **kw: b.ress_window_attn(_z(1, 1, 64), _z(1, 5000, 64), _z(1, 5000, 64), window=5000,
                                                           q_offset=4999, **kw),
    "ress_window_attn_bwd": lambda b, **kw: b.ress_window_attn_bwd(_z(2, 90, 64), _z(2, 90, 64), _z(1, 90, 64), _z(1, 90, 64),
                                                                   _z(2, 90, 64), _z(2, 90, dtype=F32), window=30, **kw),
    "ress_window_attn_decode": lambda b, **kw: b.ress_window_attn_decode(_z(1, 4, 64), _z(1, 4, 9000, 64), _z(1, 4, 9000, 64),
                                                                         torch.zeros(1, dtype=torch.int32), window=9000, **kw),
}


@pytest.mark.parametrize("name", CALLS)
def test_workspace_lives_until_its_kernels_are_enqueued(layer, traced, name):
    """A workspace that the binding makes is held while the entry point runs: a block returned before that may be given to
    another thread's call, or, on a stream of the caller's, counted as idle before its kernels are there."""
    fake, calls = traced
    CALLS[name](layer)
    (called, addresses, made), = calls
    assert called == name
    workspaces = [m for m, (_, _, dtype) in zip(made, fake.made) if dtype == torch.uint8]
    assert len(workspaces) == 1
    (address, alive), = workspaces
    assert address in addresses and alive


CALLS_ALL = dict(
    CALLS,
    ress_layer_norm=lambda b, **kw: b.ress_layer_norm(_z(40, 64), want_stats=True, **kw),
    ress_rope=lambda b, **kw: b.ress_rope(_z(2, 5, 64), _z(1, 5, 64), torch.zeros(5, 2, dtype=torch.int32), dims=(32, 32), **kw),
    lse=lambda b, **kw: b.ress_window_attn(_z(1, 5, 64), _z(1, 5, 64), _z(1, 5, 64), window=5, want_lse=True, **kw))


@pytest.mark.parametrize("name", CALLS_ALL)
@pytest.mark.parametrize("stream", [_Stream(9), 9], ids=["object", "address"])
def test_memory_for_another_stream_is_that_streams(layer, traced, name, stream):
    """Outputs and workspaces of a call on a stream that is not the current one are allocated with that stream current: a
    block of the current stream's may still be in use by work queued there, which the other does not wait for. Outputs are
    marked as in use on the current stream, where the caller goes on with them."""
    fake, _ = traced
    CALLS_ALL[name](layer, stream=stream)
    assert fake.made and fake.on == [9] * len(fake.made) and fake.cuda.current == 7
    for (_, _, dtype), used in zip(fake.made, fake.used):
        assert used == ([] if dtype == torch.uint8 else [7])


@pytest.mark.parametrize("name", CALLS_ALL)
@pytest.mark.parametrize("stream", [None, _Stream(7), 7], ids=["none", "object", "address"])
def test_memory_on_the_current_stream(layer, traced, name, stream):
    fake, _ = traced
    CALLS_ALL[name](layer, stream=stream)
    assert fake.made and fake.on == [7] * len(fake.made) and not any(fake.used)


# ----------------------------------------------------- the functions of include/ress.h


def _select(r, **kw):
    q = _z(4, 200, 64)
    return r.ress_select(q, q, q, _z(4, 64, 64, dtype=F32), [1] * 4, bq=128, bk=128, want_debug=True, **kw)


BASE = {
    "ress_select": _select,
    "ress_sparse_attn": lambda r, **kw: r.ress_sparse_attn(*[_z(4, 200, 64)] * 3, _z(4, 2, dtype=torch.int32),
                                                           _z(4, 2, 2, dtype=torch.int32), bq=128, bk=128, **kw),
    "ress_sparse_attn_out_f32": lambda r, **kw: r.ress_sparse_attn_out_f32(*[_z(4, 200, 64)] * 3, _z(4, 2, dtype=torch.int32),
                                                                           _z(4, 2, 2, dtype=torch.int32), bq=128, bk=128, **kw),
    "ress_dense_attn": lambda r, **kw: r.ress_dense_attn(*[_z(4, 200, 64)] * 3, bq=128, bk=128, **kw),
    "ress_qkv_proj_pool": lambda r, **kw: r.ress_qkv_proj_pool(_z(200, 256), _z(768, 256), _z(4, 64, 64, dtype=F32), bq=128,
                                                               bk=128, **kw),
    "ress_out_proj_residual": lambda r, **kw: r.ress_out_proj_residual(_z(4, 200, 64), _z(256, 256), _z(200, 256), **kw),
    "ress_out_proj_residual_f32": lambda r, **kw: r.ress_out_proj_residual_f32(_z(4, 200, 64), _z(256, 256),
                                                                               _z(200, 256, dtype=F32), **kw),
    "ress_block_drift_sq": lambda r, **kw: r.ress_block_drift_sq(_z(4, 200, 64, dtype=F32), _z(4, 200, 64, dtype=F32),
                                                                 _z(4, 64, 64, dtype=F32), bq=128, **kw),
}


class _Lib:
    """Entry points that enqueue nothing, and the real sizes."""

    def __init__(self, real):
        self.real = real

    def __getattr__(self, name):
        return getattr(self.real, name) if name.endswith("_size") else lambda *a: 0


@pytest.mark.parametrize("name", BASE)
@pytest.mark.parametrize("stream", [_Stream(9), 9], ids=["object", "address"])
def test_memory_of_the_attention_path_is_the_streams(memory, monkeypatch, name, stream):
    """The same for the functions of include/ress.h: all that they return is marked as in use on the current stream, the
    projection's workspace too; the selection's own workspace is not returned."""
    import paper_2609_35593_amd as r

    fake = _Torch()
    monkeypatch.setattr(memory, "torch", fake)
    monkeypatch.setattr(memory, "raw_stream", lambda index: fake.cuda.current)
    monkeypatch.setattr(r, "lib", _Lib(r.lib))
    for check in ("_check_qkv", "_check_out", "_check_bf16"):
        monkeypatch.setattr(r, check, lambda *a: None)
    monkeypatch.setattr(r, "_workspace_bytes", lambda t, dev: t.numel())
    if "sparse" in name:
        monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    BASE[name](r, stream=stream)
    assert fake.made and fake.on == [9] * len(fake.made) and fake.cuda.current == 7
    for (_, _, dtype), used in zip(fake.made, fake.used):
        assert used == ([] if dtype == torch.uint8 and name == "ress_select" else [7])


def test_masking_reference_stays_on_its_stream(monkeypatch):
    """Lists made, kernels' calls and the copy to the host of block_masking_change all belong to the stream that it is
    given: made on the current one, its lists and the copy would not wait for the kernels, nor they for the lists."""
    from paper_2609_35593_amd import masking

    fake, on = _Torch(), []

    def made(name):
        def f(*a, **kw):
            on.append((name, fake.cuda.current))
            return getattr(torch, name)(*a, **kw)
        return f

    for name in ("arange", "full", "cat", "empty_like"):
        setattr(fake, name, made(name))

    def attention(q, k, v, count, kept, *, bq, bk, out=None, stream=None):
        on.append(("attention", stream.cuda_stream if stream is not None else fake.cuda.current))
        return torch.zeros(q.shape) if out is None else out

    def drift(a, b, gram, *, bq, out, stream=None):
        on.append(("drift", stream.cuda_stream if stream is not None else fake.cuda.current))
        return out.fill_(4.0)

    monkeypatch.setattr(masking, "torch", fake)
    monkeypatch.setattr(masking, "ress_sparse_attn_out_f32", attention)
    monkeypatch.setattr(masking, "ress_block_drift_sq", drift)
    q = _z(2, 300, 64)
    for stream, where in ((_Stream(9), 9), (9, 9), (None, 7)):
        on.clear()
        fake.on.clear()
        r = masking.block_masking_change(q, q, q, _z(2, 64, 64, dtype=F32), bq=128, bk=128, stream=stream)
        assert r.shape == (2, 3, 3) and (r == 2).all() and fake.cuda.current == 7
        assert {s for _, s in on} == {where} and set(fake.on) == {where} and len(on) > 10
