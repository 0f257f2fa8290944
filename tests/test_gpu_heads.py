"""Norm of heads with the rotary positions against float64: forward, into pages, backward; layouts, widths, types, strides, in place,
captured calls."""
import pytest
import torch

import pages_refs as PR
from gpu_helpers import say
from layer_refs import within

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
WIDTHS = [(64, (32, 32)), (64, (64,)), (64, (16, 24, 24)), (64, (20, 20, 24)), (64, (8, 8)), (128, (32, 48, 32)),
          (256, (64, 64, 64, 64)), (256, (62, 64)), (2, (2,)), (6, (2, 2)), (48, (16, 16, 16)), (64, (0, 32)), (64, (0,)),
          (80, (48, 16)), (200, (100, 100)), (130, (130,))]


@pytest.fixture(scope="module")
def ress():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_35593_amd as r

    return r


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _inputs(seed, H, H_kv, N, D, axes, dtype, far=1000):
    g = _gen(seed)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    q, k = ((rn(h, N, D) * 1.5 + rn(D)).to(dtype) for h in (H, H_kv))
    pos = torch.randint(-far, far + 1, (N, axes), generator=g, device="cuda", dtype=torch.int32)
    w = dict(q_gamma=1 + 0.3 * rn(D), q_beta=0.2 * rn(D), k_gamma=1 + 0.3 * rn(D), k_beta=0.2 * rn(D))
    return q, k, pos, w


def _check(r, q, k, pos, w, norm, eps, dims, layout, base):
    for n, x in (("q", q), ("k", k)):
        if x is not None:
            y, b = PR.heads(x, pos, w.get(n + "_gamma"), w.get(n + "_beta"), norm, eps, dims, layout, base)
            within(r[n], y, b, f"{n} {norm} {layout}")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("layout", ["split", "interleaved", "sections"])
@pytest.mark.parametrize("D,dims", WIDTHS)
def test_forward(ress, D, dims, layout, dtype):
    say(f"[heads] D {D} {dims} {layout} {dtype}")
    for i, (H, H_kv, N) in enumerate(((3, 1, 77), (1, 5, 1), (9, 2, 300), (2, 7, 9001))):
        q, k, pos, w = _inputs(D + N, H, H_kv, N, D, len(dims), dtype)
        norm = ("layer", "rms")[i % 2]
        if i == 2:
            w.pop("q_beta"), w.pop("k_gamma")
        if i == 3:
            w = {}
        r = ress.ress_qk_norm_rope(q, k, pos, dims=dims, norm=norm, layout=layout, base=1e4, **w)
        _check(r, q, k, pos, w, norm, 1e-5, dims, layout, 1e4)


def _grads(ress, q, k, gq, gk, pos, w, norm, dims, layout, base=1e4, eps=1e-5, **kw):
    gam = {n: t for n, t in w.items() if n.endswith("gamma")}
    return ress.ress_qk_norm_rope_bwd(gq, gk, q, k, pos, dims=dims, norm=norm, layout=layout, base=base, eps=eps, **gam, **kw)


def _check_bwd(r, q, k, dq, dk, pos, w, norm, dims, layout, base=1e4, eps=1e-5):
    for n, x, dy in (("q", q, dq), ("k", k, dk)):
        if x is not None:
            ref, b = PR.heads_bwd(dy, x, pos, w.get(n + "_gamma"), norm, eps, dims, layout, base)
            for name, want, bound in zip(("d" + n, n + "_dgamma", n + "_dbeta"), ref, b):
                if r.get(name) is not None:
                    within(r[name], want, bound, f"{name} {norm} {layout}")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("layout", ["split", "interleaved", "sections"])
@pytest.mark.parametrize("D,dims", WIDTHS)
def test_backward(ress, D, dims, layout, dtype):
    say(f"[heads bwd] D {D} {dims} {layout} {dtype}")
    for i, (H, H_kv, N) in enumerate(((3, 1, 77), (1, 5, 1), (9, 2, 300), (2, 3, 9001))):
        q, k, pos, w = _inputs(D + N, H, H_kv, N, D, len(dims), dtype)
        dq, dk, _, _ = _inputs(D + N + 1, H, H_kv, N, D, len(dims), dtype)
        norm = ("rms", "layer")[i % 2]
        if i == 2:
            w.pop("q_gamma")
        r = _grads(ress, q, k, dq, dk, pos, w, norm, dims, layout)
        _check_bwd(r, q, k, dq, dk, pos, w, norm, dims, layout)
        again = _grads(ress, q, k, dq, dk, pos, w, norm, dims, layout)
        assert all(torch.equal(r[n], again[n]) for n in r)


def test_many_tokens(ress):
    """More tokens than workgroups of the backward pass have at once; few heads and many."""
    for H, H_kv, N in ((1, 1, 100003), (16, 4, 20011), (1, 0, 70001), (0, 2, 5)):
        q, k, pos, w = _inputs(N, H, H_kv, N, 64, 2, BF)
        dq, dk, _, _ = _inputs(N + 1, H, H_kv, N, 64, 2, BF)
        q, dq = (q, dq) if H else (None, None)
        k, dk = (k, dk) if H_kv else (None, None)
        r = ress.ress_qk_norm_rope(q, k, pos, dims=(32, 32), **w)
        _check(r, q, k, pos, w, "layer", 1e-5, (32, 32), "split", 100.0)
        g = _grads(ress, q, k, dq, dk, pos, w, "layer", (32, 32), "split", 100.0)
        _check_bwd(g, q, k, dq, dk, pos, w, "layer", (32, 32), "split", 100.0)
        for n, x in (("q", q), ("k", k)):
            if x is None:
                assert r[n] is None and g["d" + n] is None and not g[n + "_dgamma"].any() and not g[n + "_dbeta"].any()


def test_far_positions_keep_their_phase(ress):
    q, k, pos, w = _inputs(1, 2, 2, 500, 64, 2, F32, far=1 << 24)
    r = ress.ress_qk_norm_rope(q, k, pos, dims=(32, 32), norm="rms", **w)
    _check(r, q, k, pos, w, "rms", 1e-5, (32, 32), "split", 100.0)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("scale", [2.0 ** -60, 2.0 ** 56])
def test_tiny_and_huge_rows(ress, scale, dtype):
    """Rows whose squares leave float32's small end (eps decides) or come near its large one; rows of one value."""
    q, k, pos, w = _inputs(2, 2, 2, 50, 64, 1, dtype)
    q, k = ((x.float().clamp(-1, 1) * scale).to(dtype) for x in (q, k))
    q[:, 7] = 0.0
    k[:, 9] = 0.25
    for norm in ("layer", "rms"):
        r = ress.ress_qk_norm_rope(q, k, pos, dims=(64,), norm=norm, **w)
        _check(r, q, k, pos, w, norm, 1e-5, (64,), "split", 100.0)


def _strided(x, kind, dtype):
    """x's values in another layout."""
    H, N, D = x.shape
    if kind == "token_major":
        y = torch.empty(N, H, D, dtype=dtype, device="cuda").transpose(0, 1)
    elif kind == "packed":  # a slice of a packed projection
        y = torch.zeros(N, 3 * H * D + 16, dtype=dtype, device="cuda")[:, 16:16 + H * D].view(N, H, D).transpose(0, 1)
    else:  # odd strides and address
        y = torch.zeros(H * (N * (D + 3) + 5) + 1, dtype=dtype, device="cuda")[1:].as_strided((H, N, D), (N * (D + 3) + 5, D + 3, 1))
    y.copy_(x)
    return y


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("kind", ["token_major", "packed", "odd"])
@pytest.mark.parametrize("dims", [(32, 32), (20, 24)])
def test_strides_and_in_place(ress, dims, kind, dtype):
    q, k, pos, w = _inputs(3, 4, 2, 333, 64, 2, dtype)
    dq, dk, _, _ = _inputs(4, 4, 2, 333, 64, 2, dtype)
    qs, ks, dqs, dks = (_strided(x, kind, dtype) for x in (q, k, dq, dk))
    r = ress.ress_qk_norm_rope(qs, ks, pos, dims=dims, q_out=torch.empty_like(q), **w)
    _check(r, q, k, pos, w, "layer", 1e-5, dims, "split", 100.0)
    g = _grads(ress, qs, ks, dqs, dks, pos, w, "layer", dims, "split", 100.0)
    _check_bwd(g, q, k, dq, dk, pos, w, "layer", dims, "split", 100.0)
    for in_place in ("of the gradients", "of the inputs"):
        a, b, c, d = (_strided(x, kind, dtype) for x in (q, k, dq, dk))
        to = (c, d) if in_place == "of the gradients" else (a, b)
        g2 = _grads(ress, a, b, c, d, pos, w, "layer", dims, "split", 100.0, dq=to[0], dk=to[1])
        assert all(torch.equal(g[n], g2[n]) for n in g), in_place
    r2 = ress.ress_qk_norm_rope(qs, ks, pos, dims=dims, q_out=qs, k_out=ks, **w)
    assert torch.equal(r2["q"], r["q"]) and torch.equal(r2["k"], r["k"])
    assert r2["q"].data_ptr() == qs.data_ptr()


def test_gradients_wanted_apart(ress):
    q, k, pos, w = _inputs(5, 2, 2, 60, 64, 1, BF)
    dq, dk, _, _ = _inputs(6, 2, 2, 60, 64, 1, BF)
    full = _grads(ress, q, k, dq, dk, pos, w, "layer", (64,), "split")
    one = _grads(ress, q, k, dq, dk, pos, w, "layer", (64,), "split", k_dbeta=torch.empty(64, device="cuda"))
    assert torch.equal(one["k_dbeta"], full["k_dbeta"]) and one["q_dgamma"] is None and torch.equal(one["dq"], full["dq"])
    none = _grads(ress, q, k, dq, dk, pos, w, "layer", (64,), "split", want_weights=False)
    assert torch.equal(none["dk"], full["dk"]) and none["k_dgamma"] is None
    z = torch.zeros(2, 0, 64, dtype=BF, device="cuda")
    r = _grads(ress, z, z, z, z, pos[:0], w, "layer", (64,), "split")
    assert not any(r[n].any() for n in ("q_dgamma", "q_dbeta", "k_dgamma", "k_dbeta"))


def test_gradients_against_differences(ress):
    """Of the call's own forward pass in float32, a channel at a time: central differences of 2^-6 are off by their third
    derivative, some 2^-12 of values of order one, and by 64 x 2^-23 / 2^-5 of the forward pass's roundings."""
    q, k, pos, w = _inputs(7, 1, 1, 3, 64, 2, F32, far=30)
    dq, dk, _, _ = _inputs(8, 1, 1, 3, 64, 2, F32)
    kw = dict(dims=(32, 32), norm="layer")
    g = ress.ress_qk_norm_rope_bwd(dq, dk, q, k, pos, q_gamma=w["q_gamma"], k_gamma=w["k_gamma"], **kw)
    f = lambda x: (ress.ress_qk_norm_rope(x, k, pos, **kw, **w)["q"].double() * dq.double()).sum()
    for c in (0, 5, 16, 40, 63):
        e = torch.zeros_like(q)
        e[0, 1, c] = 2.0 ** -6
        d = (f(q + e) - f(q - e)) / 2.0 ** -5
        scale = (dq[0, 1].double().abs().sum()).item()
        assert abs(d.item() - g["dq"][0, 1, c].item()) < 2.0 ** -11 * scale, c


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D,dims,page", [(64, (32, 32), 16), (64, (64,), 7), (64, (20, 24), 64), (128, (128,), 1), (6, (2, 2), 5)])
def test_into_pages(ress, D, dims, page, dtype):
    """Each token in its slot, the rest of the pages untouched; tokens without a slot leave nothing."""
    say(f"[heads pages] D {D} page {page} {dtype}")
    H, H_kv, N, n_pages = 5, 3, 211, 400 // page + 3
    q, k, pos, w = _inputs(D + page, H, H_kv, N, D, len(dims), dtype)
    v = torch.randn(H_kv, N, D, generator=_gen(9), device="cuda").to(dtype)
    v[1, 5, 1] = float("nan")  # (copied as it is)
    slots = torch.randperm(n_pages * page, generator=_gen(10), device="cuda")[:N].int()
    slots[3], slots[50], slots[100], slots[101] = -1, n_pages * page, 2 ** 31 - 1, -2 ** 31
    for kind in ("plain", "tokens first", "far apart"):
        shape = (n_pages, H_kv, page, D)
        mk = {"plain": lambda: torch.full(shape, 7.0, dtype=dtype, device="cuda"),
              "tokens first": lambda: torch.full((n_pages, page, H_kv, D), 7.0, dtype=dtype, device="cuda").transpose(1, 2),
              "far apart": lambda: torch.full((H_kv, n_pages, page, D + 1), 7.0, dtype=dtype, device="cuda").transpose(0, 1)[..., :D]}
        kp, vp = mk[kind](), mk[kind]()
        r = ress.ress_qk_norm_rope_pages(q, k, v, pos, slots, kp, vp, dims=dims, norm="rms", **w)
        yq, bq = PR.heads(q, pos, w["q_gamma"], w["q_beta"], "rms", 1e-5, dims, "split", 100.0)
        within(r["q"], yq, bq, "q")
        plain = ress.ress_qk_norm_rope(q, k, pos, dims=dims, norm="rms", **w)
        ok = (slots >= 0) & (slots < n_pages * page)
        at = slots[ok].long()
        wk, wv = mk["plain"](), mk["plain"]()
        wk[at // page, :, at % page] = plain["k"][:, ok].transpose(0, 1)
        wv[at // page, :, at % page] = v[:, ok].transpose(0, 1)
        if kind == "far apart":  # (other alignments sum a row in another order: within the bound, the rest untouched)
            yk, bk = PR.heads(k, pos, w["k_gamma"], w["k_beta"], "rms", 1e-5, dims, "split", 100.0)
            within(kp[at // page, :, at % page].transpose(0, 1), yk[:, ok], bk[:, ok], "k")
            kp[at // page, :, at % page] = wk[at // page, :, at % page]
        assert torch.equal(kp, wk), kind
        assert torch.equal(vp.contiguous().view(torch.uint8), wv.view(torch.uint8)), kind
    kp, kp2, vp2 = mk["plain"](), mk["plain"](), mk["plain"]()
    ress.ress_qk_norm_rope_pages(q, k, v, pos, slots, kp, vp2, dims=dims, norm="rms", **w)
    ress.ress_qk_norm_rope_pages(None, k, v, pos, slots, kp2, vp2, dims=dims, norm="rms", **w)
    assert torch.equal(kp2[at // page, :, at % page], kp[at // page, :, at % page])


def test_pages_beyond_32_bits(ress):
    """Slots whose rows lie behind 2^31 elements."""
    page, n_pages = 1 << 12, 520
    kp = torch.zeros(n_pages, 1, page, 1024, dtype=BF, device="cuda")[..., :64]  # 2^31.02 elements
    vp = torch.zeros(n_pages, 1, page, 64, dtype=BF, device="cuda")
    q, k, pos, w = _inputs(11, 1, 1, 3, 64, 1, BF)
    slots = torch.tensor([n_pages * page - 1, 512 * page + 5, 0], dtype=torch.int32, device="cuda")
    ress.ress_qk_norm_rope_pages(q, k, k, pos, slots, kp, vp, dims=(64,), **w)
    want = ress.ress_qk_norm_rope(q, k, pos, dims=(64,), **w)["k"]
    for t, (a, b) in enumerate(((n_pages - 1, page - 1), (512, 5), (0, 0))):
        assert torch.equal(kp[a, 0, b], want[0, t]) and torch.equal(vp[a, 0, b], k[0, t])


def test_captured_calls(ress):
    """Forward, backward and into pages in one graph, replayed beside eager work on other data; every replay as the eager calls."""
    N, H, H_kv = 700, 8, 2
    q, k, pos, w = _inputs(12, H, H_kv, N, 64, 2, BF)
    dq, dk, _, _ = _inputs(13, H, H_kv, N, 64, 2, BF)
    slots = torch.arange(N, device="cuda", dtype=torch.int32)
    kp, vp = (torch.zeros(50, H_kv, 16, 64, dtype=BF, device="cuda") for _ in range(2))
    ws = torch.empty(ress.ress_qk_norm_rope_bwd_workspace_size(H, H_kv, N, 64), dtype=torch.uint8, device="cuda")
    kw = dict(dims=(32, 32), layout="split")

    def calls():
        return (ress.ress_qk_norm_rope(q, k, pos, **kw, **w), _grads(ress, q, k, dq, dk, pos, w, "layer", (32, 32), "split", workspace=ws),
                ress.ress_qk_norm_rope_pages(q, k, k, pos, slots, kp, vp, **kw, **w))

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = calls()
    for turn in range(3):
        for x in (q, k, dq, dk):
            x.copy_(torch.randn(x.shape, generator=_gen(20 + turn), device="cuda"))
        slots.copy_(torch.randperm(800, generator=_gen(30 + turn), device="cuda")[:N])
        graph.replay()
        torch.cuda.synchronize()
        got = [{n: t.clone() for n, t in c.items()} for c in captured]
        want = calls()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(a[n], b[n]) for n in b), turn
