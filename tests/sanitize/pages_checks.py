"""Host code of ress_pages.h's C ABI and plans under AddressSanitizer and UndefinedBehaviorSanitizer, in a child process (no
GPU, no torch): shapes at and beyond every limit and random ones; what passes validation ends in a launcher that looks at its
parameters and fails (RESS_E_HIP).
Usage: python pages_checks.py <library>"""
import ctypes as C
import itertools
import random
import sys

from layer_structs import ress_rope_shape, ress_strides
from pages_structs import (ress_head_norm_grads, ress_head_norm_shape, ress_page_cache, ress_page_strides, ress_paged_shape,
                           ress_table_shape)

lib = C.CDLL(sys.argv[1])
vp, f32, sz = C.c_void_p, C.c_float, C.c_size_t
lib.ress_qk_norm_rope.argtypes = [vp] * 11
lib.ress_qk_norm_rope_pages.argtypes = [vp] * 15
lib.ress_qk_norm_rope_bwd.argtypes = [vp] * 16 + [sz, vp]
lib.ress_page_tables.argtypes = [vp] * 13
lib.ress_pages_release.argtypes = [vp] * 8 + [sz, vp]
lib.ress_paged_attn.argtypes = [vp] * 7 + [f32, vp, vp, vp, sz, vp]
P = [(1 << 41) + (n << 33) for n in range(16)]
BIG, TOP, TOKENS = 1 << 60, (1 << 31) - 1, 1 << 24
E_HIP = -4
edge = (-(1 << 31), -1, 0, 1, 2, TOKENS, TOKENS + 1, TOP)
rng = random.Random(12)
checks = 0


def legal(st):
    global checks
    checks += 1
    assert st in (0, -1, -2, -3, -4), st
    return st


def size(fn, s):
    n = sz(0)
    st = legal(fn(C.byref(s), C.byref(n)))
    return n.value if st == 0 else None


# ------------------------------------------------------------ norm of heads
reached = {"fwd": 0, "pages": 0, "bwd": 0}
strides = [lambda D: (D * 100, D), lambda D: (D, D * 4), lambda D: (1 << 46, 1 << 22), lambda D: (0, 0), lambda D: (1 << 62, 1 << 62),
           lambda D: (-8, 8), lambda D: ((D + 1) * 101, D + 1), lambda D: (7, 3)]
for D, axes, dims, layout, dtype in itertools.product(
        (2, 6, 48, 64, 80, 128, 250, 256), (1, 2, 3, 4),
        ((64, 0, 0, 0), (32, 32, 0, 0), (2, 2, 2, 0), (0, 64, 0, 16), (16, 24, 24, 0), (128, 64, 32, 32), ((TOP - 1),) * 4, (10, 14, 8, 4)),
        (0, 1, 2), (0, 1)):
    for st in strides:
        x = ress_strides(*st(D))
        rope = ress_rope_shape(4, 2, 100, D, axes, (C.c_int * 4)(*dims), layout, 0, dtype, 100.0, x, x, x, x)
        s = ress_head_norm_shape(rope, D // 2 % 2, 1e-5)
        reached["fwd"] += legal(lib.ress_qk_norm_rope(C.byref(s), *P[:9], None)) == E_HIP
        for odd in (0, 4):  # (pages aligned to less than a chunk)
            pg = ress_page_strides(1 << 20, 1 << 14, D + odd)
            c = ress_page_cache(10, 16, pg, pg, x)
            reached["pages"] += legal(lib.ress_qk_norm_rope_pages(C.byref(s), C.byref(c), *P[:12], None)) == E_HIP
        n = size(lib.ress_qk_norm_rope_bwd_workspace_size, s)
        g = ress_head_norm_grads(x, x, x, x)
        got = legal(lib.ress_qk_norm_rope_bwd(C.byref(s), C.byref(g), *P[:13], P[13], n or 0, None))
        reached["bwd"] += got == E_HIP
        if got == E_HIP:
            assert legal(lib.ress_qk_norm_rope_bwd(C.byref(s), C.byref(g), *P[:13], P[13], n - 1, None)) == -3
assert min(reached.values()) > 300, reached
x = ress_strides(64 << 24, 64)
for field, value in itertools.product(("H", "H_kv", "N", "D", "n_axes", "layout", "inverse", "dtype"), edge):
    rope = ress_rope_shape(4, 2, 100, 64, 1, (C.c_int * 4)(64), 0, 0, 0, 100.0, x, x, x, x)
    setattr(rope, field, value)
    s = ress_head_norm_shape(rope, 0, 1e-5)
    legal(lib.ress_qk_norm_rope(C.byref(s), *P[:9], None))
    n = size(lib.ress_qk_norm_rope_bwd_workspace_size, s)
    assert n is None or n <= 4 << 20
    g = ress_head_norm_grads(x, x, x, x)
    legal(lib.ress_qk_norm_rope_bwd(C.byref(s), C.byref(g), *P[:13], P[13], BIG, None))
for n_pages, page, st in itertools.product(edge, edge, ((0, 0, 0), (1 << 20, 64, 128), (1 << 62, 1 << 62, 1 << 62), (64, 1 << 40, 1 << 30),
                                                        (1 << 31, 1 << 46, 1 << 22), (-1, -1, -1))):
    rope = ress_rope_shape(4, 2, 100, 64, 1, (C.c_int * 4)(64), 0, 0, 0, 100.0, x, x, x, x)
    pg = ress_page_strides(*st)
    s, c = ress_head_norm_shape(rope, 1, 1e-5), ress_page_cache(n_pages, page, pg, pg, x)
    legal(lib.ress_qk_norm_rope_pages(C.byref(s), C.byref(c), *P[:12], None))
out = (C.c_int * 5)()
for _ in range(20000):
    H, N, each = rng.choice((0, 1, 2, 20, 511, 512)), rng.choice((0, 1, 2 ** rng.randrange(25), rng.randrange(1, TOKENS))), rng.choice((4, 8, 16, 32, 64, 128))
    lib.plan_head_bwd(H, N, each, out)
    tokens, heads, parts, most = out[:4]
    if H == 0 or N == 0:
        assert parts == 0 and most == 1
        continue
    assert 1 <= tokens <= -(-N // each) and 1 <= heads <= H and parts == tokens * -(-H // heads) and parts <= most <= 768, (H, N, each)
    assert tokens == min(-(-N // each), 768)

# -------------------------------------------------------------------- pages
reached = 0
for B, N, page, n_pages, max_pages in itertools.product((-1, 0, 3, 65535, 65536), (-1, 0, TOKENS, TOKENS + 1), edge, edge, edge):
    for stride in (max_pages, 1 << 46, 1 << 50):
        s = ress_table_shape(B, N, page, n_pages, max_pages, stride, 1)
        reached += legal(lib.ress_page_tables(C.byref(s), *P[:11], None)) == E_HIP
        n = size(lib.ress_pages_release_workspace_size, s)
        assert n is None or n == ((B + 1) * 4 + 255) // 256 * 256
        reached += legal(lib.ress_pages_release(C.byref(s), *P[:6], P[6], BIG, None)) == E_HIP
assert reached > 100, reached

# ---------------------------------------------------------------- attention
seen = {"rows": set(), "splits": set()}


def paged(B, N, H, H_kv, page, n_pages, max_pages, frame, window, sink, k=(1 << 20, 1 << 14, 64)):
    st, pg = ress_strides(64 << 24, 64), ress_page_strides(*k)
    s = ress_paged_shape(B, N, H, H_kv, 64, page, n_pages, max_pages, frame, window, sink, max_pages, st, st, pg, pg)
    what = (B, N, H, H_kv, page, n_pages, max_pages, frame, window, sink)
    n = size(lib.ress_paged_attn_workspace_size, s)
    if n is None:
        return False
    lib.plan_paged(C.byref(s), out)
    rows, blocks, splits, most, target = out[:5]
    assert n <= 100e6, what
    if B and N and H:
        seen["rows"].add(rows)
        seen["splits"].add((rows, splits))
        parts = 0
        if splits > 1:
            parts = H * N * (splits * 264 + 4) if rows == 32 else H_kv * most * 128 * 264 + 16 * blocks
            assert B <= 256 and 1 <= target and most == blocks + target // H_kv + 1, what
        assert n == (parts + (4 * (B + 1) if B > 512 else 0) + 255) // 256 * 256, what
    st = legal(lib.ress_paged_attn(C.byref(s), *P[:6], 0.125, P[6], P[7], P[8], n, None))
    assert st == (E_HIP if B and N and H else 0), (what, st)
    if n:
        assert legal(lib.ress_paged_attn(C.byref(s), *P[:6], 0.125, P[6], P[7], P[8], n - 1, None)) == -3, what
    return True


HEADS = [(1, 1), (8, 2), (16, 16), (256, 1), (256, 256), (12, 4)]
for (H, H_kv), B, N, (page, max_pages) in itertools.product(HEADS, (0, 1, 24, 512, 513, 65535), (0, 1, 127, 1374, TOKENS),
                                                            ((1, TOKENS), (16, 1 << 20), (64, 700), (TOKENS, 1), (24, 0), (7, 1))):
    for frame, window, sink in ((1, 1, 0), (TOP, TOP, TOP), (1, TOP, 0), (1374, 4, 1374)):
        assert paged(B, N, H, H_kv, page, min(TOP // page, 1000), max_pages, frame, window, sink)


def spread(top):
    return rng.choice((0, 1, top, min(top, int(2 ** rng.uniform(0, top.bit_length()))), min(top, int(2 ** rng.uniform(0, top.bit_length())))))


for _ in range(30000):
    H, H_kv = rng.choice(HEADS)
    page = max(1, spread(4096))
    paged(spread(65535), spread(TOKENS), H, H_kv, page, spread(TOP // page), spread(TOKENS // page), max(spread(TOP), 1),
          max(spread(TOP), 1), spread(TOP))
for _ in range(30000):  # sizes of calls that fit a chip
    H, H_kv = rng.choice(HEADS)
    page = rng.choice((1, 7, 16, 24, 64, 128))
    paged(max(1, spread(300)), max(1, spread(8000)), H, H_kv, page, 1000, max(1, spread(50000)) // page, max(spread(2000), 1),
          max(spread(4000), 1), spread(2000))
for field, value in itertools.product(("B", "N", "H", "H_kv", "D", "page", "n_pages", "max_pages", "frame", "window", "n_sink", "table_stride"),
                                      edge + (65535, 65536, 1 << 50)):
    st, pg = ress_strides(64 << 24, 64), ress_page_strides(1 << 20, 1 << 14, 64)
    s = ress_paged_shape(3, 100, 8, 4, 64, 16, 100, 50, 1, 10, 0, 50, st, st, pg, pg)
    if value > TOP and field != "table_stride":
        continue
    setattr(s, field, value)
    size(lib.ress_paged_attn_workspace_size, s)
    legal(lib.ress_paged_attn(C.byref(s), *P[:6], 0.125, P[6], P[7], P[8], BIG, None))
for k in ((0, 0, 0), (1 << 61, 64, 64), (1 << 50, 1 << 46, 1 << 22), (8, 1 << 47, 8), (8, 8, (1 << 22) + 8)):
    paged(3, 100, 8, 4, 16, 100, 50, 1, 10, 0, k=(1 << 20, 1 << 14, 64))
    st, pg = ress_strides(64 << 24, 64), ress_page_strides(*k)
    s = ress_paged_shape(3, 100, 8, 4, 64, 16, 100, 50, 1, 10, 0, 50, st, st, pg, pg)
    legal(lib.ress_paged_attn(C.byref(s), *P[:6], 0.125, P[6], P[7], P[8], BIG, None))
assert seen["rows"] == {32, 128} and {(32, 1), (32, 64), (128, 1), (128, 3), (128, 64)} <= seen["splits"], sorted(seen["splits"])
print(f"pages checks ok: {checks}", flush=True)
