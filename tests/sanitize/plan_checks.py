"""The plans of ress_layer.h's kernels (layer_plan.cpp) under AddressSanitizer and UndefinedBehaviorSanitizer, in a child
process (no GPU, no torch): shapes at every limit and random ones over the whole range, and what the kernels and the
workspaces take for granted of a plan.
Usage: python plan_checks.py <library>"""
import ctypes as C
import itertools
import random
import sys

from layer_structs import ress_decode_shape, ress_strides, ress_window_grads, ress_window_shape

lib = C.CDLL(sys.argv[1])
vp, f32, sz = C.c_void_p, C.c_float, C.c_size_t
lib.plan_norm_bwd.argtypes = [C.c_int64]
lib.ress_window_attn.argtypes = [vp] * 4 + [f32, vp, vp, vp, sz, vp]
lib.ress_window_attn_bwd.argtypes = [vp] * 8 + [f32] + [vp] * 4 + [sz, vp]
lib.ress_window_attn_decode.argtypes = [vp] * 5 + [f32, vp, vp, sz, vp]
P = [(1 << 41) + (n << 33) for n in range(12)]
TOP, TOKENS = (1 << 31) - 1, 1 << 24
E_HIP = -4
rng = random.Random(11)
seen = {"groups": set(), "splits": set(), "bwd": set(), "decode": set()}


def size(fn, s):
    n = sz(0)
    assert fn(C.byref(s), C.byref(n)) == 0
    return n.value


def joined(sinks, sink_slices, slices, blocks):
    """The blocks whose slices the join adds up."""
    first = C.c_int(0)
    n = lib.plan_joined(sinks, sink_slices, slices, blocks, C.byref(first))
    return range(first.value, first.value + n)


def window(H, H_kv, n_q, n_k, off, frame, win, sink, causal):
    x = ress_strides(64 << 24, 64)
    s = ress_window_shape(H, H_kv, n_q, n_k, 64, off, frame, win, sink, causal, x, x, x, x)
    what = (H, H_kv, n_q, n_k, off, frame, win, sink, causal)
    out = (C.c_int * 5)()
    lib.plan_window(C.byref(s), out)
    groups, splits = out[0], out[1]
    assert groups in (1, 2, 4) and 1 <= splits <= 32, what
    seen["groups"].add((groups, splits > 1))
    seen["splits"].add(splits)
    need = size(lib.ress_window_attn_workspace_size, s)
    assert need == (0 if splits == 1 else (splits * H * n_q * 66 * 4 + 255) // 256 * 256), what
    assert need <= 69.2e6, what
    st = lib.ress_window_attn(C.byref(s), P[0], P[1], P[2], 0.125, P[3], P[4], P[5], need, None)
    assert st == (0 if n_q == 0 else E_HIP), (what, st)
    if need:
        assert lib.ress_window_attn(C.byref(s), P[0], P[1], P[2], 0.125, P[3], P[4], P[5], need - 1, None) == -3, what

    lib.plan_window_bwd(C.byref(s), out)
    groups, sinks, sink_slices, slices, items = out
    blocks = (n_k + 127) // 128
    assert groups in (1, 2, 4) and sinks == (min(sink, n_k) + 127) // 128, what
    assert 1 <= sink_slices <= 64 and 1 <= slices <= 16, what
    assert items == sinks * sink_slices + (blocks - sinks) * slices and H_kv * items <= TOP, what
    seen["bwd"].add((sink_slices > 1, slices > 1))
    # Every slice of a list that was cut has a tile; blocks that were cut fit a grid's second dimension.
    all_tiles = (n_q + 63) // 64 * (H // H_kv)
    assert sink_slices <= max(all_tiles, 1) and slices <= max(all_tiles, 1), what
    cut = joined(sinks, sink_slices, slices, blocks)
    assert H_kv * len(cut) <= 65535, what
    need = size(lib.ress_window_attn_bwd_workspace_size, s)
    rows = (H * n_q * 4 + 255) // 256 * 256
    assert need == 2 * rows + (H_kv * items * 2 * 128 * 64 * 4 if sink_slices > 1 or slices > 1 else 0), what
    g = ress_window_grads(x, x, x, x)
    st = lib.ress_window_attn_bwd(C.byref(s), C.byref(g), *P[:6], 0.125, *P[6:9], P[9], need, None)
    assert st == (0 if n_q == 0 and n_k == 0 else E_HIP), (what, st)


def decode(B, H, H_kv, cap, frame, win, sink):
    x = ress_strides(64 << 24, 64)
    s = ress_decode_shape(B, H, H_kv, cap, 64, frame, win, sink, H * 64, 64, 1 << 40, 1 << 40, x, x, H * 64, 64)
    what = (B, H, H_kv, cap, frame, win, sink)
    splits = lib.plan_decode(C.byref(s))
    assert 1 <= splits <= 32, what
    keys = min(frame * win + sink, cap)
    if keys <= 512:
        assert splits == 1, what
    else:  # each split holds a turn of a full window at least
        turn, waves = (32, 8) if H == H_kv else (64, 4)
        turns = (keys + turn - 1) // turn
        each = -(-turns // (splits * waves))
        assert (splits - 1) * waves * each < turns, what
    seen["decode"].add(splits)
    need = size(lib.ress_window_attn_decode_workspace_size, s)
    assert need == (0 if splits == 1 else (B * H * splits * 66 * 4 + 255) // 256 * 256), what
    assert lib.ress_window_attn_decode(C.byref(s), *P[:4], 0.125, P[4], P[5], need, None) == (0 if B == 0 else E_HIP), what


def spread(top):
    """0 to top, evenly over the logarithm, the ends often."""
    return rng.choice((0, 1, top, min(top, int(2 ** rng.uniform(0, top.bit_length()))), min(top, int(2 ** rng.uniform(0, top.bit_length())))))


HEADS = [(1, 1), (8, 2), (16, 16), (256, 1), (256, 256), (12, 4)]
edges = (1, 2, 127, 128, 129, 1374, TOKENS - 1, TOKENS)
for (H, H_kv), n_q, n_k in itertools.product(HEADS, (0,) + edges, (0,) + edges):
    for off, frame, win, sink, causal in ((0, 1, 1, 0, 1), (TOKENS, TOP, TOP, TOP, 0), (5, 1, TOP, 7, 1), (TOKENS, 1374, 4, 1374, 1),
                                          (0, TOP, 1, 200, 0)):
        window(H, H_kv, n_q, n_k, off, frame, win, sink, causal)
for _ in range(20000):
    H, H_kv = rng.choice(HEADS)
    window(H, H_kv, spread(TOKENS), spread(TOKENS), spread(TOKENS), max(spread(TOP), 1), max(spread(TOP), 1), spread(TOP),
           rng.randrange(2))
for _ in range(20000):  # sizes of calls that fit a chip
    H, H_kv = rng.choice(HEADS)
    window(H, H_kv, spread(4096), spread(50000), spread(50000), max(spread(2000), 1), max(spread(4000), 1), spread(2000),
           rng.randrange(2))
for (H, H_kv), B, cap in itertools.product(HEADS, (0, 1, 24, 65535), (0,) + edges):
    for frame, win, sink in ((1, 1, 0), (TOP, TOP, TOP), (1, TOP, 0), (1374, 4, 1374)):
        decode(B, H, H_kv, cap, frame, win, sink)
for _ in range(20000):
    H, H_kv = rng.choice(HEADS)
    decode(spread(65535), H, H_kv, spread(TOKENS), max(spread(TOP), 1), max(spread(TOP), 1), spread(TOP))
# The join reads the sums that a cut block's slices left, so it covers the blocks that were cut and no other, of any plan:
# the others' gradients are written at once, and their part of the workspace is not.
for sinks, rest, sink_slices, slices in itertools.product((0, 1, 3), (0, 1, 5), (1, 2, 64), (1, 2, 16)):
    cut = [b for b in range(sinks + rest) if (sink_slices if b < sinks else slices) > 1]
    assert list(joined(sinks, sink_slices, slices, sinks + rest)) == cut, (sinks, rest, sink_slices, slices)
def groups_of(H, n, frame, win, off=0, sink=0, causal=1, n_k=None):
    x = ress_strides(64, 64)
    out = (C.c_int * 5)()
    lib.plan_window(C.byref(ress_window_shape(H, H, n, n_k or n + off, 64, off, frame, win, sink, causal, x, x, x, x)), out)
    return out[0]


# Two key groups from 512 blocks on are for blocks on a frame's edge, which see a frame more than the others: not without
# edges inside blocks, nor where every key is in reach (there they cost 5 to 26%).
for H, n in ((16, 4200), (8, 11008), (16, 5504), (16, 7904), (16, 8960)):
    assert groups_of(H, n, 1374, 1) == 2 and groups_of(H, n, 1374, 1, off=1374, n_k=n + 1374) == 2, (H, n)
    for frame in (768, 896, 1024, 1280, 2048):
        assert groups_of(H, n, frame, 1) == 1, (H, n, frame)
    assert groups_of(H, n, 2048, 1, off=100) == 2, (H, n)  # (edges inside blocks)
    for frame, win, causal in ((TOP, TOP, 0), (TOP, 1, 1), (n, 1, 0), (n // 2, 2, 1), (3000, 4, 1), (1374, n, 0)):
        assert groups_of(H, n, frame, win, causal=causal) == 1, (H, n, frame, win)
    assert groups_of(H, n, 1374, 1, sink=n - 1000) == 1, (H, n)
for rows in (0, 1, 2, 511, 512, 513, TOP):
    assert lib.plan_norm_bwd(rows) == min(max(rows, 1), 512)
assert seen["groups"] == {(1, False), (1, True), (2, False), (2, True), (4, False), (4, True)}, seen["groups"]
assert {2, 5, 8, 16, 32} <= seen["splits"] and {1, 2, 8, 31, 32} <= seen["decode"], seen
assert {(False, False), (True, False), (True, True)} <= seen["bwd"], seen["bwd"]
print(f"plan checks ok: {sorted(seen['splits'])} {sorted(seen['decode'])} {sorted(seen['bwd'])}", flush=True)
