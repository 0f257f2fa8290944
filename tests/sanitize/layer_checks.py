"""Host code of ress_layer.h's C ABI under AddressSanitizer and UndefinedBehaviorSanitizer, in a child process (no GPU,
no torch): shapes at and beyond every limit; what passes validation ends in a launcher that only fails (RESS_E_HIP).
Usage: python layer_checks.py <library>"""
import ctypes as C
import itertools
import sys

from layer_structs import (ress_decode_shape, ress_norm_shape, ress_rope_shape, ress_strides, ress_window_grads,
                           ress_window_shape)

lib = C.CDLL(sys.argv[1])
vp, f32, sz = C.c_void_p, C.c_float, C.c_size_t
lib.ress_layer_norm.argtypes = [vp] * 8
lib.ress_layer_norm_bwd.argtypes = [vp] * 10 + [sz, vp]
lib.ress_rope.argtypes = [vp] * 7
lib.ress_window_attn.argtypes = [vp] * 4 + [f32, vp, vp, vp, sz, vp]
lib.ress_window_attn_bwd.argtypes = [vp] * 8 + [f32] + [vp] * 4 + [sz, vp]
lib.ress_window_attn_decode.argtypes = [vp] * 5 + [f32, vp, vp, sz, vp]
P = [(1 << 41) + (n << 33) for n in range(12)]
BIG = 1 << 60
edge = (-(1 << 31), -1, 0, 1, 2, (1 << 24), (1 << 24) + 1, (1 << 31) - 1)
checks = 0


def legal(st):
    global checks
    checks += 1
    assert st in (0, -1, -2, -3, -4), st
    return st


for rows, width, stride, eps in itertools.product((-1, 0, 1, (1 << 31) - 1, 1 << 31, 1 << 62), (0, 1, 64, 16384, 16385),
                                                  (-1, 0, 64, 16384, 1 << 62), (0.0, 1e-5, 1e300, float("nan"))):
    s = ress_norm_shape(rows, width, 1, 0, stride, stride, eps)
    n = sz(0)
    legal(lib.ress_layer_norm_bwd_workspace_size(C.byref(s), C.byref(n)))
    legal(lib.ress_layer_norm(C.byref(s), *P[:6], None))
    legal(lib.ress_layer_norm_bwd(C.byref(s), *P[:9], BIG, None))
reached = 0
for D, axes, dims, layout, dtype in itertools.product((2, 6, 64, 80, 256), (1, 2, 4), ((64, 0, 0, 0), (32, 32, 0, 0), (2, 2, 2, 0),
                                                      (128, 64, 32, 32), ((1 << 31) - 2,) * 4, (10, 14, 8, 4)), (0, 1, 2), (0, 1)):
    for st in ((0, 0), (D * 100, D), (D, D * 4), (1 << 46, 1 << 22), (1 << 62, 1 << 62), (-8, 8), (7, 3)):
        x = ress_strides(*st)
        s = ress_rope_shape(4, 2, 100, D, axes, (C.c_int * 4)(*dims), layout, 0, dtype, 100.0, x, x, x, x)
        reached += legal(lib.ress_rope(C.byref(s), P[0], P[1], P[2], P[3], P[4], None)) == -4
assert reached > 50, reached
reached = 0
for n_q, n_k, off, frame, window, sink in itertools.product((0, 1, 1 << 24), (0, 5, 1 << 24), (0, 1 << 24), *([(1, (1 << 31) - 1)] * 2),
                                                            (0, (1 << 31) - 1)):
    for causal in (0, 1):
        x = ress_strides(64 << 24, 64)
        s = ress_window_shape(8, 4, n_q, n_k, 64, off, frame, window, sink, causal, x, x, x, x)
        n = sz(0)
        legal(lib.ress_window_attn_workspace_size(C.byref(s), C.byref(n)))
        reached += legal(lib.ress_window_attn(C.byref(s), P[0], P[1], P[2], 0.125, P[3], P[4], P[5], BIG, None)) == -4
        legal(lib.ress_window_attn_bwd_workspace_size(C.byref(s), C.byref(n)))
        g = ress_window_grads(x, x, x, x)
        reached += legal(lib.ress_window_attn_bwd(C.byref(s), C.byref(g), *P[:6], 0.125, *P[6:9], P[9], BIG, None)) == -4
assert reached > 50, reached
for field, value in itertools.product(("H", "H_kv", "n_q", "n_k", "D", "q_offset", "frame", "window", "n_sink"), edge):
    x = ress_strides(64 << 24, 64)
    s = ress_window_shape(8, 4, 100, 100, 64, 0, 1, 10, 0, 1, x, x, x, x)
    setattr(s, field, value)
    legal(lib.ress_window_attn(C.byref(s), P[0], P[1], P[2], 0.125, P[3], P[4], P[5], BIG, None))
    g = ress_window_grads(x, x, x, x)
    legal(lib.ress_window_attn_bwd(C.byref(s), C.byref(g), *P[:6], 0.125, *P[6:9], P[9], BIG, None))
for field, value in itertools.product(("B", "H", "H_kv", "capacity", "D", "frame", "window", "n_sink"), edge + (65535, 65536)):
    x = ress_strides(64 << 24, 64)
    s = ress_decode_shape(3, 8, 4, 1000, 64, 1, 10, 0, 512, 64, 1 << 40, 1 << 40, x, x, 512, 64)
    setattr(s, field, value)
    n = sz(0)
    legal(lib.ress_window_attn_decode_workspace_size(C.byref(s), C.byref(n)))
    legal(lib.ress_window_attn_decode(C.byref(s), *P[:4], 0.125, P[4], P[5], BIG, None))
# Divisions by a product and a shift: the ends of every quotient's run, where one off by the least would show.
top = (1 << 31) - 1
for d in (1, 2, 3, 5, 7, 63, 64, 65, 641, 1374, 5496, 65535, (1 << 20) + 1, (1 << 26) - 1, 1 << 26, (1 << 30) + 1, top):
    for q in (0, 1, 2, 3, 1000, 12345, top // d // 2, top // d - 1, top // d):
        for n in (q * d - 1, q * d, q * d + 1, q * d + d - 1, top):
            if 0 <= n <= top:
                assert lib.divided(n, d) == n // d, (n, d)
print(f"layer checks ok: {checks}", flush=True)
