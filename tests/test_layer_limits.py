"""Limits of include/ress_layer.h that lie beyond the sizes (CPU only: every call here fails validation)."""
import ctypes as C

import pytest

import layer_structs as S

INVALID = -1
P = [C.c_void_p((1 << 41) + (n << 33)) for n in range(12)]


@pytest.fixture(scope="module")
def lib():
    import paper_2609_35593_amd as r

    return r.lib


@pytest.mark.parametrize("scale", [2.0 ** 121, 3e38, 1e-46])
def test_scales_beyond_the_references(lib, scale):
    """Scales above 2^120 would leave scaled scores no room in float32; one that float32 rounds to 0 is none."""
    st = S.ress_strides(6400, 64)
    w = S.ress_window_shape(2, 2, 100, 100, 64, 0, 1, 10, 0, 1, st, st, st, st)
    g = S.ress_window_grads(st, st, st, st)
    d = S.ress_decode_shape(1, 2, 2, 100, 64, 1, 10, 0, 128, 64, 12800, 12800, st, st, 128, 64)
    big = 1 << 40
    assert lib.ress_window_attn(C.byref(w), P[0], P[1], P[2], scale, P[3], None, P[5], big, None) == INVALID
    assert lib.ress_window_attn_bwd(C.byref(w), C.byref(g), *P[:6], scale, *P[6:9], P[9], big, None) == INVALID
    assert lib.ress_window_attn_decode(C.byref(d), *P[:4], scale, P[4], P[5], big, None) == INVALID
