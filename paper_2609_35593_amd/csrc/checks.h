// What the C ABI layers check of pointers and strides, on the host.
#pragma once

#include "layer_internal.h"

namespace ress {

constexpr int64_t kMaxTokenStride = 1 << 22;      // 63 rows of it in bytes fit 31 bits
constexpr int64_t kMaxStride = (int64_t)1 << 46;  // times 2^16 rows stays in 63 bits

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
inline bool aligned(const void *ptr, size_t to) { return ((uintptr_t)ptr & (to - 1)) == 0; }
inline bool dtype_ok(int t) { return t == RESS_DTYPE_BF16 || t == RESS_DTYPE_F32; }
inline size_t dtype_size(int t) { return t == RESS_DTYPE_F32 ? 4 : 2; }
inline bool same(const ress_strides &a, const ress_strides &b) { return a.head == b.head && a.token == b.token; }

// [n][m] rows of `width` elements, `outer` and `inner` apart, that do not overlap: one
// dimension lies whole between two steps of the other.
inline bool disjoint(int64_t n, int64_t outer, int64_t m, int64_t inner, int64_t width)
{
    if (n <= 1 && m <= 1) return true;
    if (m <= 1) return outer >= width;
    if (n <= 1) return inner >= width;
    return (inner >= width && outer >= (m - 1) * inner + width) || (outer >= width && inner >= (n - 1) * outer + width);
}

inline bool strides_ok(const ress_strides &s, int64_t multiple)
{
    return s.head >= 0 && s.head <= kMaxStride && s.token >= 0 && s.token <= kMaxTokenStride && s.head % multiple == 0 &&
           s.token % multiple == 0;
}

// Scales up to 2^120, which leaves the references' unit and most scores room in float32.
inline bool scale_ok(float scale) { return scale > 0.f && scale <= 0x1p120f; }

inline int check_heads(int H, int H_kv)
{
    if (H < 0 || H_kv < 0) return RESS_E_INVALID_ARG;
    if (H > RESS_MAX_HEADS) return RESS_E_UNSUPPORTED;
    if (H_kv == 0 ? H != 0 : H % H_kv != 0) return RESS_E_INVALID_ARG;
    if (H == 0 && H_kv != 0) return RESS_E_INVALID_ARG;
    return RESS_OK;
}

// The sizes and the rotation of a ress_rope_shape; `turned`: channels that turn.
inline int check_rope(const ress_rope_shape &s, int &turned)
{
    if (s.H < 0 || s.H_kv < 0 || s.N < 0 || s.D < 2 || s.D % 2 || s.n_axes < 1 || !dtype_ok(s.dtype) ||
        s.layout < RESS_ROPE_SPLIT || s.layout > RESS_ROPE_SECTIONS || !(s.base >= 1.0) || !isfinite(s.base))
        return RESS_E_INVALID_ARG;
    if (s.H > RESS_MAX_HEADS || s.H_kv > RESS_MAX_HEADS || s.N > RESS_MAX_TOKENS || s.D > RESS_MAX_ROPE_D ||
        s.n_axes > RESS_MAX_ROPE_AXES)
        return RESS_E_UNSUPPORTED;
    turned = 0;
    for (int a = 0; a < s.n_axes; ++a) {
        if (s.dims[a] < 0 || s.dims[a] % 2 || s.dims[a] > s.D) return RESS_E_INVALID_ARG;
        turned += s.dims[a];
    }
    return turned > s.D ? RESS_E_INVALID_ARG : RESS_OK;
}

// Whether chunks of `per` channels hold whole runs of one side of the pairs (or whole pairs,
// interleaved), and a wave a token's.
inline bool rope_chunks(const ress_rope_shape &s, int per, int turned)
{
    if (s.D % per || s.D / per > kMaxChunks) return false;
    if (s.layout == RESS_ROPE_SECTIONS) return turned % (2 * per) == 0;
    if (s.layout == RESS_ROPE_INTERLEAVED) return turned % per == 0;
    for (int a = 0; a < s.n_axes; ++a)
        if (s.dims[a] % (2 * per)) return false;
    return true;
}

// The pairs of a checked shape: axis, turns a position, channels (copied channels pair up behind
// them); and with chunks of p.chunk channels their first pairs and others. Sizes and flags too.
inline void rope_tables(const ress_rope_shape &s, int turned, RopeParams &p)
{
    const double two_pi = 6.283185307179586476925;
    int n = 0, at = 0;
    for (int a = 0; a < s.n_axes; ++a) {
        for (int i = 0; i < s.dims[a] / 2; ++i, ++n) {
            p.axis[n] = (uint8_t)a;
            if (s.layout == RESS_ROPE_SECTIONS) {
                p.turns[n] = pow(s.base, -2.0 * n / turned) / two_pi;
                p.ca[n] = (uint8_t)n;
                p.cb[n] = (uint8_t)(n + turned / 2);
            } else {
                const bool inter = s.layout == RESS_ROPE_INTERLEAVED;
                p.turns[n] = pow(s.base, -2.0 * i / s.dims[a]) / two_pi;
                p.ca[n] = (uint8_t)(at + (inter ? 2 * i : i));
                p.cb[n] = (uint8_t)(at + (inter ? 2 * i + 1 : i + s.dims[a] / 2));
            }
        }
        at += s.dims[a];
    }
    for (int i = 0; n < s.D / 2; ++i, ++n) {
        p.turns[n] = -1.0;
        p.ca[n] = (uint8_t)(turned + 2 * i);
        p.cb[n] = (uint8_t)(turned + 2 * i + 1);
    }
    for (int c = 0; p.chunk && c < s.D / p.chunk; ++c) p.other[c] = (uint8_t)c;
    for (int i = 0; p.chunk && i < turned / 2; ++i) {
        const int a = p.ca[i] / p.chunk, b = p.cb[i] / p.chunk;
        if (p.ca[i] % p.chunk == 0) p.pair_of[a] = (uint8_t)i, p.other[a] = (uint8_t)b;
        if (p.cb[i] % p.chunk == 0) p.pair_of[b] = (uint8_t)i, p.other[b] = (uint8_t)a;
    }
    p.H = s.H;
    p.H_all = s.H + s.H_kv;
    p.N = s.N;
    p.n_axes = s.n_axes;
    p.n_pairs = s.D / 2;
    p.D = s.D;
    p.turned = turned;
    p.f32 = s.dtype == RESS_DTYPE_F32;
    p.inverse = s.inverse != 0;
    p.interleaved = s.layout == RESS_ROPE_INTERLEAVED;
}

}  // namespace ress
