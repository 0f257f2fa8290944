// Windowed attention of one new token per sequence over its cache.
//
// Bound by the read of the visible keys and values (256 bytes a key and head for 4 D = 256
// flops a query head), so the products run on the vector unit: 8 lanes hold a key's or a
// value's 64 channels, a wave 8 keys at a time, and the up to R query heads that share a
// K/V head are formed from one read. The visible keys, sinks and window, are numbered
// through (j -> key), so no work goes into masked ones and nothing outside them is read.
// They are cut over `splits` workgroups of 4 or 8 waves, a run of turns of 32 keys each, the next
// turn's loads under way; every 8 lanes keep an online softmax of their own, joined in a
// fixed order in the wave, the workgroup, and for more than one split by join_kernel.
//
// 24 streams of 1 to 20,000 keys, 4 K/V heads, window 4,096: 26.6 us, 3.3 TB/s; one of 16 heads and
// 6,863 visible keys: 10.9 us. Both kernels are chains of memory round trips (lengths, first turn,
// partial results), not bandwidth.
#include "layer_internal.h"

namespace ress {
namespace {

typedef __bf16 bf16x2 __attribute__((__vector_size__(2 * sizeof(__bf16))));
typedef unsigned int u32x4 __attribute__((__vector_size__(16)));

constexpr int kMaxSplits = 32;
constexpr int kPart = 66;  // floats of a partial result: reference, sum, 64 channels

__device__ __forceinline__ float lo_f(unsigned int x) { return __builtin_bit_cast(float, x << 16); }
__device__ __forceinline__ float hi_f(unsigned int x) { return __builtin_bit_cast(float, x & 0xffff0000u); }

// c + a . b of two pairs of bf16. (By value: the bit cast of a vector's element in place
// reads its first one.)
__device__ __forceinline__ float dot2(unsigned int a, unsigned int b, float c)
{
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, a), __builtin_bit_cast(bf16x2, b), c, false);
}

// The reference of a part without keys: below every logit, and finite, so that its weight and
// that of a masked key are 0 without a test.
constexpr float kNone = -1e30f;

// Sum over the 8 lanes of a key, the same in each.
template <int CTRL>
__device__ __forceinline__ float add_from(float x)
{
    return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float sum8(float x)
{
    x = add_from<0xB1>(x);   // lanes 1 0 3 2
    x = add_from<0x4E>(x);   // lanes 2 3 0 1
    return add_from<0x141>(x);  // mirrored in 8 lanes
}

// What sequence b's token sees, numbered through: j < sk is key j, else key j - sk + lo.
struct Visible {
    int sk, lo, n;
};
__device__ __forceinline__ Visible visible(const DecodeParams &p, int b)
{
    const int len = min(max(p.lens[b], 0), p.capacity);
    Visible v = {0, 0, 0};
    if (len == 0) return v;
    v.lo = max((p.frames(len - 1) - p.window + 1) * p.frame, 0);
    v.sk = min(p.n_sink, v.lo);
    v.n = v.sk + len - v.lo;
    return v;
}

// Waves of a workgroup: one head's lanes leave registers for twice the waves of four heads' (us
// with 4 / 8: 16 heads of 6,870 keys, one a K/V head, 10.5 / 9.3; 24 streams, four a K/V head, 27 / 34).
constexpr int waves_of(int heads) { return heads == 1 ? 8 : 4; }

template <int R>
__global__ void __launch_bounds__(64 * waves_of(R)) decode_kernel(const DecodeParams p)
{
    constexpr int kWaves = waves_of(R);
    __shared__ float lds[kWaves][R][kPart];
    const int split = blockIdx.x, b = blockIdx.z;
    const int tiles = (p.group + R - 1) / R;
    const int hk = blockIdx.y / tiles, h0 = hk * p.group + (blockIdx.y % tiles) * R;
    const int heads = min(R, (hk + 1) * p.group - h0);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, ch = lane & 7, oct = lane >> 3;
    const Visible vis = visible(p, b);

    // Whole turns of 32 keys, evenly over the splits' waves.
    const int turns = (vis.n + 31) / 32, waves = p.splits * kWaves, each = (turns + waves - 1) / waves;
    const int first = (split * kWaves + wave) * each, last = min(first + each, turns);

    u32x4 q[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int h = h0 + min(r, heads - 1);
        q[r] = *reinterpret_cast<const u32x4 *>(p.q + b * p.q_batch + h * p.q_head + ch * 8);
    }
    const uint16_t *kb = p.k + b * p.k_batch + hk * p.ks.head + ch * 8;
    const uint16_t *vb = p.v + b * p.v_batch + hk * p.vs.head + ch * 8;

    float m[R], l[R], acc[R][8];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        m[r] = kNone;
        l[r] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[r][e] = 0.f;
    }
    u32x4 kx[4], vx[4], kn[4], vn[4];
    auto fetch = [&](int t) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // (Past the end: the last key again, its weight 0 and its value left out.)
            const int j = min(t * 32 + i * 8 + oct, vis.n - 1);
            const int64_t key = j < vis.sk ? j : j - vis.sk + vis.lo;
            kn[i] = *reinterpret_cast<const u32x4 *>(kb + key * p.ks.token);
            vn[i] = *reinterpret_cast<const u32x4 *>(vb + key * p.vs.token);
        }
    };
    if (first < last) fetch(first);
    for (int t = first; t < last; ++t) {
#pragma unroll
        for (int i = 0; i < 4; ++i) kx[i] = kn[i], vx[i] = vn[i];
        if (t + 1 < last) fetch(t + 1);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float s[4], top = m[r];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float d = 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) d = dot2(kx[i][e], q[r][e], d);
                d = sum8(d) * p.scale_log2;
                s[i] = t * 32 + i * 8 + oct < vis.n ? d : -INFINITY;
                top = fmaxf(top, s[i]);
            }
            const float a = __builtin_amdgcn_exp2f(m[r] - top);
            m[r] = top;
            l[r] *= a;
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[r][e] *= a;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float w = __builtin_amdgcn_exp2f(s[i] - top);
                l[r] += w;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    acc[r][2 * e] = fmaf(w, lo_f(vx[i][e]), acc[r][2 * e]);
                    acc[r][2 * e + 1] = fmaf(w, hi_f(vx[i][e]), acc[r][2 * e + 1]);
                }
            }
        }
    }
    // The wave's 8 groups of lanes, then the workgroup's waves.
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float top = m[r];
#pragma unroll
        for (int o = 8; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
        const float a = __builtin_amdgcn_exp2f(m[r] - top);
        l[r] *= a;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[r][e] *= a;
#pragma unroll
        for (int o = 8; o < 64; o <<= 1) {
            l[r] += __shfl_xor(l[r], o);
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[r][e] += __shfl_xor(acc[r][e], o);
        }
        if (oct == 0) {
            float *d = lds[wave][r];
            if (ch == 0) d[0] = top, d[1] = l[r];
#pragma unroll
            for (int e = 0; e < 8; ++e) d[2 + ch * 8 + e] = acc[r][e];
        }
    }
    __syncthreads();
    for (int r = wave; r < heads; r += kWaves) {
        float top = kNone, sum = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, lds[w][r][0]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float a = __builtin_amdgcn_exp2f(lds[w][r][0] - top);
            sum = fmaf(lds[w][r][1], a, sum);
            o = fmaf(lds[w][r][2 + lane], a, o);
        }
        const int h = h0 + r;
        if (p.splits == 1) {
            const float y = sum == 0.f ? 0.f : o / sum;
            p.o[b * p.o_batch + h * p.o_head + lane] = __builtin_bit_cast(uint16_t, (__bf16)y);
        } else {
            float *d = p.part + (((int64_t)b * p.H + h) * p.splits + split) * kPart;
            if (lane == 0) d[0] = top, d[1] = sum;
            d[2 + lane] = o;
        }
    }
}

// A wave a query head, a channel a lane: its at most 32 splits in order, their weights one a
// lane first.
__global__ void __launch_bounds__(256) join_kernel(const DecodeParams p)
{
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= (int64_t)p.B * p.H) return;
    const int lane = threadIdx.x & 63;
    const float *d = p.part + row * p.splits * kPart;
    // (All parts are on their way with their references: one round trip.)
    float m = kNone, sum = 0.f, o = 0.f, x[kMaxSplits];
    if (lane < p.splits) m = d[lane * kPart], sum = d[lane * kPart + 1];
#pragma unroll
    for (int s0 = 0; s0 < kMaxSplits; s0 += 4)
        if (s0 < p.splits)
#pragma unroll
            for (int s = s0; s < s0 + 4; ++s) x[s] = d[min(s, p.splits - 1) * kPart + 2 + lane];
    float top = m;
#pragma unroll
    for (int e = 1; e < 64; e <<= 1) top = fmaxf(top, __shfl_xor(top, e));
    const float w = __builtin_amdgcn_exp2f(m - top);
    sum *= w;
#pragma unroll
    for (int e = 1; e < 64; e <<= 1) sum += __shfl_xor(sum, e);
    auto weight = [&](int s) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), s)); };
#pragma unroll
    for (int s = 0; s < kMaxSplits; ++s)
        if (s < p.splits) o = fmaf(weight(s), x[s], o);
    const int64_t b = row / p.H, h = row - b * p.H;
    p.o[b * p.o_batch + h * p.o_head + lane] = __builtin_bit_cast(uint16_t, (__bf16)(sum == 0.f ? 0.f : o / sum));
}

template <int R>
hipError_t go(const DecodeParams &p, hipStream_t s)
{
    const dim3 grid((unsigned)p.splits, (unsigned)(p.H_kv * ((p.group + R - 1) / R)), (unsigned)p.B);
    hipLaunchKernelGGL(decode_kernel<R>, grid, dim3(64 * waves_of(R)), 0, s, p);
    if (hipError_t e = hipGetLastError()) return e;
    if (p.splits > 1) {
        hipLaunchKernelGGL(join_kernel, dim3((unsigned)(((int64_t)p.B * p.H + 3) / 4)), dim3(256), 0, s, p);
        return hipGetLastError();
    }
    return hipSuccess;
}

}  // namespace

// Workgroups per sequence and head: enough for 4 a CU, but none with less than 256 keys, and one
// up to 512 (us with at least 256 / 512 / 1,024 keys, the join counted: 4 heads of 900 keys for 16
// 10.1 / 12.2 / 13.5, of 8,000 10.6 / 12.6 / 17.2; 16 heads of 6,870 9.6 / 9.3 / 10.8; 8 streams
// of 4 heads of 4,000 19.6 / 18.1 / 20.9; 32 heads of 300 7.4 / 5.1 / 5.2; 768 heads of 2,000 in
// halves 81, whole 74).
int decode_splits(const ress_decode_shape *s)
{
    if (s->B == 0 || s->H == 0 || s->capacity == 0) return 1;
    const int64_t seen = window_tokens(s->frame, s->window) + s->n_sink;
    const int64_t keys = seen < s->capacity ? seen : s->capacity;  // at least 1
    const int64_t heads = (int64_t)s->B * s->H_kv * ((s->H / s->H_kv + 3) / 4);
    const int64_t want = 1024 / heads, most = keys <= 512 ? 1 : (keys + 255) / 256;
    int64_t n = want < most ? want : most;
    n = n < 1 ? 1 : n > kMaxSplits ? kMaxSplits : n;
    // No more than give every wave the same turns (24 streams of up to 4,160 keys: 10 splits of 3.25
    // turns a wave 29.8 us, 9 of 3.6 27.4: both take 4).
    const int64_t turns = (keys + 31) / 32, waves = waves_of(s->H == s->H_kv ? 1 : 4);
    const int64_t each = (turns + n * waves - 1) / (n * waves);
    return (int)((turns + each * waves - 1) / (each * waves));
}

hipError_t launch_decode(const DecodeParams &p, hipStream_t s)
{
    return p.group == 1 ? go<1>(p, s) : p.group == 2 ? go<2>(p, s) : go<4>(p, s);
}

}  // namespace ress
