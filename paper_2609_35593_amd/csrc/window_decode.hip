// Windowed attention of one new token per sequence over its cache.
//
// Bound by the read of the visible keys and values: 256 bytes a key and K/V head. The visible keys,
// sinks and window, are numbered through (j -> key), so no work goes into masked ones and nothing
// outside them is read. They are cut over `splits` workgroups and their waves, a run of turns each,
// the next turn's loads under way; every wave keeps an online softmax of its own, joined in a
// fixed order in the workgroup, and for more than one split by join_kernel.
//
//   decode_kernel       one head a K/V head: products on the vector unit, 8 lanes a key's or
//                       a value's 64 channels, a wave 8 keys at a time
//   decode_tile_kernel  several heads, formed from one read: products on the matrix unit, the heads
//                       its columns. (On the vector unit, four heads from one read: 24 streams of up
//                       to 4,160 keys, 16 heads for 4, 28.0 us, here 23.3; 3 of 12,400, 32 heads for 4,
//                       26.5 / 13.7; 64 of 8,000, 32 for 8, 231 / 190; two heads of 16 x 3,000 15.3 / 14.8;
//                       one head there: 16 of 6,863 keys 9.1, here 11.2.)
//
// 24 streams of 1 to 20,000 keys, 4 K/V heads, window 4,096: 25.1 us, 3.6 TB/s (64 of 8,000: 190, 5.5); one of 16 heads and
// 6,863 visible keys: 10.9 us. Both kernels are chains of memory round trips (lengths, first turn,
// partial results) as much as bandwidth.
#include <float.h>

#include "tiles.h"

namespace ress {
namespace {

using namespace tiles;

typedef unsigned int u32x4 __attribute__((__vector_size__(16)));

constexpr int kPart = 66;  // floats of a partial result: reference, sum, 64 channels

__device__ __forceinline__ float lo_f(unsigned int x) { return __builtin_bit_cast(float, x << 16); }
__device__ __forceinline__ float hi_f(unsigned int x) { return __builtin_bit_cast(float, x & 0xffff0000u); }

// c + a . b of two pairs of bf16. (By value: the bit cast of a vector's element in place
// reads its first one.)
__device__ __forceinline__ float dot2(unsigned int a, unsigned int b, float c)
{
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, a), __builtin_bit_cast(bf16x2, b), c, false);
}

// References are scores before their scale: what a scaled one's rounding takes, all of a weight from 2^31 on, is
// not taken here. A part without keys has one at or below every score, and finite: its sums are 0 without a
// test, whatever their weight, and masked keys (-inf) have none.
constexpr float kNone = -FLT_MAX;

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

// A head's channel `lane` of a workgroup: the output, or its part of it.
__device__ __forceinline__ void finish(const DecodeParams &p, int b, int h, int split, int lane, float top, float sum, float o)
{
    if (p.splits == 1) {
        const float y = sum == 0.f ? 0.f : o / sum;
        p.o[b * p.o_batch + h * p.o_head + lane] = __builtin_bit_cast(uint16_t, (__bf16)y);
    } else {
        float *d = p.part + (((int64_t)b * p.H + h) * p.splits + split) * kPart;
        if (lane == 0) d[0] = top, d[1] = sum;
        d[2 + lane] = o;
    }
}

__global__ void __launch_bounds__(64 * kHeadWaves) decode_kernel(const DecodeParams p)
{
    __shared__ float lds[kHeadWaves][kPart];
    const int split = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, ch = lane & 7, oct = lane >> 3;
    const Visible vis = visible(p, b);

    // Whole turns of 32 keys, evenly over the splits' waves.
    const int turns = (vis.n + 31) / 32, waves = p.splits * kHeadWaves, each = (turns + waves - 1) / waves;
    const int first = (split * kHeadWaves + wave) * each, last = min(first + each, turns);

    const u32x4 q = *reinterpret_cast<const u32x4 *>(p.q + b * p.q_batch + h * p.q_head + ch * 8);
    const uint16_t *kb = p.k + b * p.k_batch + h * p.ks.head + ch * 8;
    const uint16_t *vb = p.v + b * p.v_batch + h * p.vs.head + ch * 8;

    const float c = p.scale_log2;
    float m = kNone, l = 0.f, acc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
    u32x4 kx[4], vx[4], kn[4], vn[4];
    auto fetch = [&](int t) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // (Past the end: the last key again, its weight 0.)
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
        float s[4], top = m;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float d = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) d = dot2(kx[i][e], q[e], d);
            d = sum8(d);
            s[i] = t * 32 + i * 8 + oct < vis.n ? d : -INFINITY;
            top = fmaxf(top, s[i]);
        }
        const float a = __builtin_amdgcn_exp2f((m - top) * c);
        m = top;
        l *= a;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] *= a;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float w = __builtin_amdgcn_exp2f((s[i] - top) * c);
            l += w;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                acc[2 * e] = fmaf(w, lo_f(vx[i][e]), acc[2 * e]);
                acc[2 * e + 1] = fmaf(w, hi_f(vx[i][e]), acc[2 * e + 1]);
            }
        }
    }
    // The wave's 8 groups of lanes, then the workgroup's waves.
    float top = m;
#pragma unroll
    for (int o = 8; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float a = __builtin_amdgcn_exp2f((m - top) * c);
    l *= a;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] *= a;
#pragma unroll
    for (int o = 8; o < 64; o <<= 1) {
        l += __shfl_xor(l, o);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += __shfl_xor(acc[e], o);
    }
    if (oct == 0) {
        float *d = lds[wave];
        if (ch == 0) d[0] = top, d[1] = l;
#pragma unroll
        for (int e = 0; e < 8; ++e) d[2 + ch * 8 + e] = acc[e];
    }
    __syncthreads();
    if (wave > 0) return;
    float sum = 0.f, o = 0.f;
    top = kNone;
#pragma unroll
    for (int w = 0; w < kHeadWaves; ++w) top = fmaxf(top, lds[w][0]);
#pragma unroll
    for (int w = 0; w < kHeadWaves; ++w) {
        const float x = __builtin_amdgcn_exp2f((lds[w][0] - top) * c);
        sum = fmaf(lds[w][1], x, sum);
        o = fmaf(lds[w][2 + lane], x, o);
    }
    finish(p, b, h, split, lane, top, sum, o);
}

// Up to 32 heads of a K/V head a workgroup, the columns of the products (tiles.h). A wave's turn is 64 of the numbered keys, their rows of K straight in
// registers as the product's operand, those of V through LDS slots of the wave's own, so that no
// wave waits for another before the join. A weight enters its product as two bf16 numbers, itself
// rounded and what that leaves (2^-16 of it at most is lost), so that the outputs are those of
// float32 weights, as in decode_kernel.
__global__ void __launch_bounds__(64 * kTileWaves, 2) decode_tile_kernel(const DecodeParams p)
{
    constexpr int kWaves = kTileWaves, kStep = 33;  // floats between a part's rows in LDS: one of 32 heads each, no conflicts
    __shared__ __attribute__((aligned(1024))) unsigned char v_0[kWaves * kTileBytes], v_1[kWaves * kTileBytes];
    static_assert(2 * kPart * kStep * 4 <= (int)sizeof v_0, "two waves' parts fit a slot array");
    const int split = blockIdx.x, b = blockIdx.z;
    const int tiles = (p.group + 31) / 32;
    const int hk = blockIdx.y / tiles, h0 = hk * p.group + (blockIdx.y % tiles) * 32;
    const int heads = min(32, (hk + 1) * p.group - h0);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hh = lane >> 5, ql = lane & 31;
    const Visible vis = visible(p, b);
    const int turns = (vis.n + 63) / 64, waves = p.splits * kWaves, each = (turns + waves - 1) / waves;
    const int first = (split * kWaves + wave) * each, last = min(first + each, turns);

    bf16x8 qf[4];
    {
        const uint16_t *q = p.q + b * p.q_batch + (h0 + min(ql, heads - 1)) * p.q_head + hh * 8;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) qf[kk] = *reinterpret_cast<const bf16x8 *>(q + kk * 16);
    }
    const uint16_t *kb = p.k + b * p.k_batch + hk * p.ks.head + hh * 8;
    const uint16_t *vb = p.v + b * p.v_batch + hk * p.vs.head;
    // (Past the end: the last key again, its weight 0.)
    auto key_of = [&](int j) __attribute__((always_inline)) -> int64_t {
        j = min(j, vis.n - 1);
        return j < vis.sk ? j : j - vis.sk + vis.lo;
    };
    auto fetch = [&](int t, bf16x8 (&k)[2][4], unsigned char *slot) __attribute__((always_inline)) {
        if (t >= last) return;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint16_t *row = kb + key_of(t * 64 + u * 32 + ql) * p.ks.token;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) k[u][kk] = *reinterpret_cast<const bf16x8 *>(row + kk * 16);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int r = u * 8 + (lane >> 3);
            const uint16_t *row = vb + key_of(t * 64 + r) * p.vs.token + (((lane & 7) ^ swz(r)) << 3);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)row, (lds_void *)(slot + u * 1024),
                                             16, 0, 0);
        }
    };
    const Reader rd(lane);
    const float c = p.scale_log2;
    float m = kNone, sum = 0.f;
    f32x16 acc[2];
#pragma unroll
    for (int dh = 0; dh < 2; ++dh)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[dh][v] = 0.f;
    int t = first;
    auto step = [&](const bf16x8 (&k)[2][4], const unsigned char *vt, bf16x8 (&kn)[2][4], unsigned char *vn)
                    __attribute__((always_inline)) -> bool {
        fetch(t + 1, kn, vn);
        f32x16 s[2];
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int v = 0; v < 16; ++v) s[u][v] = 0.f;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) s[u] = mfma(k[u][kk], qf[kk], s[u]);
            if ((t + 1) * 64 > vis.n)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    if (t * 64 + u * 32 + (v >> 2) * 8 + hh * 4 + (v & 3) >= vis.n) s[u][v] = -INFINITY;
#pragma unroll
            for (int v = 0; v < 16; ++v) top = fmaxf(top, s[u][v]);
        }
        top = fmaxf(fmaxf(top, __shfl_xor(top, 32)), m);
        if (__any(top > m)) {
            const float a = __builtin_amdgcn_exp2f((m - top) * c);
            sum *= a;
#pragma unroll
            for (int dh = 0; dh < 2; ++dh)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[dh][v] *= a;
            m = top;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            bf16x8 pb[2], rest[2];
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                s[u][v] = __builtin_amdgcn_exp2f((s[u][v] - m) * c);
                sum += s[u][v];
            }
            pack(s[u], pb);
#pragma unroll
            for (int v = 0; v < 16; ++v) s[u][v] -= (float)pb[v >> 3][v & 7];
            pack(s[u], rest);
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int dh = 0; dh < 2; ++dh) {
                    const bf16x8 vc = rd.cols(vt, u, e, dh);
                    acc[dh] = mfma(vc, pb[e], acc[dh]);
                    acc[dh] = mfma(vc, rest[e], acc[dh]);
                }
        }
        __builtin_amdgcn_s_waitcnt(0x0070);  // the next turn's loads, and this one's reads of its slot
        asm volatile("" ::: "memory");
        return ++t < last;
    };
    if (t < last) {
        unsigned char *const a = v_0 + wave * kTileBytes, *const z = v_1 + wave * kTileBytes;
        bf16x8 ka[2][4], kz[2][4];
        fetch(t, ka, a);
        __builtin_amdgcn_s_waitcnt(0x0070);
        asm volatile("" ::: "memory");
        while (step(ka, a, kz, z) && step(kz, z, ka, a)) {
        }
    }
    sum += __shfl_xor(sum, 32);
    __syncthreads();  // (slots of other waves become parts)
    auto part = [&](int w) __attribute__((always_inline)) -> float * {
        return reinterpret_cast<float *>(w < 2 ? v_0 : v_1) + (w & 1) * kPart * kStep;
    };
    {
        float *d = part(wave) + ql;
        if (hh == 0) d[0] = m, d[kStep] = sum;
#pragma unroll
        for (int dh = 0; dh < 2; ++dh)
#pragma unroll
            for (int v = 0; v < 16; ++v) d[(2 + dh * 32 + (v >> 2) * 8 + hh * 4 + (v & 3)) * kStep] = acc[dh][v];
    }
    __syncthreads();
    for (int r = wave; r < heads; r += kWaves) {
        float top = kNone, l = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, part(w)[r]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float a = __builtin_amdgcn_exp2f((part(w)[r] - top) * c);
            l = fmaf(part(w)[kStep + r], a, l);
            o = fmaf(part(w)[(2 + lane) * kStep + r], a, o);
        }
        finish(p, b, h0 + r, split, lane, top, l, o);
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
    const float w = __builtin_amdgcn_exp2f((m - top) * p.scale_log2);
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

}  // namespace

hipError_t launch_decode(const DecodeParams &p, hipStream_t s)
{
    const bool one = p.group == 1;
    const dim3 grid((unsigned)p.splits, (unsigned)(p.H_kv * ((p.group + 31) / 32)), (unsigned)p.B);
    if (one)
        hipLaunchKernelGGL(decode_kernel, grid, dim3(64 * kHeadWaves), 0, s, p);
    else
        hipLaunchKernelGGL(decode_tile_kernel, grid, dim3(64 * kTileWaves), 0, s, p);
    if (hipError_t e = hipGetLastError()) return e;
    if (p.splits > 1) {
        hipLaunchKernelGGL(join_kernel, dim3((unsigned)(((int64_t)p.B * p.H + 3) / 4)), dim3(256), 0, s, p);
        return hipGetLastError();
    }
    return hipSuccess;
}

}  // namespace ress
