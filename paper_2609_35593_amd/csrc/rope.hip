// Rotary positions with several axes.
//
// Memory bound: every element of Q and K is read and written once. A thread owns one
// token's group of channel pairs and walks over the heads, so that the angles (float64,
// reduced to a turn's fraction before the sine) are formed once per token and pair and
// stay in registers. Where pairs come in whole 16-byte chunks (chunk ca against chunk cb,
// or pairs inside a chunk), a group is two chunks of 8 channels; otherwise it is a pair.
#include "layer_internal.h"

namespace ress {
namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 4;  // heads of a thread in flight

__device__ __forceinline__ float from_bf16(uint16_t b) { return __builtin_bit_cast(float, (uint32_t)b << 16); }

template <typename T>
struct alignas(16) Chunk {  // 8 channels
    T e[8];
};

__device__ __forceinline__ float get(float x) { return x; }
__device__ __forceinline__ float get(uint16_t x) { return from_bf16(x); }
__device__ __forceinline__ void put(float &d, float x) { d = x; }
__device__ __forceinline__ void put(uint16_t &d, float x) { d = __builtin_bit_cast(uint16_t, (__bf16)x); }

// cos and sin of `turns` turns a position (the sine negated for the inverse). At most
// 2^31 / 2 pi turns, known to 2^-23 of one at worst, to 2^-30 for positions below 2^24.
__device__ __forceinline__ void angle(const RopeParams &p, const int32_t *pos, int pair, float &c, float &s)
{
    const double t = (double)pos[p.axis[pair]] * p.turns[pair];
    sincospif((float)(2.0 * (t - rint(t))), &s, &c);
    if (p.inverse) s = -s;
}

// The turned pair, the same roundings in every form of the kernel.
__device__ __forceinline__ float turn_a(float a, float b, float c, float s) { return fmaf(a, c, -(b * s)); }
__device__ __forceinline__ float turn_b(float a, float b, float c, float s) { return fmaf(a, s, b * c); }

// Head h of q and k together, its input and output rows of token t.
template <typename T>
__device__ __forceinline__ void rows_of(const RopeParams &p, int h, int64_t t, const T *&in, T *&out)
{
    if (h < p.H) {
        in = static_cast<const T *>(p.q_in) + h * p.qi.head + t * p.qi.token;
        out = static_cast<T *>(p.q_out) + h * p.qo.head + t * p.qo.token;
    } else {
        in = static_cast<const T *>(p.k_in) + (h - p.H) * p.ki.head + t * p.ki.token;
        out = static_cast<T *>(p.k_out) + (h - p.H) * p.ko.head + t * p.ko.token;
    }
}

// A thread: token i / units, chunks ca and cb of unit i % units; heads h0 .. h0 + heads - 1.
template <typename T, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads) rope_chunk_kernel(const RopeParams p, int units, int heads)
{
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t t = i / units;
    const int u = (int)(i - t * units);
    if (t >= p.N) return;
    const int32_t *pos = p.pos + t * p.n_axes;
    const int ca = p.ca[8 * u], cb = INTERLEAVED ? p.ca[8 * u + 4] : p.cb[8 * u];
    const bool copy_a = p.turns[8 * u] < 0.0, copy_b = p.turns[8 * u + 4] < 0.0;
    float c[8], s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        c[e] = 1.f, s[e] = 0.f;
        if (p.turns[8 * u + e] >= 0.0) angle(p, pos, 8 * u + e, c[e], s[e]);
    }
    const int h0 = blockIdx.y * heads, h1 = min(h0 + heads, p.H_all);
    // (kBatch heads at a time, all loads ahead of the stores: an output may be its input.)
    for (int hb = h0; hb < h1; hb += kBatch) {
        Chunk<T> a[kBatch], b[kBatch];
        T *out[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const T *in;
            rows_of(p, min(hb + j, h1 - 1), t, in, out[j]);
            a[j] = *reinterpret_cast<const Chunk<T> *>(in + ca);
            b[j] = *reinterpret_cast<const Chunk<T> *>(in + cb);
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (hb + j >= h1) break;
            Chunk<T> ya, yb;
            if constexpr (INTERLEAVED) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float a0 = get(a[j].e[2 * e]), a1 = get(a[j].e[2 * e + 1]);
                    const float b0 = get(b[j].e[2 * e]), b1 = get(b[j].e[2 * e + 1]);
                    put(ya.e[2 * e], turn_a(a0, a1, c[e], s[e]));
                    put(ya.e[2 * e + 1], turn_b(a0, a1, c[e], s[e]));
                    put(yb.e[2 * e], turn_a(b0, b1, c[e + 4], s[e + 4]));
                    put(yb.e[2 * e + 1], turn_b(b0, b1, c[e + 4], s[e + 4]));
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float x = get(a[j].e[e]), y = get(b[j].e[e]);
                    put(ya.e[e], turn_a(x, y, c[e], s[e]));
                    put(yb.e[e], turn_b(x, y, c[e], s[e]));
                }
            }
            // (Copied channels keep their bits, infinities and NaN too.)
            *reinterpret_cast<Chunk<T> *>(out[j] + ca) = copy_a ? a[j] : ya;
            *reinterpret_cast<Chunk<T> *>(out[j] + cb) = copy_b ? b[j] : yb;
        }
    }
}

// A thread: token i / pairs, one pair; heads as above.
template <typename T>
__global__ void __launch_bounds__(kThreads) rope_pair_kernel(const RopeParams p, int heads)
{
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t t = i / p.n_pairs;
    const int pr = (int)(i - t * p.n_pairs);
    if (t >= p.N) return;
    const int ca = p.ca[pr], cb = p.cb[pr];
    const bool copy = p.turns[pr] < 0.0;
    float c = 1.f, s = 0.f;
    if (!copy) angle(p, p.pos + t * p.n_axes, pr, c, s);
    const int h0 = blockIdx.y * heads, h1 = min(h0 + heads, p.H_all);
    for (int hb = h0; hb < h1; hb += kBatch) {
        T a[kBatch], b[kBatch], *out[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const T *in;
            rows_of(p, min(hb + j, h1 - 1), t, in, out[j]);
            a[j] = in[ca];
            b[j] = in[cb];
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (hb + j >= h1) break;
            T ya, yb;
            put(ya, turn_a(get(a[j]), get(b[j]), c, s));
            put(yb, turn_b(get(a[j]), get(b[j]), c, s));
            out[j][ca] = copy ? a[j] : ya;
            out[j][cb] = copy ? b[j] : yb;
        }
    }
}

template <typename T>
hipError_t go(const RopeParams &p, hipStream_t s)
{
    const int units = p.chunks ? p.n_pairs / 8 : p.n_pairs;
    const int64_t threads = (int64_t)p.N * units;
    const int64_t blocks = (threads + kThreads - 1) / kThreads;
    // Heads per thread: all that leave 4,096 workgroups, at least 4 to share the angles.
    int heads = p.H_all;
    while (heads > 4 && blocks * ((p.H_all + heads - 1) / heads) < 4096) heads = (heads + 1) / 2;
    const dim3 grid((unsigned)blocks, (unsigned)((p.H_all + heads - 1) / heads));
    if (!p.chunks)
        hipLaunchKernelGGL(rope_pair_kernel<T>, grid, dim3(kThreads), 0, s, p, heads);
    else if (p.interleaved)
        hipLaunchKernelGGL((rope_chunk_kernel<T, true>), grid, dim3(kThreads), 0, s, p, units, heads);
    else
        hipLaunchKernelGGL((rope_chunk_kernel<T, false>), grid, dim3(kThreads), 0, s, p, units, heads);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const RopeParams &p, hipStream_t s) { return p.f32 ? go<float>(p, s) : go<uint16_t>(p, s); }

}  // namespace ress
