// Rotary positions with several axes.
//
// Memory bound: every element of Q and K is read and written once. A thread owns one chunk of
// a token's channels and walks over the heads, so that the angles (float64, reduced to a turn's
// fraction before the sine) are formed once per token and stay in registers. Neighbouring
// threads own neighbouring chunks, so that loads and stores cover whole rows; the chunk that a
// chunk's pairs meet is read a second time, from the L1 (with a pair of chunks a thread, rows
// went to memory as two halves each: 32 + 32 views' heads 173 us, now 70: 5.15 TB/s), and the
// two threads form half of their angles each and exchange them. Chunks have 16 bytes where
// the axes' halves, strides and addresses allow it, else 8 (32 + 32 views' heads with axes of 16,
// 24 and 24 channels 75 us, in pairs 84; in chunks of 4 bytes no better than in pairs). Else a
// thread owns a pair.
// One view of 1,374 tokens, 16 heads in float32, takes 5.5 us and is latency.
#include "layer_internal.h"

namespace ress {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float from_bf16(uint16_t b) { return __builtin_bit_cast(float, (uint32_t)b << 16); }

template <typename T, int V>
struct alignas(sizeof(T) * V) Chunk {
    T e[V];
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
__device__ __forceinline__ float turn_b(float a, float b, float c, float s) { return fmaf(b, c, a * s); }

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

// A thread: token i / lanes, chunk i % lanes (a token's lanes lie in one wave: its loads are
// ahead of its stores, also where an output is its input); heads blockIdx.y * heads ..., B of
// them in flight.
template <typename T, int V, int B, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads) rope_chunk_kernel(const RopeParams p, int lanes_log2, int heads)
{
    using Chunk = Chunk<T, V>;
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t t = i >> lanes_log2;
    const int c = (int)i & ((1 << lanes_log2) - 1);
    if (t >= p.N || c * V >= p.D) return;
    const bool copy = c * V >= p.turned;
    const int pair = p.pair_of[c], other = p.other[c];  // first pair; the chunk that its pairs meet
    const bool second = other < c;                      // (halves: this chunk is the pairs' b)
    const int h0 = blockIdx.y * heads, h1 = min(h0 + heads, p.H_all);
    // (The first heads are on their way while the angles are formed.)
    Chunk x[B], y[B];
    T *out[B];
    auto fetch = [&](int hb) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const T *in;
            rows_of(p, min(hb + j, h1 - 1), t, in, out[j]);
            x[j] = *reinterpret_cast<const Chunk *>(in + c * V);
            if constexpr (!INTERLEAVED) y[j] = *reinterpret_cast<const Chunk *>(in + other * V);
        }
    };
    fetch(h0);
    float cs[V], sn[V];
    if (!copy) {
        const int32_t *pos = p.pos + t * p.n_axes;
        if constexpr (INTERLEAVED) {
#pragma unroll
            for (int e = 0; e < V / 2; ++e) angle(p, pos, pair + e, cs[e], sn[e]);
        } else {
            // The a's thread forms the first half, the b's the second.
            const int mate = (threadIdx.x & 63) - c + other;
#pragma unroll
            for (int e = 0; e < V / 2; ++e) {
                float c0, s0;
                angle(p, pos, pair + e + (second ? V / 2 : 0), c0, s0);
                const float c1 = __shfl(c0, mate), s1 = __shfl(s0, mate);
                cs[e] = second ? c1 : c0;
                sn[e] = second ? s1 : s0;
                cs[e + V / 2] = second ? c0 : c1;
                sn[e + V / 2] = second ? s0 : s1;
            }
        }
    }
    for (int hb = h0; hb < h1; hb += B) {
#pragma unroll
        for (int j = 0; j < B; ++j) {
            if (hb + j >= h1) break;
            if (!copy) {  // (copied channels keep their bits, infinities and NaN too)
                if constexpr (INTERLEAVED) {
#pragma unroll
                    for (int e = 0; e < V / 2; ++e) {
                        const float a = get(x[j].e[2 * e]), b = get(x[j].e[2 * e + 1]);
                        put(x[j].e[2 * e], turn_a(a, b, cs[e], sn[e]));
                        put(x[j].e[2 * e + 1], turn_b(a, b, cs[e], sn[e]));
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float a = get(x[j].e[e]), b = get(y[j].e[e]);
                        put(x[j].e[e], second ? turn_b(b, a, cs[e], sn[e]) : turn_a(a, b, cs[e], sn[e]));
                    }
                }
            }
            *reinterpret_cast<Chunk *>(out[j] + c * V) = x[j];
        }
        if (hb + B < h1) fetch(hb + B);
    }
}

// A thread: token i / lanes, pair i % lanes; heads as above.
template <typename T, int B>
__global__ void __launch_bounds__(kThreads) rope_pair_kernel(const RopeParams p, int lanes_log2, int heads)
{
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t t = i >> lanes_log2;
    const int pr = (int)i & ((1 << lanes_log2) - 1);
    if (t >= p.N || pr >= p.n_pairs) return;
    const int ca = p.ca[pr], cb = p.cb[pr];
    const bool copy = p.turns[pr] < 0.0;
    float c = 1.f, s = 0.f;
    if (!copy) angle(p, p.pos + t * p.n_axes, pr, c, s);
    const int h0 = blockIdx.y * heads, h1 = min(h0 + heads, p.H_all);
    for (int hb = h0; hb < h1; hb += B) {
        T a[B], b[B], *out[B];
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const T *in;
            rows_of(p, min(hb + j, h1 - 1), t, in, out[j]);
            a[j] = in[ca];
            b[j] = in[cb];
        }
#pragma unroll
        for (int j = 0; j < B; ++j) {
            if (hb + j >= h1) break;
            T ya, yb;
            put(ya, turn_a(get(a[j]), get(b[j]), c, s));
            put(yb, turn_b(get(a[j]), get(b[j]), c, s));
            out[j][ca] = copy ? a[j] : ya;
            out[j][cb] = copy ? b[j] : yb;
        }
    }
}

template <typename T, int V, int B>
hipError_t go(const RopeParams &p, hipStream_t s)
{
    int lanes_log2 = 0;
    while ((V > 0 ? V : 2) << lanes_log2 < p.D) ++lanes_log2;
    const int64_t blocks = (((int64_t)p.N << lanes_log2) + kThreads - 1) / kThreads;
    // Heads per thread: all that leave 2,048 workgroups, at least one batch.
    int heads = p.H_all;
    while (heads > B && blocks * ((p.H_all + heads - 1) / heads) < 2048) heads = (heads + 1) / 2;
    heads = (heads + B - 1) / B * B;
    const dim3 grid((unsigned)blocks, (unsigned)((p.H_all + heads - 1) / heads));
    if constexpr (V > 0) {
        if (p.interleaved)
            hipLaunchKernelGGL((rope_chunk_kernel<T, V, B, true>), grid, dim3(kThreads), 0, s, p, lanes_log2, heads);
        else
            hipLaunchKernelGGL((rope_chunk_kernel<T, V, B, false>), grid, dim3(kThreads), 0, s, p, lanes_log2, heads);
    } else {
        hipLaunchKernelGGL((rope_pair_kernel<T, B>), grid, dim3(kThreads), 0, s, p, lanes_log2, heads);
    }
    return hipGetLastError();
}

// Heads that a thread has in flight: four, or one where there are fewer than four (one head of
// 392,025 tokens, four of which three repeat 37 us, one 30; three heads of 200,000 28 either way).
template <typename T, int V>
hipError_t by_heads(const RopeParams &p, hipStream_t s)
{
    return p.H_all < 4 ? go<T, V, 1>(p, s) : go<T, V, 4>(p, s);
}

template <typename T>
hipError_t by_chunk(const RopeParams &p, hipStream_t s)
{
    constexpr int V = 16 / sizeof(T);
    return p.chunk == V ? by_heads<T, V>(p, s) : p.chunk == V / 2 ? by_heads<T, V / 2>(p, s) : by_heads<T, 0>(p, s);
}

}  // namespace

hipError_t launch_rope(const RopeParams &p, hipStream_t s) { return p.f32 ? by_chunk<float>(p, s) : by_chunk<uint16_t>(p, s); }

}  // namespace ress
