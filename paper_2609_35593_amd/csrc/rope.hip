// Rotary positions with several axes.
//
// Memory bound: every element of Q and K is read and written once. A thread owns one
// 16-byte chunk of a token's channels and walks over the heads, so that the angles (float64,
// reduced to a turn's fraction before the sine) are formed once per token and stay in
// registers. Neighbouring threads own neighbouring chunks, so that loads and stores cover
// whole rows; the chunk that a chunk's pairs meet is read a second time, from the L1 (with a
// pair of chunks a thread, rows went to memory as two halves each: 32 + 32 views' heads 173
// us, now 72: 5.0 TB/s). Where pairs do not come in whole chunks, a thread owns a pair.
// One view of 1,374 tokens, 16 heads in float32, takes 5.5 us and is latency.
#include "layer_internal.h"

namespace ress {
namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 4;  // heads of a thread in flight

__device__ __forceinline__ float from_bf16(uint16_t b) { return __builtin_bit_cast(float, (uint32_t)b << 16); }

template <typename T>
struct alignas(16) Chunk {
    static constexpr int V = 16 / sizeof(T);
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
// ahead of its stores, also where an output is its input); heads blockIdx.y * heads ...
template <typename T, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads) rope_chunk_kernel(const RopeParams p, int lanes_log2, int heads)
{
    constexpr int V = Chunk<T>::V;
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t t = i >> lanes_log2;
    const int c = (int)i & ((1 << lanes_log2) - 1);
    if (t >= p.N || c * V >= p.D) return;
    const bool copy = c * V >= p.turned;
    const int pair = p.pair_of[c], other = p.other[c];  // first pair; the chunk that its pairs meet
    const bool second = other < c;                      // (halves: this chunk is the pairs' b)
    float cs[V], sn[V];
    if (!copy) {
        const int32_t *pos = p.pos + t * p.n_axes;
#pragma unroll
        for (int e = 0; e < (INTERLEAVED ? V / 2 : V); ++e) angle(p, pos, pair + e, cs[e], sn[e]);
    }
    const int h0 = blockIdx.y * heads, h1 = min(h0 + heads, p.H_all);
    for (int hb = h0; hb < h1; hb += kBatch) {
        Chunk<T> x[kBatch], y[kBatch];
        T *out[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const T *in;
            rows_of(p, min(hb + j, h1 - 1), t, in, out[j]);
            x[j] = *reinterpret_cast<const Chunk<T> *>(in + c * V);
            if constexpr (!INTERLEAVED) y[j] = *reinterpret_cast<const Chunk<T> *>(in + other * V);
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
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
            *reinterpret_cast<Chunk<T> *>(out[j] + c * V) = x[j];
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
    int lanes_log2 = 0;
    while (Chunk<T>::V << lanes_log2 < p.D) ++lanes_log2;
    const int64_t threads = p.chunks ? (int64_t)p.N << lanes_log2 : (int64_t)p.N * p.n_pairs;
    const int64_t blocks = (threads + kThreads - 1) / kThreads;
    // Heads per thread: all that leave 2,048 workgroups, at least one batch.
    int heads = p.H_all;
    while (heads > kBatch && blocks * ((p.H_all + heads - 1) / heads) < 2048) heads = (heads + 1) / 2;
    heads = (heads + kBatch - 1) / kBatch * kBatch;
    const dim3 grid((unsigned)blocks, (unsigned)((p.H_all + heads - 1) / heads));
    if (!p.chunks)
        hipLaunchKernelGGL(rope_pair_kernel<T>, grid, dim3(kThreads), 0, s, p, heads);
    else if (p.interleaved)
        hipLaunchKernelGGL((rope_chunk_kernel<T, true>), grid, dim3(kThreads), 0, s, p, lanes_log2, heads);
    else
        hipLaunchKernelGGL((rope_chunk_kernel<T, false>), grid, dim3(kThreads), 0, s, p, lanes_log2, heads);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const RopeParams &p, hipStream_t s) { return p.f32 ? go<float>(p, s) : go<uint16_t>(p, s); }

}  // namespace ress
