// Internal declarations shared by the kernels and the C ABI layer of ress_layer.h.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include "ress_layer.h"

namespace ress {

struct NormParams {
    int64_t rows, x_stride, y_stride;
    int width;
    float eps;
    bool x_f32, y_f32;
    const void *x;
    const float *gamma, *beta;  // null: 1, 0
    void *y;
    float *mean, *rstd;  // null: not wanted
};

struct NormBwdParams {
    int64_t rows, x_stride, y_stride;
    int width;
    int parts;  // workgroups, each with a row of partial sums (null `part`: none wanted)
    bool x_f32, y_f32;
    const void *dy, *x;
    const float *gamma, *mean, *rstd;
    void *dx;
    float *part;  // [parts][2][width]: dgamma, dbeta
    float *dgamma, *dbeta;
};

// Workgroups of the backward pass at most, each with a row of partial sums.
int norm_bwd_parts(int64_t rows);

// n / d for 0 <= n < 2^31 by a product and a shift (a division is some 30 instructions, which
// calls of a few tiles felt). With 2^(l-1) < d <= 2^l and mul = ceil(2^(31+l) / d) < 2^32, the product's
// excess over n / d, below 2^31 / 2^(31+l) <= 1 / d, reaches no next integer.
struct Divider {
    uint32_t mul;
    int shift;
    __host__ __device__ int operator()(int n) const
    {
        return (int)((uint32_t)((uint64_t)((uint32_t)n << 1) * mul >> 32) >> shift);
    }
};
inline Divider divider(int d)
{
    int l = 0;
    while (((int64_t)1 << l) < d) ++l;
    return {(uint32_t)((((uint64_t)1 << (31 + l)) + d - 1) / d), l};
}

constexpr int kMaxPairs = RESS_MAX_ROPE_D / 2;
constexpr int kMaxChunks = 64;  // of a token: one wave's

struct RopeParams {
    int H, H_all;  // heads of q; of q and k together
    int N, n_axes, n_pairs, D;
    int turned;  // channels that turn, the first ones
    bool f32, inverse, interleaved;
    int chunk;  // channels of the chunks that pairs come in (see rope.hip); 0: none
    const int32_t *pos;
    const void *q_in, *k_in;
    void *q_out, *k_out;
    ress_strides qi, ki, qo, ko;
    double turns[kMaxPairs];   // turns per position; < 0: a pair that is copied
    uint8_t axis[kMaxPairs];
    uint8_t ca[kMaxPairs], cb[kMaxPairs];  // the pair's channels
    // chunk > 0: the first pair of chunk c, and the chunk that holds its pairs' other channels
    uint8_t pair_of[kMaxChunks], other[kMaxChunks];
};

// References of softmax rows: the base-2 logit s `scale` of a score s, in one of two forms. A near one
// is that product, rounded. A far one, from 2^24 on, is s `unit`, the power of two at or above the scale: exact, so that
// differences from it are, and never below 2^24 itself, so that it tells its form, and references compare as their logits do.
struct References {
    float scale, unit, rest;  // rest = scale / unit, in (1/2, 1]
#ifdef __HIPCC__
    __device__ __forceinline__ bool far(float ref) const { return !(fabsf(ref) < 0x1p24f); }
    __device__ __forceinline__ float of(float score) const { return far(score * unit) ? score * unit : score * scale; }
    __device__ __forceinline__ float base2(float ref) const { return far(ref) ? ref * rest : ref; }
    // a - b in base 2, each as its form holds it: one rounding, or two of far ones.
    __device__ __forceinline__ float difference(float a, float b) const
    {
        if (far(a)) return far(b) ? (a - b) * rest : fmaf(a, rest, -b);
        return far(b) ? fmaf(-b, rest, a) : a - b;
    }
#endif
};

inline References references(float scale)
{
    int e;
    const float f = frexpf(scale, &e);  // scale = f 2^e, f in [1/2, 1)
    return f == 0.5f ? References{scale, scale, 1.f} : References{scale, ldexpf(1.f, e), f};
}

constexpr int kMaxSplits = 32;  // workgroups that share a block's or sequence's keys, whose parts one wave joins

struct WindowParams {
    int H, H_kv, group;  // group = H / H_kv
    int n_q, n_k, q_offset;
    int frame, window, n_sink;  // (window x frame below 2^28, see sights)
    Divider frames, q_blocks, groups;  // of frame, n_qb, group
    bool causal;
    int n_qb, n_kb;  // blocks of 128 / groups queries, of 128 keys
    int splits;      // workgroups that share a block's keys (forward)
    float scale, scale_log2;  // of dq and dk; of the logits, in base 2
    References refs;          // (forward)
    ress_strides qs, ks, vs, os;
    const uint16_t *q, *k, *v;
    uint16_t *o;
    float *lse;
    float *part;        // splits > 1: [splits][H][n_q][64], unnormalised outputs,
    float2 *part_row;   // and [splits][H][n_q], references (scores) and sums
};

// Positions stay below 2^25, so frames and windows beyond 2^26 act as 2^26 does, whose product
// leaves room in 64 bits.
inline int at_most_2_26(int x) { return x < (1 << 26) ? x : 1 << 26; }
// The frame and window that kernels take: positions stay below 2^25, so a window of 2^25 / frame +
// 2 frames reaches all of them, and its products with frame fit 32 bits.
inline void sights(int frame, int window, int &f, int &w)
{
    f = at_most_2_26(frame);
    const int most = (1 << 25) / f + 2;
    w = window < most ? window : most;
}
inline int64_t window_tokens(int frame, int window) { return (int64_t)at_most_2_26(frame) * at_most_2_26(window); }

// How the forward pass spreads over the chip: key groups in a workgroup (1, 2, 4),
// workgroups per block of 128 / groups queries. A function of the shape alone.
struct WindowPlan {
    int groups, splits;
};
WindowPlan window_plan(const ress_window_shape *s);

struct WindowBwdParams {
    WindowParams w;  // o: the forward's output, read; lse: read
    ress_strides dos, dqs, dks, dvs;
    const uint16_t *d_o;
    uint16_t *dq, *dk, *dv;
    float *ndelta;  // [H][n_q]: -sum_d d_o o
    float *lse2;    // [H][n_q]: lse in base 2, +inf where a query sees nothing
    // The keys' pass: blocks of 128 keys, those with sinks first, in slices; items per head.
    int sink_blocks, sink_slices, slices, items;
    float *part;    // [H_kv items][2][128][64]: dk, dv of the slices of a block that has several
};

// How the backward pass spreads over the chip. A function of the shape alone.
struct WindowBwdPlan {
    int groups;  // key groups of the queries' pass
    int sink_blocks, sink_slices, slices, items;
};
WindowBwdPlan window_bwd_plan(const ress_window_shape *s);
// Of `blocks` blocks of keys those whose lists are cut: how many, from block `first` on.
int window_bwd_joined(const WindowBwdPlan &p, int blocks, int &first);

struct DecodeParams {
    int B, H, H_kv, group;
    int capacity, frame, window, n_sink;  // (frame, window: see sights)
    Divider frames;  // of frame
    int splits;
    float scale_log2;
    int64_t q_batch, q_head, k_batch, v_batch, o_batch, o_head;
    ress_strides ks, vs;
    const uint16_t *q, *k, *v;
    const int32_t *lens;
    uint16_t *o;
    float *part;  // [B][H][splits][66]: reference, sum, output
};

constexpr int kHeadWaves = 8;  // of decode_kernel (us with 4 / 8: 16 heads of 6,870 keys 10.5 / 9.3)
constexpr int kTileWaves = 4;  // of decode_tile_kernel: 64 KiB of slots, two workgroups a CU
int decode_splits(const ress_decode_shape *s);

hipError_t launch_norm(const NormParams &p, hipStream_t s);
hipError_t launch_norm_bwd(const NormBwdParams &p, hipStream_t s);
hipError_t launch_rope(const RopeParams &p, hipStream_t s);
hipError_t launch_window(const WindowParams &p, int groups, hipStream_t s);
hipError_t launch_window_bwd(const WindowBwdParams &p, int groups, hipStream_t s);
hipError_t launch_decode(const DecodeParams &p, hipStream_t s);

}  // namespace ress
