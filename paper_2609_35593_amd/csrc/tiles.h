// Tiles of 64 rows by 64 bf16 channels in LDS and their bf16 MFMA operands, shared by
// the windowed attention's kernels.
//
// A tile is row-major, 128 bytes a row, its 16-byte chunks XOR-swizzled per row (swz), so
// that both ways of reading it are free of bank conflicts: "rows" (one row a lane, 8
// neighbouring channels) and "columns" (one channel a lane, 8 rows, by
// ds_read_b64_tr_b16). It comes from global memory by direct loads to LDS; the swizzle is
// applied by choosing each lane's source chunk.
//
// v_mfma_f32_32x32x16_bf16: A lane l holds row l%32, contraction entries 8(l/32)..+7; B
// lane l column l%32, the same entries; D lane l column l%32, rows 8(v/4) + 4(l/32) + v%4
// for v = 0..15. A product's D, rounded to bf16, is the next product's B operand as it
// lies: entries 8u..8u+7 of a lane are contraction rows 16u + {0..3} + 4(l/32) and
// 16u + 8 + {0..3} + 4(l/32), and column reads take the rows in that order.
#pragma once

#include "layer_internal.h"

namespace ress {
namespace tiles {

typedef __bf16 bf16x8 __attribute__((__vector_size__(8 * sizeof(__bf16))));
typedef __bf16 bf16x2 __attribute__((__vector_size__(2 * sizeof(__bf16))));
typedef short s16x4 __attribute__((__vector_size__(4 * sizeof(short))));
typedef short s16x8 __attribute__((__vector_size__(8 * sizeof(short))));
typedef float f32x16 __attribute__((__vector_size__(16 * sizeof(float))));
typedef float f32x4 __attribute__((__vector_size__(4 * sizeof(float))));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int kHead = 64;            // channels of a head
constexpr int kTile = 64;            // rows of a tile
constexpr int kTileBytes = 64 * 128;

__device__ __forceinline__ int swz(int row) { return (((row >> 1) & 1) << 2) | ((row >> 2) & 3); }

__device__ __forceinline__ void wait_vm_all() { __builtin_amdgcn_s_waitcnt(0x0F70); }  // vmcnt(0)

__device__ __forceinline__ unsigned int bf16_bits(float x)
{
    return (unsigned int)__builtin_bit_cast(unsigned short, (__bf16)x);
}

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Loads of one tensor's tiles by WAVES waves: this lane's share is rows r0 + 8 WAVES u, physical
// chunk lane & 7. (The swizzle depends on row bits 1-3 only, so one source chunk serves all u,
// but for a single wave, where bit 3 alternates with u and the source chunk by 2.)
// 64-bit scalar arithmetic up to a tile's first row, 32 bits inside it (63 rows of at most
// 2^22 elements); a whole tile takes no vector arithmetic at all.
template <int WAVES>
struct Loader {
    const uint16_t *base;
    int64_t stride;  // elements between rows
    int wave, lane;
    unsigned int whole, whole1;  // byte offsets in a whole tile, for even and odd u
    __device__ __forceinline__ Loader(const uint16_t *base_, int64_t stride_, int wave_, int lane_)
        : base(base_), stride(stride_), wave(wave_), lane(lane_)
    {
        const int r0 = wave * 8 + (lane >> 3);
        whole = (unsigned int)r0 * (unsigned int)(2 * stride) + source(r0, lane);
        whole1 = (unsigned int)r0 * (unsigned int)(2 * stride) + (source(r0, lane) ^ (WAVES == 1 ? 32u : 0u));
    }
    static __device__ __forceinline__ unsigned int source(int r0, int l) { return (unsigned int)(((l & 7) ^ swz(r0)) << 4); }
    // Rows row0 .. row0 + 63 into `dst`; rows outside [lo, hi) (hi > lo) repeat the nearest
    // one inside, rows in [gap, end) (end < hi, inside the tile, or gap >= end) row `end`; none
    // of them is read.
    __device__ __forceinline__ void operator()(int row0, int lo, int hi, int gap, int end, unsigned char *dst) const
    {
        const unsigned int step = (unsigned int)(2 * stride);  // bytes
        if (row0 >= lo && row0 + kTile <= hi && gap >= end) {
            const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
                const_cast<uint16_t *>(base + (int64_t)row0 * stride), 0, (int)((kTile - 1) * step + 128u), 0x00020000);
#pragma unroll
            for (int u = 0; u < 8 / WAVES; ++u)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void *)(dst + (u * WAVES + wave) * 1024), 16,
                                                         WAVES == 1 && u % 2 ? whole1 : whole,
                                                         (int)(8 * WAVES * u * step), 0, 0);
        } else {
            // (Formed from the lane each time: kept over the caller's loop, these values would be
            // spilled, and their reload would wait for the loads in flight.)
            int l = lane;
            asm volatile("" : "+v"(l));
            const int r0 = wave * 8 + (l >> 3);
            const unsigned int coff = source(r0, l);
            const int first = min(max(row0, lo), hi - 1);
            const int last = max(min(row0 + kTile, hi) - 1, first);
            const __amdgpu_buffer_rsrc_t rs =
                __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(base + (int64_t)first * stride), 0,
                                                  (int)((unsigned int)(last - first) * step + 128u), 0x00020000);
#pragma unroll
            for (int u = 0; u < 8 / WAVES; ++u) {
                int row = min(max(row0 + r0 + 8 * WAVES * u, first), last);
                row = (row >= gap && row < end ? end : row) - first;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void *)(dst + (u * WAVES + wave) * 1024), 16,
                                                         (unsigned int)row * step + (WAVES == 1 && u % 2 ? coff ^ 32u : coff),
                                                         0, 0, 0);
            }
        }
    }
};

// Per-lane offsets of the two kinds of reads.
struct Reader {
    int row[4];     // row l%32, channels 16 kk + 8 (l/32) .. +7
    int col[2][2];  // rows 8 r + 4 (l/32) + (l%16)/4, channels 32 dh + 16 ((l/16)&1) + 4 (l%4)
    __device__ __forceinline__ explicit Reader(int lane)
    {
        const int hh = lane >> 5, ql = lane & 31, g16 = (lane >> 4) & 1, s16 = lane & 15;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) row[kk] = ql * 128 + (((2 * kk + hh) ^ swz(ql)) << 4);
#pragma unroll
        for (int dh = 0; dh < 2; ++dh)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int k = 8 * r + 4 * hh + (s16 >> 2);
                const int d = 32 * dh + 16 * g16 + 4 * (s16 & 3);
                col[dh][r] = k * 128 + (((d >> 3) ^ swz(k)) << 4) + (d & 7) * 2;
            }
    }
    // Rows 32 t .. 32 t + 31 of a tile, channels 16 kk .. +15.
    __device__ __forceinline__ bf16x8 rows(const unsigned char *tile, int t, int kk) const
    {
        return *reinterpret_cast<const bf16x8 *>(tile + t * 32 * 128 + row[kk]);
    }
    // Channels 32 dh .. +31 (one a lane) of rows 32 t + 16 u .. +15.
    __device__ __forceinline__ bf16x8 cols(const unsigned char *tile, int t, int u, int dh) const
    {
        const unsigned char *base = tile + (t * 32 + u * 16) * 128;
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(base + col[dh][0]));
        const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(base + col[dh][1]));
        return __builtin_bit_cast(bf16x8, s16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
    }
};

// A lane's 16 products rounded to the B operands of two 16-row steps.
__device__ __forceinline__ void pack(const f32x16 &x, bf16x8 (&b)[2])
{
#pragma unroll
    for (int u = 0; u < 2; ++u)
        b[u] = bf16x8{(__bf16)x[8 * u + 0], (__bf16)x[8 * u + 1], (__bf16)x[8 * u + 2], (__bf16)x[8 * u + 3],
                      (__bf16)x[8 * u + 4], (__bf16)x[8 * u + 5], (__bf16)x[8 * u + 6], (__bf16)x[8 * u + 7]};
}

// sum + the 16 values of two packed operands, in pairs.
__device__ __forceinline__ float add_up(const bf16x8 (&b)[2], float sum)
{
    const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int j = 0; j < 8; j += 2) sum = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{b[u][j], b[u][j + 1]}, ones, sum, false);
    return sum;
}

// The keys that query position p sees: [lo, hi) and [0, sk).
struct Seen {
    int lo, hi, sk;
};
__device__ __forceinline__ Seen seen_by(const WindowParams &p, int pos)
{
    const int f = p.frames(pos);
    Seen s;
    s.hi = min((f + (p.causal ? 1 : p.window)) * p.frame, p.n_k);
    s.lo = min(max((f - p.window + 1) * p.frame, 0), s.hi);
    s.sk = min(p.n_sink, p.causal ? s.hi : p.n_k);
    return s;
}

// Scores (keys or queries base .. base + 31, the lane's from 4 (l/32) on, which `lo` and `sk`
// allow for) outside [lo, lo + span), and with `sinks` (wave-uniform) not below sk, become -inf.
// One vector comparison and selection a score and condition: conditions joined as masks go
// through the scalar unit and wait for it each time.
__device__ __forceinline__ void hide(f32x16 &s, int base, int lo, unsigned int span, bool sinks, int sk)
{
    asm volatile("" ::: "memory");  // (a real branch around this: whole tiles skip it)
    if (sinks) {
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int key = __builtin_amdgcn_readfirstlane(base + (v >> 2) * 8 + (v & 3));
            float x = (unsigned int)(key - lo) < span ? s[v] : -INFINITY;
            asm volatile("" : "+v"(x));
            s[v] = key < sk ? s[v] : x;
        }
    } else {
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int key = __builtin_amdgcn_readfirstlane(base + (v >> 2) * 8 + (v & 3));
            s[v] = (unsigned int)(key - lo) < span ? s[v] : -INFINITY;
        }
    }
}

// One row (column l%32 of two transposed accumulators of 32 channels each) times `f`, to
// bf16 global memory.
__device__ __forceinline__ void store_row(uint16_t *row, const f32x16 (&acc)[2], float f, int hh)
{
#pragma unroll
    for (int dh = 0; dh < 2; ++dh)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const unsigned int lo = bf16_bits(acc[dh][g * 4 + 0] * f) | (bf16_bits(acc[dh][g * 4 + 1] * f) << 16);
            const unsigned int hi = bf16_bits(acc[dh][g * 4 + 2] * f) | (bf16_bits(acc[dh][g * 4 + 3] * f) << 16);
            *reinterpret_cast<uint2 *>(row + dh * 32 + g * 8 + hh * 4) = make_uint2(lo, hi);
        }
}

// The queries [lo, hi) that see key s (by their index, not their position).
struct SeenBy {
    int lo, hi;
};
__device__ __forceinline__ SeenBy queries_of(const WindowParams &p, int s)
{
    const int f = p.frames(s);
    const bool sink = s < p.n_sink;
    const int lo = p.causal ? f * p.frame : sink ? 0 : (f - p.window + 1) * p.frame;
    SeenBy r;
    r.lo = min(max(lo - p.q_offset, 0), p.n_q);
    r.hi = sink ? p.n_q : min(max((f + p.window) * p.frame - p.q_offset, r.lo), p.n_q);
    return r;
}

}  // namespace tiles
}  // namespace ress
