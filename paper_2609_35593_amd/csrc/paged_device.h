// What the kernels of attention over pages share: which sequence a block of rows is of, what its
// rows see, and how its keys are cut.
#pragma once

#include "pages_internal.h"
#include "scan.h"
#include "tiles.h"

namespace ress {
namespace paged {

using namespace tiles;

// Rows that keys which are not to be read come from.
__device__ const uint16_t zero_row[64] __attribute__((aligned(128))) = {};

// A block: `left` rows (token t, head hk group + g; t outer) of sequence b from head g0 of its token t0 on. The
// sequence's tokens begin at row cu of q, the first one's position is pos0.
struct Block {
    int b, t0, g0, left, cu, pos0, len;
};
// Row j of a block: token of the sequence, head of the K/V head's.
struct Row {
    int t, g;
};
__device__ __forceinline__ Row row_of(const PagedParams &p, const Block &x, int j)
{
    const int n = p.groups(x.g0 + j);
    return {x.t0 + n, x.g0 + j - n * p.group};
}

// A sequence's rows of q, clamped (so a block's rows lie in [0, N) whatever the offsets hold), and its blocks.
struct Rows {
    int cu, end;
    template <int ROWS>
    __device__ __forceinline__ int blocks(const PagedParams &p) const
    {
        return (int)(((int64_t)(end - cu) * p.group + ROWS - 1) / ROWS);
    }
};
__device__ __forceinline__ Rows rows_of(const PagedParams &p, int from, int to)
{
    const int cu = min(max(from, 0), p.N);
    return {cu, min(max(to, cu), p.N)};
}

template <int ROWS>
__device__ __forceinline__ void block_of(const PagedParams &p, Block &x, int b, int index, const Rows &r, int len)
{
    const int n = r.end - r.cu;
    x.b = b;
    x.cu = r.cu;
    x.len = min(max(len, 0), p.capacity);
    x.pos0 = x.len - n;
    const int64_t first = (int64_t)index * ROWS, rows = (int64_t)n * p.group;
    x.t0 = (int)((uint32_t)first / (uint32_t)p.group);  // (2^24 tokens of 256 heads at most)
    x.g0 = (int)(first - (int64_t)x.t0 * p.group);
    x.left = (int)(rows - first < ROWS ? rows - first : ROWS);
}

constexpr int kMostBlocks = 1 << 29;  // sums of blocks stop here
__device__ __forceinline__ int sum_of(int a, int b) { return min(a + b, kMostBlocks); }

// Block `index` of all sequences' blocks of ROWS rows; false behind the last. Each wave looks for itself: at all sequences, 256 of
// them in one round trip, or, where there are more than kMostScanned, in the list of where each one's blocks begin, 64 ways at a
// time. (One token of each of 512 / 768 / 1,024 / 4,096 / 16,384 sequences over 1,000 keys, us: 28.2 / 44.2 / 56.7 / 377 /
// 3,927 by scans; 31.3 / 42.0 / 52 / 203 / 778 with the list and its launch.)
template <int ROWS>
__device__ __forceinline__ bool find_block(const PagedParams &p, int index, Block &x)
{
    const int lane = threadIdx.x & 63;
    if (p.starts) {
        if (index >= p.starts[p.B]) return false;
        int b = 0;
        for (int n = p.B; n > 1;) {
            const int step = (n + 63) / 64, at = lane * step;
            const int l = __popcll(__ballot(at < n && p.starts[b + min(at, n - 1)] <= index)) - 1;
            b += l * step;
            n = min(step, n - l * step);
        }
        b = __builtin_amdgcn_readfirstlane(b);
        block_of<ROWS>(p, x, b, index - p.starts[b], rows_of(p, p.cu_q[b], p.cu_q[b + 1]), p.lens[b]);
        return true;
    }
    int before = 0;
    for (int b0 = 0; b0 < p.B; b0 += 256) {
        int from[4], to[4], len[4];
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (b0 + c * 64 < p.B) {
                const int b = min(b0 + c * 64 + lane, p.B - 1);
                from[c] = p.cu_q[b];
                to[c] = p.cu_q[b + 1];
                len[c] = p.lens[b];
            }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int first = b0 + c * 64;
            if (first >= p.B) break;
            const Rows r = rows_of(p, from[c], to[c]);
            const int blocks = first + lane < p.B ? r.blocks<ROWS>(p) : 0;
            const int sum = sum_of(scan_wave(blocks, sum_of), before);
            const uint64_t here = __ballot(blocks > 0 && index < sum && index >= sum - blocks);
            if (here) {
                const int l = __builtin_ctzll(here);
                block_of<ROWS>(p, x, first + l, index - __builtin_amdgcn_readlane(sum - blocks, l),
                               {__builtin_amdgcn_readlane(r.cu, l), __builtin_amdgcn_readlane(r.end, l)},
                               __builtin_amdgcn_readlane(len[c], l));
                return true;
            }
            before = __builtin_amdgcn_readlane(sum, 63);
        }
    }
    return false;
}

// A block's part: of `cuts`, the block's index among all sequences', and among all parts the first one's and how far apart they
// are.
struct Part {
    Block x;
    int split, cuts, block, first, step;
};

// The part that `pick` names by its index among all blocks' parts; false where there is none. pick is given how many parts there are,
// with COUNT, and may answer -1. A block's parts go by its share of all keys, so that workgroups hold about as many each, whatever
// the sequences' lengths (by as many parts for each block, single tokens of 24 sequences of 1 to 20,000 keys on a log scale, 16
// heads for 4, 90 us, so 21; of 28 of up to 33,462 evenly, 8 heads for one, 51 and 33). Of a sequence the parts of one
// range of keys lie side by side. Each wave looks by itself. The weights are the keys that a sequence's last token sees, their sums
// float32 in a fixed order: the same in every workgroup.
template <int ROWS, bool COUNT, class Pick>
__device__ __forceinline__ bool find_part(const PagedParams &p, Pick pick, Part &part)
{
    const int lane = threadIdx.x & 63;
    int from = 0, to = 0, len = 0, blocks = 0;
    float keys = 0.f, all = 0.f;
    auto look = [&](int b0) __attribute__((always_inline)) {
        const int b = min(b0 + lane, p.B - 1);
        from = p.cu_q[b];
        to = p.cu_q[b + 1];
        len = p.lens[b];
        blocks = b0 + lane < p.B ? rows_of(p, from, to).blocks<ROWS>(p) : 0;
        keys = (float)min(max(len, 0), p.most_keys);
    };
#pragma nounroll
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        look(b0);
        all = fmaf((float)blocks, keys, all);
    }
    const float each = 1.f / fmaxf(sum_wave(all) * p.share, (float)((ROWS == 32 ? kTileLeast : kWideLeast) * kTile));
    auto cuts_each = [&]() __attribute__((always_inline)) { return min(max((int)fmaf(keys, each, 0.5f), 1), p.splits); };
    int total = 0;
    if constexpr (COUNT)
#pragma nounroll
        for (int b0 = 0; b0 < p.B; b0 += 64) {
            if (p.B > 64) look(b0);
            total = sum_of(total, __builtin_amdgcn_readlane(scan_wave(blocks * cuts_each(), sum_of), 63));
        }
    const int index = pick(total);
    int before = 0, blocks_before = 0;
#pragma nounroll
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        if (p.B > 64) look(b0);
        const int cuts = cuts_each(), parts = blocks * cuts;
        const int sum = sum_of(scan_wave(parts, sum_of), before), blocks_sum = COUNT ? sum_of(scan_wave(blocks, sum_of), blocks_before) : 0;
        const uint64_t here = __ballot(parts > 0 && index < sum && index >= sum - parts);
        if (here) {
            const int l = __builtin_ctzll(here), first = __builtin_amdgcn_readlane(sum - parts, l), at = index - first;
            const Rows r = rows_of(p, from, to);
            part.cuts = __builtin_amdgcn_readlane(cuts, l);
            part.step = __builtin_amdgcn_readlane(blocks, l);
            part.split = __builtin_amdgcn_readfirstlane((int)((uint32_t)at / (uint32_t)part.step));
            const int block = at - part.split * part.step;
            part.first = first + block;
            part.block = __builtin_amdgcn_readlane(blocks_sum - blocks, l) + block;
            block_of<ROWS>(p, part.x, b0 + l, block, {__builtin_amdgcn_readlane(r.cu, l), __builtin_amdgcn_readlane(r.end, l)},
                           __builtin_amdgcn_readlane(len, l));
            return true;
        }
        before = __builtin_amdgcn_readlane(sum, 63);
        blocks_before = __builtin_amdgcn_readlane(blocks_sum, 63);
    }
    return false;
}

// The keys that position pos of a sequence of len tokens sees: [lo, hi) and [0, sk). (Before its first: none.)
__device__ __forceinline__ Seen seen_at(const PagedParams &p, int pos, int len)
{
    Seen s = {0, 0, 0};
    if (pos < 0) return s;
    const int f = p.frames(pos);
    s.hi = min((f + 1) * p.frame, len);
    s.lo = min(max((f - p.window + 1) * p.frame, 0), s.hi);
    s.sk = min(p.n_sink, s.hi);
    return s;
}

// The 64-key tiles that any row of a block sees, numbered through: [0, ns) and [w0, w1).
struct Tiles {
    int ns, w0, n;
    __device__ __forceinline__ int key(int i) const { return (i < ns ? i : i - ns + w0) * kTile; }
};
__device__ __forceinline__ Tiles tiles_of(const Seen &first, const Seen &last)
{
    Tiles t;
    t.ns = (last.sk + kTile - 1) / kTile;
    int w1 = (last.hi + kTile - 1) / kTile;
    t.w0 = first.lo / kTile;
    if (first.lo >= last.hi) t.w0 = w1 = t.ns;
    if (t.w0 < t.ns) t.w0 = t.ns;
    if (w1 < t.w0) w1 = t.w0;
    t.n = t.ns + w1 - t.w0;
    return t;
}

// Scores of keys that are not there become -inf: bit 8 (v / 4) + v % 4 of `bits` tells of score v. (By masks in vector registers:
// sixteen conditions held as scalars made the kernels spill.)
__device__ __forceinline__ void drop(f32x16 &s, unsigned int bits)
{
    asm volatile("" : "+v"(bits));  // (formed here each time, else the masks are kept over the caller's loops)
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        const int there = (int)(bits << (31 - ((v >> 2) * 8 + (v & 3)))) >> 31;
        const float x = s[v];  // (the bit cast of a vector's element in place reads its first one)
        s[v] = __builtin_bit_cast(float, (__builtin_bit_cast(int, x) & there) | (~there & (int)0xff800000));
    }
}

}  // namespace paged
}  // namespace ress
