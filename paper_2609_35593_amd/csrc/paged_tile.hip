// Attention of new tokens over pages, and the join of keys that were split.
//
// tile_kernel: a workgroup owns 32 rows, the columns of its matrix products: a row is a new token
// and one of the query heads that share a K/V head, so that those heads' products come from one
// read of the keys. Its tiles of 64 keys go to its four waves, a run of them each. A lane finds its key's page
// in the table a tile ahead; the rows of K come straight to registers as the product's operand, those
// of V through LDS slots of the wave's own, so that no wave waits for another before the join. A
// weight enters its product as two bf16 numbers, itself rounded and what that leaves (see window_decode.hip).
//
// Keys on a page outside the cache, and keys that no row of the block sees, are not read: a row of zeros
// takes their place, and their scores are hidden.
//
// Measured: one token of 16 heads for 4 over 43,961 keys 12.8 us and the join 3.8, where their 45 MB take 8.7: 256 workgroups, a wave of
// which waits for 2 or 3 tiles one behind the other. One token of each of 4,096 sequences over 1,000 keys of one K/V head 203 us, 5.2
// TB/s, a copy's rate. One token of each of 24 sequences of 1 to 20,000 keys on a log scale, 16 heads for 4, 21 us.
#include <float.h>

#include "paged_device.h"

namespace ress {
namespace {

using namespace paged;

constexpr int kWaves = 4, kRows = 32;
constexpr int kPart = 66;  // floats of a wave's part of a row: reference, sum, 64 channels
// References are scores before their scale. A part without keys has one at or below every score,
// and finite: its sums are 0 whatever their weight.
constexpr float kNone = -FLT_MAX;

__global__ void __launch_bounds__(64 * kWaves, 2) tile_kernel(const PagedParams p)
{
    constexpr int kStep = 33;  // floats between a part's rows in LDS: no conflicts
    __shared__ __attribute__((aligned(1024))) unsigned char v_0[kWaves * kTileBytes], v_1[kWaves * kTileBytes];
    static_assert(2 * kPart * kStep * 4 <= (int)sizeof v_0, "two waves' parts fit a slot array");
    Part part;
    if (!(p.splits > 1 ? find_part<kRows, false>(p, [](int) { return (int)blockIdx.y; }, part) : find_block<kRows>(p, blockIdx.x, part.x)))
        return;
    const Block &x = part.x;
    const int hk = p.splits > 1 ? blockIdx.x : blockIdx.y, split = p.splits > 1 ? part.split : 0, cuts = p.splits > 1 ? part.cuts : 1;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hh = lane >> 5, ql = lane & 31;

    const Seen sa = seen_at(p, x.pos0 + x.t0, x.len), sb = seen_at(p, x.pos0 + row_of(p, x, x.left - 1).t, x.len);
    const Tiles tl = tiles_of(sa, sb);
    const int begin = (int)((int64_t)tl.n * split / cuts), end = (int)((int64_t)tl.n * (split + 1) / cuts);
    const int each = (end - begin + kWaves - 1) / kWaves;
    const int first = min(begin + wave * each, end), last = min(first + each, end);

    // This lane's row (rows behind the last repeat it).
    const Row r = row_of(p, x, min(ql, x.left - 1));
    Seen sl = seen_at(p, x.pos0 + r.t, x.len);
    sl.lo -= 4 * hh;
    sl.hi -= 4 * hh;
    sl.sk -= 4 * hh;
    bf16x8 qf[4];
    {
        const uint16_t *q = p.q + (hk * p.group + r.g) * p.qs.head + (int64_t)(x.cu + r.t) * p.qs.token + hh * 8;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) qf[kk] = *reinterpret_cast<const bf16x8 *>(q + kk * 16);
    }
    const uint16_t *kb = p.k + hk * p.ks.head, *vb = p.v + hk * p.vs.head;
    const int32_t *table = p.tables + (int64_t)x.b * p.table_stride;

    // The page of key `lane` of tile i, -1 where no row sees it.
    auto page_of = [&](int i) __attribute__((always_inline)) {
        if (i >= last) return -1;
        const int key = tl.key(i) + lane;
        return key < sb.sk || (key >= sa.lo && key < sb.hi) ? table[p.pages(key)] : -1;
    };
    // Starts the loads of tile i, whose keys' pages are known; the keys that are read.
    auto fetch = [&](int i, int page, bf16x8 (&k)[2][4], unsigned char *slot) __attribute__((always_inline)) -> uint64_t {
        if (i >= last) return 0;
        const int key = tl.key(i) + lane, row = key - p.pages(key) * p.page;
        const bool good = (unsigned int)page < (unsigned int)p.n_pages;
        page = good ? page : -1;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int from = u * 32 + ql, pg = __shfl(page, from), rw = __shfl(row, from);
            const uint16_t *src = pg < 0 ? zero_row : kb + pg * p.ks.page + rw * p.ks.token;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) k[u][kk] = *reinterpret_cast<const bf16x8 *>(src + hh * 8 + kk * 16);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int from = u * 8 + (lane >> 3), pg = __shfl(page, from), rw = __shfl(row, from);
            const uint16_t *src = pg < 0 ? zero_row : vb + pg * p.vs.page + rw * p.vs.token;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(src + (((lane & 7) ^ swz(from)) << 3)),
                                             (lds_void *)(slot + u * 1024), 16, 0, 0);
        }
        return __ballot(good);
    };

    const Reader rd(lane);
    const float c = p.scale_log2;
    float m = kNone, sum = 0.f;
    f32x16 acc[2];
#pragma unroll
    for (int dh = 0; dh < 2; ++dh)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[dh][v] = 0.f;
    int i = first, page = -1;
    uint64_t keys = 0;  // of tile i
    auto step = [&](const bf16x8 (&k)[2][4], const unsigned char *vt, bf16x8 (&kn)[2][4], unsigned char *vn)
                    __attribute__((always_inline)) -> bool {
        const uint64_t next = fetch(i + 1, page, kn, vn);
        page = page_of(i + 2);
        const int key0 = tl.key(i);
        const bool part = !(key0 + kTile <= sa.sk || (key0 >= sb.lo && key0 + kTile <= sa.hi));
        f32x16 s[2];
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int v = 0; v < 16; ++v) s[u][v] = 0.f;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) s[u] = mfma(k[u][kk], qf[kk], s[u]);
            if (part) hide(s[u], key0 + u * 32, sl.lo, (unsigned int)(sl.hi - sl.lo), key0 < sb.sk, sl.sk);
            if (keys != ~(uint64_t)0) drop(s[u], (unsigned int)(keys >> (32 * u)) >> (4 * hh));
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
        __builtin_amdgcn_s_waitcnt(0x0070);  // the next tile's loads, and this one's reads of its slot
        asm volatile("" ::: "memory");
        keys = next;
        return ++i < last;
    };
    if (i < last) {
        unsigned char *const a = v_0 + wave * kTileBytes, *const z = v_1 + wave * kTileBytes;
        bf16x8 ka[2][4], kz[2][4];
        keys = fetch(i, page_of(i), ka, a);
        page = page_of(i + 1);
        __builtin_amdgcn_s_waitcnt(0x0070);
        asm volatile("" ::: "memory");
        while (step(ka, a, kz, z) && step(kz, z, ka, a)) {
        }
    }
    sum += __shfl_xor(sum, 32);
    __syncthreads();  // (slots of other waves become parts)
    auto part_of = [&](int w) __attribute__((always_inline)) -> float * {
        return reinterpret_cast<float *>(w < 2 ? v_0 : v_1) + (w & 1) * kPart * kStep;
    };
    {
        float *d = part_of(wave) + ql;
        if (hh == 0) d[0] = m, d[kStep] = sum;
#pragma unroll
        for (int dh = 0; dh < 2; ++dh)
#pragma unroll
            for (int v = 0; v < 16; ++v) d[(2 + dh * 32 + (v >> 2) * 8 + hh * 4 + (v & 3)) * kStep] = acc[dh][v];
    }
    __syncthreads();
    for (int j = wave; j < x.left; j += kWaves) {
        float top = kNone, l = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, part_of(w)[j]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float a = __builtin_amdgcn_exp2f((part_of(w)[j] - top) * c);
            l = fmaf(part_of(w)[kStep + j], a, l);
            o = fmaf(part_of(w)[(2 + lane) * kStep + j], a, o);
        }
        const Row row = row_of(p, x, j);
        const int hq = hk * p.group + row.g;
        const int64_t at = (int64_t)hq * p.N + x.cu + row.t;
        if (cuts == 1) {
            p.o[hq * p.os.head + (int64_t)(x.cu + row.t) * p.os.token + lane] = (uint16_t)bf16_bits(l == 0.f ? 0.f : o / l);
            if (p.lse && lane == 0) p.lse[at] = l == 0.f ? -INFINITY : top * p.scale + logf(l);
        } else {
            const int64_t to = (int64_t)split * p.H * p.N + at;
            p.part[to * 64 + lane] = o;
            if (lane == 0) p.part_row[to] = make_float2(top, l);
        }
        if (p.splits > 1 && split == 0 && lane == 0) p.cuts[at] = cuts;
    }
}

// Where every sequence's blocks of `rows` rows begin, and how many blocks there are: one workgroup.
constexpr int kStartThreads = 1024;
__global__ void __launch_bounds__(kStartThreads) starts_kernel(const PagedParams p, int rows)
{
    __shared__ int ends[kStartThreads / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int before = 0;
    for (int b0 = 0; b0 < p.B; b0 += kStartThreads) {
        const int b = b0 + threadIdx.x;
        const Rows r = b < p.B ? rows_of(p, p.cu_q[b], p.cu_q[b + 1]) : Rows{0, 0};
        const int own = rows == kRows ? r.blocks<kRows>(p) : r.blocks<128>(p);
        const int sum = scan_wave(own, sum_of);
        if (lane == 63) ends[wave] = sum;
        __syncthreads();
        int start = min(before + (sum - own), kMostBlocks);
        for (int w = 0; w < kStartThreads / 64; ++w) {
            if (w < wave) start = min(start + ends[w], kMostBlocks);
            before = min(before + ends[w], kMostBlocks);
        }
        if (b < p.B) p.starts[b] = start;
        __syncthreads();
    }
    if (threadIdx.x == 0) p.starts[p.B] = before;
}

// A row by W waves, a channel a lane, 16 parts a wave: all of a wave's parts are on their way at once, their weights one
// a lane first; the waves' sums are added in order. Rows outside every sequence, and those that one workgroup
// finished, are left as they are. (What a row does not have of p.splits parts may hold anything.)
constexpr int kParts = 16;
template <int W>
__global__ void __launch_bounds__(256) join_kernel(const PagedParams p)
{
    __shared__ float tops[4], sums[4], outs[4][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, first = W > 1 ? wave * kParts : 0;
    const int64_t rows = (int64_t)p.H * p.N, row = W > 1 ? blockIdx.x : (int64_t)blockIdx.x * 4 + wave;
    if (row >= rows) return;
    const int64_t h = row / p.N, t = row - h * p.N;
    const int from = p.cu_q[0], to = p.cu_q[p.B], cuts = p.cuts[row];
    // (Few rows: their parts are on their way before it is known how many there are. Many: no more are read than there are.)
    if (W == 1 && (t < from || t >= to || cuts <= 1)) return;
    float y[kParts];
    float2 r = make_float2(kNone, 0.f);
    const int most = (W == 1 ? min(cuts, p.splits) : p.splits) - first;
    if (lane < kParts && lane < most) r = p.part_row[(first + lane) * rows + row];
#pragma unroll
    for (int s0 = 0; s0 < kParts; s0 += 2)
        if (s0 < most)
#pragma unroll
            for (int s = s0; s < s0 + 2; ++s) y[s] = p.part[(first + min(s, most - 1)) * rows * 64 + row * 64 + lane];
    if (t < from || t >= to || cuts <= 1) return;
    const int n = min(cuts, p.splits) - first;
    if (lane >= n) r = make_float2(kNone, 0.f);
    float top = r.y == 0.f ? kNone : r.x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    if constexpr (W > 1) {
        if (lane == 0) tops[wave] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) top = fmaxf(top, tops[w]);
    }
    const float w = r.y == 0.f ? 0.f : __builtin_amdgcn_exp2f((r.x - top) * p.scale_log2);
    float sum = w == 0.f ? 0.f : r.y * w, o = 0.f;
#pragma unroll
    for (int e = 1; e < 64; e <<= 1) sum += __shfl_xor(sum, e);
#pragma unroll
    for (int s = 0; s < kParts; ++s)
        if (s < n)
            o = fmaf(__builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), s)), y[s], o);
    if constexpr (W > 1) {
        outs[wave][lane] = o;
        if (lane == 0) sums[wave] = sum;
        __syncthreads();
        if (wave > 0) return;
        sum = o = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) sum += sums[i], o += outs[i][lane];
    }
    p.o[h * p.os.head + t * p.os.token + lane] = (uint16_t)bf16_bits(sum == 0.f ? 0.f : o / sum);
    if (p.lse && lane == 0)
        p.lse[row] = sum == 0.f ? -INFINITY : top * p.scale + logf(sum);
}

}  // namespace

hipError_t launch_paged(const PagedParams &p, int rows, hipStream_t s)
{
    static_assert(kMaxPagedSplits <= 4 * kParts, "four waves hold a row's parts");
    if (p.starts) {
        hipLaunchKernelGGL(starts_kernel, dim3(1), dim3(kStartThreads), 0, s, p, rows);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (rows == 128) return launch_paged_wide(p, s);
    // Parts of all blocks: a block's share of kTileParts, rounded, and at least one. Heads first, so that workgroups without a part come
    // last: between the others each left a CU with two and one with none (one token over 43,961 keys 17.5 us, so 14). (Blocks that
    // are not cut lie head by head; those of rows that pad a batch are behind each head's.)
    const unsigned H_kv = (unsigned)p.H_kv;
    hipLaunchKernelGGL(tile_kernel, p.splits > 1 ? dim3(H_kv, (unsigned)p.parts) : dim3((unsigned)p.blocks, H_kv), dim3(64 * kWaves), 0, s, p);
    if (hipError_t e = hipGetLastError()) return e;
    if (p.splits == 1) return hipSuccess;
    const int64_t all = (int64_t)p.H * p.N;
    if (p.splits <= kParts)
        hipLaunchKernelGGL((join_kernel<1>), dim3((unsigned)((all + 3) / 4)), dim3(256), 0, s, p);
    else
        hipLaunchKernelGGL((join_kernel<4>), dim3((unsigned)all), dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace ress
