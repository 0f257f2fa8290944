// Attention of new tokens over pages, blocks of 128 rows.
//
// A workgroup owns 128 rows (new token, query head of a K/V head) of a sequence, a wave 32 of them, and walks over
// the 64-key tiles that any of them sees, as window.hip's does: score tiles S^T = K Q^T, probabilities
// that are the next product's operand as they lie, one softmax reference a row that moves only when a
// tile's sum passes 2^50. What differs is where keys come from. A wave keeps 64 entries of the table in a
// register, one a lane; its 8 rows of a load lie in one page where pages are multiples of 8 tokens, so
// that their address is scalar and costs the vector unit one read of a lane (found anew for every tile by each of
// its keys, pages took a fifth more vector instructions). Other pages, and tiles that are not seen whole, take an
// address a lane. Keys on a page
// outside the cache, and keys that no row of the block sees, come from a row of zeros, their scores hidden.
//
// Measured: 8 sequences of four new frames each over a window of 3 and the first, 16 heads, 1,031 to 1,069 us, 806 to 836 TFLOP/s by the
// formula: bound by issue slots, the matrix unit busy 40% of the cycles, the vector unit 58%, its clock lower the busier both are. A
// frame over 31, cut into 14 parts and with the logarithm, 332 us and the join 16. 24 ragged sequences 77 to 81 us and the join 11: 408
// blocks in one to three parts by their sequences' lengths, 1,052 in all, most of 22 tiles, for 1,024 places, so the last ones
// run in a nearly empty chip (matrix unit busy 30%).
#include "paged_device.h"

namespace ress {
namespace {

using namespace paged;

constexpr int kRows = 128;
constexpr int kRun = 8;
constexpr float kSumLimit = 0x1p50f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float inverse(float sum) { return sum == 0.f ? 0.f : 1.f / sum; }

// The sum of 16 values, in pairs.
__device__ __forceinline__ float add_pairs(const f32x16 &x)
{
    float y[8];
#pragma unroll
    for (int v = 0; v < 8; ++v) y[v] = x[2 * v] + x[2 * v + 1];
#pragma unroll
    for (int n = 4; n > 0; n /= 2)
#pragma unroll
        for (int v = 0; v < n; ++v) y[v] = y[2 * v] + y[2 * v + 1];
    return y[0];
}

typedef const __attribute__((address_space(1))) void global_void;

// Eight rows from one on: at most 7 token strides of 2^22 elements and a row.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_at(const unsigned char *row)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(row), 0, 7 * (1 << 23) + 128, 0x00020000);
}

template <bool LSE>
__global__ void __launch_bounds__(256, 4) wide_kernel(const PagedParams p)
{
    __shared__ __attribute__((aligned(1024))) unsigned char k_0[kTileBytes], k_1[kTileBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char v_0[kTileBytes], v_1[kTileBytes];

    // Runs of kRun blocks or parts of a K/V head, which see about the same keys, to the XCDs in turn, heads first, the last ones first.
    // Where keys are cut that is from the last part found, and workgroups that have nothing come last; else from the host's bound of
    // blocks on, and those of rows that pad a batch come first and end at once (8 prompts of 2,000 tokens, 16 heads, in 16,000 /
    // 32,000 / 64,000 rows: 399 / 397 / 407 us). (An eighth of them all to each XCD, empty ones among them: 24 prompts of 30 to
    // 6,000 tokens on a log scale, 8 heads for 2, 288 us, so 149; of equal ones 1,183 and 1,205. Runs of 4 / 8 / 16 / 32: 148 / 149
    // / 152 / 163.)
    const int id = blockIdx.x + gridDim.x * blockIdx.y, turn = id >> 3, run = turn / kRun * 8 + (id & 7);
    const int hk = run % p.H_kv;
    auto pick = [&](int n) __attribute__((always_inline)) { return n - 1 - (run / p.H_kv * kRun + turn % kRun); };
    Part part;
    part.split = 0, part.cuts = 1;
    if (p.splits > 1) {
        if (!find_part<kRows, true>(p, [&](int n) __attribute__((always_inline)) { return pick(min(n, p.parts)); }, part)) return;
    } else {
        const int block = pick(p.blocks);
        if (block < 0 || !find_block<kRows>(p, block, part.x)) return;
    }
    const Block &x = part.x;
    const int split = part.split, cuts = part.cuts;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hh = lane >> 5, ql = lane & 31;

    const Seen s_first = seen_at(p, x.pos0 + x.t0, x.len), s_last = seen_at(p, x.pos0 + row_of(p, x, x.left - 1).t, x.len);
    const Tiles tl = tiles_of(s_first, s_last);
    const int begin = (int)((int64_t)tl.n * split / cuts), end = (int)((int64_t)tl.n * (split + 1) / cuts);

    // What the wave's rows and this lane's row see (rows behind the last repeat it), the lane's against its first key
    // of a tile.
    const int j = min(wave * 32 + ql, x.left - 1);
    const Row r = row_of(p, x, j);
    const Seen sa = seen_at(p, x.pos0 + row_of(p, x, min(wave * 32, x.left - 1)).t, x.len);
    const Seen sb = seen_at(p, x.pos0 + row_of(p, x, min(wave * 32 + 31, x.left - 1)).t, x.len);
    Seen sl = seen_at(p, x.pos0 + r.t, x.len);
    sl.lo -= 4 * hh;
    sl.hi -= 4 * hh;
    sl.sk -= 4 * hh;
    const bool active = wave * 32 < x.left;

    bf16x8 qf[4];
    {
        const uint16_t *q = p.q + (hk * p.group + r.g) * p.qs.head + (int64_t)(x.cu + r.t) * p.qs.token + hh * 8;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) qf[kk] = *reinterpret_cast<const bf16x8 *>(q + kk * 16);
    }
    const uint16_t *const kb = p.k + hk * p.ks.head, *const vb = p.v + hk * p.vs.head;
    const int32_t *const table = p.tables + (int64_t)x.b * p.table_stride;
    // This lane's share of a load of 8 rows: bytes from the first one on.
    const unsigned int chunk = (unsigned int)(((lane & 7) ^ swz(wave * 8 + (lane >> 3))) << 4);
    const unsigned int k_off = (unsigned int)(lane >> 3) * (unsigned int)(2 * p.ks.token) + chunk;
    const unsigned int v_off = (unsigned int)(lane >> 3) * (unsigned int)(2 * p.vs.token) + chunk;

    // Entries base .. base + 63 of the table, one a lane, and which of them are pages of the cache.
    int entries = -1, base = -64;
    uint64_t there = 0;
    // Starts the loads of tile i; the keys that are read.
    auto fetch = [&](int i, unsigned char *kd, unsigned char *vd) __attribute__((always_inline)) -> uint64_t {
        if (i >= end) return 0;
        const int key0 = tl.key(i), e0 = p.pages(key0), e1 = min(p.pages(key0 + kTile - 1), p.max_pages - 1);
        if (e0 < base || e1 >= base + 64) {
            base = e0;
            entries = table[min(base + lane, p.max_pages - 1)];
            there = __ballot((unsigned int)entries < (unsigned int)p.n_pages);
        }
        const uint64_t need = ~(uint64_t)0 >> (63 - (e1 - e0));
        const bool whole = key0 + kTile <= s_last.sk || (key0 >= s_first.lo && key0 + kTile <= s_last.hi);
        if (p.eights && whole && (there >> (e0 - base) & need) == need) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int key = key0 + wave * 8 + 32 * u, e = p.pages(key), rw = key - e * p.page;
                const int pg = __builtin_amdgcn_readlane(entries, e - base);
                const uint64_t ko = ((uint64_t)(uint32_t)pg * p.k_page16 + (uint32_t)rw * p.k_token16) << 4;
                const uint64_t vo = p.alike ? ko : ((uint64_t)(uint32_t)pg * p.v_page16 + (uint32_t)rw * p.v_token16) << 4;
                const __amdgpu_buffer_rsrc_t kr = rows_at((const unsigned char *)kb + ko), vr = rows_at((const unsigned char *)vb + vo);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, (lds_void *)(kd + (u * 4 + wave) * 1024), 16, k_off, 0, 0, 0);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, (lds_void *)(vd + (u * 4 + wave) * 1024), 16, v_off, 0, 0, 0);
            }
            return ~(uint64_t)0;
        }
        const int key = key0 + lane, e = p.pages(key), row = key - e * p.page;
        int page = __shfl(entries, e - base);
        const bool seen = key < s_last.sk || (key >= s_first.lo && key < s_last.hi);
        const bool good = seen && (unsigned int)page < (unsigned int)p.n_pages;
        page = good ? page : -1;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int from = wave * 8 + 32 * u + (lane >> 3), pg = __shfl(page, from), rw = __shfl(row, from);
            const uint16_t *kr = pg < 0 ? zero_row : kb + pg * p.ks.page + rw * p.ks.token;
            const uint16_t *vr = pg < 0 ? zero_row : vb + pg * p.vs.page + rw * p.vs.token;
            __builtin_amdgcn_global_load_lds((global_void *)((const unsigned char *)kr + chunk),
                                             (lds_void *)(kd + (u * 4 + wave) * 1024), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((global_void *)((const unsigned char *)vr + chunk),
                                             (lds_void *)(vd + (u * 4 + wave) * 1024), 16, 0, 0);
        }
        return __ballot(good);
    };

    const Reader rd(lane);
    const References refs = p.refs;
    // Reference, and the lane's halves of the row's sums: of weights as they enter the product with V, so that those sum to one,
    // and (LSE) before they are rounded. (With the second alone a frame over 31 took 331 us for 348, but values
    // that are all alike came out off by up to 2^-8 of themselves.)
    float ref = 0.f, sum = 0.f, mass = 0.f;
    bool has = false;            // the row has a reference
    f32x16 acc[2];
#pragma unroll
    for (int dh = 0; dh < 2; ++dh)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[dh][v] = 0.f;

    // Scores of rows 32 u .. of a tile; `part`: of the keys that the lane's row sees, else -inf.
    auto scores = [&](bool part, uint64_t keys, const unsigned char *kt, int u, int key0, f32x16 &s) __attribute__((always_inline)) {
#pragma unroll
        for (int v = 0; v < 16; ++v) s[v] = 0.f;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) s = mfma(rd.rows(kt, u, kk), qf[kk], s);
        if (part) {
            hide(s, key0 + u * 32, sl.lo, (unsigned int)(sl.hi - sl.lo), key0 < sb.sk, sl.sk);
            if (keys != ~(uint64_t)0) drop(s, (unsigned int)(keys >> (32 * u)) >> (4 * hh));
        }
    };
    // The row's largest score in the tile, as a reference.
    auto top = [&](bool part, uint64_t keys, const unsigned char *kt, int key0) __attribute__((always_inline)) {
        float m = -INFINITY;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f32x16 s;
            scores(part, keys, kt, u, key0, s);
#pragma unroll
            for (int v = 0; v < 16; ++v) m = fmaxf(m, s[v]);
        }
        return refs.of(fmaxf(m, __shfl_xor(m, 32)));
    };
    // Probabilities against the row's reference, and the lane's part of their sum, rounded (returned) and as they are. (any_far:
    // some rows' references may be far.)
    auto probs = [&](bool any_far, bool part, uint64_t keys, const unsigned char *kt, int key0, bf16x8 (&pb)[2][2], float &exact)
                     __attribute__((always_inline)) {
        float l = 0.f;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f32x16 s;
            scores(part, keys, kt, u, key0, s);
            if (any_far) {
                const bool far = refs.far(ref);
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    s[v] = __builtin_amdgcn_exp2f(far ? fmaf(s[v], refs.unit, -ref) * refs.rest : fmaf(s[v], refs.scale, -ref));
            } else {
#pragma unroll
                for (int v = 0; v < 16; ++v) s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], refs.scale, -ref));
            }
            pack(s, pb[u]);
            l = add_up(pb[u], l);
            if constexpr (LSE) {
                exact = u == 0 ? add_pairs(s) : exact + add_pairs(s);
                __builtin_amdgcn_sched_barrier(0);  // (else both halves' float32 values are held: spills)
            }
        }
        return l;
    };
    auto tile = [&](bool part, uint64_t keys, const unsigned char *kt, const unsigned char *vt, int key0)
                    __attribute__((always_inline)) {
        bf16x8 pb[2][2];
        float l, exact = 0.f;
        // (Rare: a row's first tile, or logits far above those so far. Lanes l and l^32 share the
        // row and decide together.)
        bool look = __any(!has), over = false;
#pragma nounroll
        for (bool again = false;; again = true) {
            if (look) {
                const float m = top(part, keys, kt, key0);
                if (has ? over : m > -INFINITY) {
                    const float to = has ? fmaxf(ref, m) : m;
                    const float a = has ? __builtin_amdgcn_exp2f(refs.difference(ref, to)) : 0.f;
                    sum *= a;
                    mass *= a;
#pragma unroll
                    for (int dh = 0; dh < 2; ++dh)
#pragma unroll
                        for (int v = 0; v < 16; ++v) acc[dh][v] *= a;
                    ref = to;
                    has = true;
                }
            }
            l = probs(false, part, keys, kt, key0, pb, exact);
            over = !(l <= kSumLimit);
            const bool far = refs.far(ref);
            if (!__any(over || far)) break;
            if (__any(far)) {
                asm volatile("" ::: "memory");  // (code of its own: the ordinary form stays in one piece)
                l = probs(true, part, keys, kt, key0, pb, exact);
                over = !(l <= kSumLimit);
            }
            look = __any(over);
            if (!look || again) break;
            over = ((int)over | __shfl_xor((int)over, 32)) != 0;
        }
        sum += l;
        mass += exact;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int dh = 0; dh < 2; ++dh) acc[dh] = mfma(rd.cols(vt, u, e, dh), pb[u][e], acc[dh]);
    };
    int i = begin;
    uint64_t keys = 0;  // of tile i
    // Tile i from (kt, vt), tile i + 1 on its way into the other slots.
    auto step = [&](const unsigned char *kt, const unsigned char *vt, unsigned char *kd, unsigned char *vd)
                    __attribute__((always_inline)) -> bool {
        const uint64_t next = fetch(i + 1, kd, vd);
        const int key0 = tl.key(i);
        if (active && (key0 < sb.sk || (key0 + kTile > sa.lo && key0 < sb.hi)) && keys != 0)
            tile(!(key0 + kTile <= sa.sk || (key0 >= sb.lo && key0 + kTile <= sa.hi)) || keys != ~(uint64_t)0, keys, kt, vt, key0);
        wait_vm_all();
        __syncthreads();
        keys = next;
        return ++i < end;
    };
    if (i < end) {
        keys = fetch(i, k_0, v_0);
        wait_vm_all();
        __syncthreads();
        while (step(k_0, v_0, k_1, v_1) && step(k_1, v_1, k_0, v_0)) {
        }
    }

    sum += __shfl_xor(sum, 32);
    if (LSE) mass += __shfl_xor(mass, 32);
    if (p.splits > 1 && split == 0 && hk == 0 && threadIdx.x == 0 && part.block < p.blocks) p.cut[part.block] = make_int4(part.first, part.step, cuts, 0);
    if (cuts > 1) {
        // A part as the lanes hold it: whole lines, read back by wide_join_kernel the same way. (By rows they were written and read
        // in pieces of 32 bytes: 512 blocks cut in three 86 us, so 77.)
        const int64_t at = (int64_t)hk * p.parts + part.first + split * part.step;
        if constexpr (LSE) {
            // One sum goes with a part: the unrounded one, and the products as if its weights had that sum.
            const float f = sum == 0.f ? 0.f : mass / sum;
#pragma unroll
            for (int dh = 0; dh < 2; ++dh)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[dh][v] *= f;
            sum = sum == 0.f ? 0.f : mass;
        }
#pragma unroll
        for (int v = 0; v < 8; ++v)
            *reinterpret_cast<f32x4 *>(p.part + (at * 4 + wave) * 2048 + v * 256 + lane * 4) =
                f32x4{acc[v >> 2][(v & 3) * 4], acc[v >> 2][(v & 3) * 4 + 1], acc[v >> 2][(v & 3) * 4 + 2], acc[v >> 2][(v & 3) * 4 + 3]};
        if (hh == 0) p.part_row[at * kRows + wave * 32 + ql] = make_float2(ref, sum);
        return;
    }
    if (wave * 32 + ql >= x.left) return;
    const int h = hk * p.group + r.g;
    store_row(p.o + h * p.os.head + (int64_t)(x.cu + r.t) * p.os.token, acc, inverse(sum), hh);
    if (LSE && hh == 0) p.lse[(int64_t)h * p.N + x.cu + r.t] = sum == 0.f ? -INFINITY : refs.base2(ref) * kLn2 + logf(mass);
}

// A quarter of the channels of a block whose keys were split, laid out as wide_kernel's: its parts in order, 8 of them on their
// way at once.
__global__ void __launch_bounds__(256) wide_join_kernel(const PagedParams p)
{
    const int id = blockIdx.x + gridDim.x * blockIdx.y;
    if (id >= p.H_kv * p.blocks) return;
    const int hk = id / p.blocks, block = id - hk * p.blocks, quad0 = blockIdx.z * 2;
    const int4 cut = p.cut[block];
    Block x;
    if (!find_block<kRows>(p, block, x)) return;
    const int n = min(cut.z, p.splits);
    if (n <= 1) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, hh = lane >> 5, ql = lane & 31;
    const References refs = p.refs;
    // (Clamped: where offsets descend, nothing wrote it.)
    const int first = min(max(cut.x, 0), p.parts - 1), step = min(max(cut.y, 0), p.parts);
    const float2 *rows = p.part_row + (int64_t)hk * p.parts * kRows + wave * 32 + ql;
    const float *from = p.part + ((int64_t)hk * p.parts * 4 + wave) * 2048 + quad0 * 256 + lane * 4;
    float top = -INFINITY, sum = 0.f;
    f32x4 o[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    for (int s0 = 0; s0 < n; s0 += 8) {
        float2 r[8];
        f32x4 y[8][2];
#pragma unroll
        for (int s = 0; s < 8; s += 2)
            if (s0 + s < n)
#pragma unroll
                for (int e = s; e < s + 2; ++e) {
                    const int64_t at = min(first + min(s0 + e, n - 1) * step, p.parts - 1);
                    r[e] = rows[at * kRows];
                    if (s0 + e >= n) r[e].y = 0.f;
                    y[e][0] = *reinterpret_cast<const f32x4 *>(from + at * 8192);
                    y[e][1] = *reinterpret_cast<const f32x4 *>(from + at * 8192 + 256);
                }
        // (Parts without mass have none of the row's references.)
        float to = top;
#pragma unroll
        for (int s = 0; s < 8; ++s)
            if (s0 + (s & ~1) < n && r[s].y != 0.f) to = fmaxf(to, r[s].x);
        const float a = sum == 0.f ? 0.f : __builtin_amdgcn_exp2f(refs.difference(top, to));
        sum *= a;
        o[0] *= a;
        o[1] *= a;
#pragma unroll
        for (int s = 0; s < 8; ++s)
            if (s0 + (s & ~1) < n) {
                const float w = r[s].y == 0.f ? 0.f : __builtin_amdgcn_exp2f(refs.difference(r[s].x, to));
                sum = fmaf(r[s].y, w, sum);
#pragma unroll
                for (int q = 0; q < 2; ++q)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[q][e] = fmaf(y[s][q][e], w, o[q][e]);
            }
        top = to;
    }
    if (wave * 32 + ql >= x.left) return;
    const Row r = row_of(p, x, wave * 32 + ql);
    const int h = hk * p.group + r.g;
    const float f = inverse(sum);
    uint16_t *row = p.o + h * p.os.head + (int64_t)(x.cu + r.t) * p.os.token + hh * 4;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const unsigned int lo = bf16_bits(o[q][0] * f) | bf16_bits(o[q][1] * f) << 16, hi = bf16_bits(o[q][2] * f) | bf16_bits(o[q][3] * f) << 16;
        *reinterpret_cast<uint2 *>(row + (quad0 + q) * 8) = make_uint2(lo, hi);
    }
    if (p.lse && quad0 == 0 && hh == 0)
        p.lse[(int64_t)h * p.N + x.cu + r.t] = sum == 0.f ? -INFINITY : refs.base2(top) * kLn2 + logf(sum);
}

}  // namespace

hipError_t launch_paged_wide(const PagedParams &p, hipStream_t s)
{
    // (A grid's threads in one dimension stay below 2^32.)
    auto grid_of = [](int64_t ids) {
        const unsigned wide = ids < (1 << 20) ? (unsigned)ids : 1u << 20;
        return dim3(wide, (unsigned)((ids + wide - 1) / wide));
    };
    const int64_t blocks = (int64_t)p.H_kv * p.blocks, runs = (int64_t)((p.splits > 1 ? p.parts : p.blocks) + kRun - 1) / kRun * p.H_kv;
    const dim3 grid = grid_of((runs + 7) / 8 * 8 * kRun), block(256);
    if (p.lse)
        hipLaunchKernelGGL((wide_kernel<true>), grid, block, 0, s, p);
    else
        hipLaunchKernelGGL((wide_kernel<false>), grid, block, 0, s, p);
    if (hipError_t e = hipGetLastError()) return e;
    if (p.splits == 1) return hipSuccess;
    const dim3 join = grid_of(blocks);
    hipLaunchKernelGGL(wide_join_kernel, dim3(join.x, join.y, 4), block, 0, s, p);
    return hipGetLastError();
}

}  // namespace ress
