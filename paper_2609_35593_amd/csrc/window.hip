// Attention over a sliding window of frames and the first tokens (sinks).
//
// A workgroup owns 128 queries of a head, a wave 32 of them, and walks over the 64-key
// tiles that any of its queries sees: those of the sinks, then those of the window, in
// ascending order and each once. The score tile is formed transposed, S^T = K Q^T (see
// tiles.h), so a lane holds one query's scores, its softmax needs one exchange (with lane
// l^32, which holds the other half of the keys), and the probabilities are the next
// product's operand as they lie. A wave masks only the tiles that some of its queries see
// in part, by a comparison a score against its lane's range (two among sinks), and passes
// over those that none sees.
//
// Small calls: a wave's tiles come one after the other, and a chip of 1,024 SIMDs wants more
// waves than there are rows. With G > 1 a workgroup's waves split into G groups over the same
// 128 / G queries, group g with LDS slots of its own taking tiles g, g + G, ...; and a block's
// tiles are cut over `splits` workgroups, whose partial results join_kernel adds up. Both
// joins take the parts in order.
//
// Bound by issue slots beside the matrix unit: 16 heads of 32 frames of 1,374 tokens, window 4 and
// a frame of sinks, 1,239-1,300 us (892-936 TFLOP/s, 75-78% of a large library product's rate; matrix unit
// busy 48% of the cycles, vector unit 62%; no bank conflicts). 10,001 tokens, window 1,024, 16 heads
// for 4: 67-77 us, of which some 25 are the last fifth of a filling (1,264 workgroups for 1,024 places).
//
// Softmax: base 2, against a reference per row that is the row's largest logit in the
// first tile where it sees a key, and moves (O and the sum rescaled) only when a tile's
// sum exceeds 2^50; so a tile costs no maximum, float32 keeps every digit of the sum, and a
// row with a key has a sum of at least 1 against its first reference. The running sum is of
// the float32 probabilities where the logarithm is wanted, else of the bf16-rounded ones
// that the product with V takes (packed dot products, half the instructions). Those are rounded because
// the matrix unit takes bf16: outputs are 7e-4 to 1e-3 off in norm for it, up to 2e-3 where rows see few
// keys, beside 1.7e-3 by their own rounding; a second product for what is left of each weight, as
// decode affords, would make the products half again as many.
//
// A weight is exp2(s c - ref), one fma of the score s and its scale c against the scaled reference.
// That one is rounded, by up to half its step; all weights of a row see the same, and their quotient
// does not, but from 2^31 on half a step passes the 2^127 that float32 holds. So references of 2^24
// and more are kept as score times a power of two, exactly, and taken from the scores before the rest
// of the scale (References in layer_internal.h).
#include "tiles.h"

namespace ress {
namespace {

using namespace tiles;

constexpr float kSumLimit = 0x1p50f;
constexpr float kLn2 = 0.6931471805599453f;

// exp2(ref - top) for a part that holds mass, 0 for one that holds none.
__device__ __forceinline__ float share(const References &r, float ref, float sum, float top)
{
    return sum == 0.f ? 0.f : __builtin_amdgcn_exp2f(r.difference(ref, top));
}

__device__ __forceinline__ float inverse(float sum) { return sum == 0.f ? 0.f : 1.f / sum; }

template <bool LSE, int G>
__global__ void __launch_bounds__(256, G > 1 ? 2 : 4) window_kernel(const WindowParams p)
{
    constexpr int QW = 4 / G, ROWS = 32 * QW;  // waves and queries of a group
    // (Arrays of their own: of one array's parts the compiler does not see that a read of one
    // slot need not wait for the load into another.)
    __shared__ __attribute__((aligned(1024))) unsigned char k_a0[G * kTileBytes], k_a1[G * kTileBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char v_a0[G * kTileBytes], v_a1[G * kTileBytes];

    // Contiguous runs of (head, query block) per XCD, whose L2 then holds few heads'
    // windows; last blocks first (a causal row sees the more the later it is).
    const int rows = p.H * p.n_qb, per = (rows + 7) / 8;
    const int at = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || at >= rows) return;
    const int h = p.q_blocks(at), i = p.n_qb - 1 - (at - h * p.n_qb), hk = p.groups(h);
    const int lane = threadIdx.x & 63, wave_wg = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int grp = wave_wg / QW, wave = wave_wg % QW;
    const int hh = lane >> 5, ql = lane & 31;
    unsigned char *const k_0 = k_a0 + grp * kTileBytes, *const k_1 = k_a1 + grp * kTileBytes;
    unsigned char *const v_0 = v_a0 + grp * kTileBytes, *const v_1 = v_a1 + grp * kTileBytes;

    // The block's tiles: [0, ns) and [w0, w1); this workgroup's: from `begin`, tiles_n of them.
    const int t_first = i * ROWS, t_last = min(t_first + ROWS, p.n_q) - 1;
    const Seen s_first = seen_by(p, p.q_offset + t_first), s_last = seen_by(p, p.q_offset + t_last);
    const int ns = (s_last.sk + kTile - 1) / kTile;
    int w0 = s_first.lo / kTile, w1 = (s_last.hi + kTile - 1) / kTile;
    if (s_first.lo >= s_last.hi) w0 = w1 = ns;
    if (w0 < ns) w0 = ns;
    if (w1 < w0) w1 = w0;
    int begin = 0, tiles_n = ns + w1 - w0;
    if (p.splits > 1) {
        const int all = tiles_n, split = blockIdx.y;
        begin = (int)((int64_t)all * split / p.splits);
        tiles_n = (int)((int64_t)all * (split + 1) / p.splits) - begin;
    }
    // Key of the group's turn n.
    auto tile_key = [&](int n) __attribute__((always_inline)) {
        const int c = begin + n * G + grp;
        return (c < ns ? c : c - ns + w0) * kTile;
    };
    const int turns = (tiles_n + G - 1) / G;

    // What the wave's rows and this lane's row see (rows past the last repeat it), the lane's
    // against its first key of a tile.
    const int ta = min(t_first + wave * 32, t_last), tb = min(t_first + wave * 32 + 31, t_last);
    const Seen sa = seen_by(p, p.q_offset + ta), sb = seen_by(p, p.q_offset + tb);
    const int t = t_first + wave * 32 + ql, tq = min(t, t_last);
    Seen sl = seen_by(p, p.q_offset + tq);
    sl.lo -= 4 * hh;
    sl.hi -= 4 * hh;
    sl.sk -= 4 * hh;

    bf16x8 qf[4];
    {
        const uint16_t *q = p.q + h * p.qs.head + (int64_t)tq * p.qs.token + hh * 8;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) qf[kk] = *reinterpret_cast<const bf16x8 *>(q + kk * 16);
    }
    const Loader<QW> load_k(p.k + hk * p.ks.head, p.ks.token, wave, lane);
    const Loader<QW> load_v(p.v + hk * p.vs.head, p.vs.token, wave, lane);
    const Reader rd(lane);
    // Keys outside every row's sight are not read: only [0, sk) and [lo, hi) of the workgroup are.
    auto fetch = [&](int n, unsigned char *kd, unsigned char *vd) __attribute__((always_inline)) {
        if (n * G + grp >= tiles_n) return;
        const int key0 = tile_key(n);
        const bool sinks = key0 < s_last.sk, window = s_first.lo < s_last.hi && key0 + kTile > s_first.lo && key0 < s_last.hi;
        const int lo = sinks ? 0 : s_first.lo, hi = window ? max(s_last.hi, s_last.sk) : s_last.sk;
        const int end = sinks && window ? s_first.lo : 0;  // a tile of both: what lies between them
        load_k(key0, lo, hi, s_last.sk, end, kd);
        load_v(key0, lo, hi, s_last.sk, end, vd);
    };

    const References r = p.refs;
    float ref = 0.f, sum = 0.f;  // reference and the lane's half of the row's sum
    bool has = false;            // the row has a reference
    f32x16 acc[2];
#pragma unroll
    for (int dh = 0; dh < 2; ++dh)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[dh][v] = 0.f;

    // Scores of rows 32 u .. of a tile; `part`: of the keys that the lane's row sees, else -inf.
    auto scores = [&](bool part, const unsigned char *kt, int u, int key0, f32x16 &s) __attribute__((always_inline)) {
#pragma unroll
        for (int v = 0; v < 16; ++v) s[v] = 0.f;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) s = mfma(rd.rows(kt, u, kk), qf[kk], s);
        if (part) hide(s, key0 + u * 32, sl.lo, (unsigned int)(sl.hi - sl.lo), key0 < sb.sk, sl.sk);
    };
    // The row's largest score in the tile, as a reference.
    auto top = [&](bool part, const unsigned char *kt, int key0) __attribute__((always_inline)) {
        float m = -INFINITY;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f32x16 s;
            scores(part, kt, u, key0, s);
#pragma unroll
            for (int v = 0; v < 16; ++v) m = fmaxf(m, s[v]);
        }
        return r.of(fmaxf(m, __shfl_xor(m, 32)));
    };
    // Probabilities against the row's reference, and the lane's part of their sum. (any_far: some rows'
    // references may be far.)
    auto probs = [&](bool any_far, bool part, const unsigned char *kt, int key0, bf16x8 (&pb)[2][2])
                     __attribute__((always_inline)) {
        float l0 = 0.f, l1 = 0.f;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f32x16 s;
            scores(part, kt, u, key0, s);
            if (any_far) {
                const bool far = r.far(ref);
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    s[v] = __builtin_amdgcn_exp2f(far ? fmaf(s[v], r.unit, -ref) * r.rest : fmaf(s[v], r.scale, -ref));
            } else {
#pragma unroll
                for (int v = 0; v < 16; ++v) s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], r.scale, -ref));
            }
            pack(s, pb[u]);
            if constexpr (LSE) {
#pragma unroll
                for (int v = 0; v < 16; v += 2) l0 += s[v], l1 += s[v + 1];
                __builtin_amdgcn_sched_barrier(0);  // (else both halves' float32 values are held: spills)
            } else {
                l0 = add_up(pb[u], l0);
            }
        }
        return l0 + l1;
    };
    auto tile = [&](bool part, const unsigned char *kt, const unsigned char *vt, int key0) __attribute__((always_inline)) {
        bf16x8 pb[2][2];
        float l;
        // (Rare: a row's first tile, or logits far above those so far. Lanes l and l^32 share the
        // row and decide together.)
        bool look = __any(!has), over = false;
#pragma nounroll
        for (bool again = false;; again = true) {
            if (look) {
                const float m = top(part, kt, key0);
                if (has ? over : m > -INFINITY) {
                    const float to = has ? fmaxf(ref, m) : m;
                    const float a = has ? __builtin_amdgcn_exp2f(r.difference(ref, to)) : 0.f;
                    sum *= a;
#pragma unroll
                    for (int dh = 0; dh < 2; ++dh)
#pragma unroll
                        for (int v = 0; v < 16; ++v) acc[dh][v] *= a;
                    ref = to;
                    has = true;
                }
            }
            l = probs(false, part, kt, key0, pb);
            over = !(l <= kSumLimit);
            const bool far = r.far(ref);
            if (!__any(over || far)) break;
            if (__any(far)) {
                asm volatile("" ::: "memory");  // (code of its own: the ordinary form stays in one piece)
                l = probs(true, part, kt, key0, pb);
                over = !(l <= kSumLimit);
            }
            look = __any(over);
            if (!look || again) break;
            over = ((int)over | __shfl_xor((int)over, 32)) != 0;
        }
        sum += l;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int dh = 0; dh < 2; ++dh) acc[dh] = mfma(rd.cols(vt, u, e, dh), pb[u][e], acc[dh]);
    };
    int n = 0;
    // Turn n from (kt, vt), turn n + 1 on its way into the other slots. (Slots by name: with
    // addresses formed at run time every read takes an addition.)
    auto step = [&](const unsigned char *kt, const unsigned char *vt, unsigned char *kd, unsigned char *vd)
                    __attribute__((always_inline)) -> bool {
        const int key0 = tile_key(n);
        fetch(n + 1, kd, vd);
        if ((G == 1 || n * G + grp < tiles_n) && (key0 < sb.sk || (key0 + kTile > sa.lo && key0 < sb.hi)))
            tile(!(key0 + kTile <= sa.sk || (key0 >= sb.lo && key0 + kTile <= sa.hi)), kt, vt, key0);
        wait_vm_all();
        __syncthreads();
        return ++n < turns;
    };
    if (turns > 0) {
        fetch(0, k_0, v_0);
        wait_vm_all();
        __syncthreads();
        while (step(k_0, v_0, k_1, v_1) && step(k_1, v_1, k_0, v_0)) {
        }
    }

    sum += __shfl_xor(sum, 32);
    if constexpr (G > 1) {
        // The groups behind the first leave reference, sum and O in the slots (34 floats a lane).
        constexpr int PER = 34 * 64;
        constexpr int FIT = G * kTileBytes / (PER * 4);  // waves per slot array
        static_assert((G - 1) * QW <= 2 * FIT, "the joined parts fit the key slots");
        auto area = [&](int w) __attribute__((always_inline)) -> float * {
            return reinterpret_cast<float *>(w < FIT ? k_a0 : k_a1) + w % FIT * PER + lane;
        };
        if (grp > 0) {
            float *m = area((grp - 1) * QW + wave);
            m[0] = ref;
            m[64] = sum;
#pragma unroll
            for (int v = 0; v < 32; ++v) m[(2 + v) * 64] = acc[v >> 4][v & 15];
        }
        __syncthreads();
        if (grp > 0) return;
        float to = sum == 0.f ? -INFINITY : ref;
#pragma unroll
        for (int g = 1; g < G; ++g) {
            const float *m = area((g - 1) * QW + wave);
            if (m[64] != 0.f) to = fmaxf(to, m[0]);
        }
        const float a0 = share(r, ref, sum, to);
        sum *= a0;
#pragma unroll
        for (int v = 0; v < 32; ++v) acc[v >> 4][v & 15] *= a0;
#pragma unroll
        for (int g = 1; g < G; ++g) {
            const float *m = area((g - 1) * QW + wave);
            const float a = share(r, m[0], m[64], to);
            sum = fmaf(m[64], a, sum);
#pragma unroll
            for (int v = 0; v < 32; ++v) acc[v >> 4][v & 15] = fmaf(m[(2 + v) * 64], a, acc[v >> 4][v & 15]);
        }
        ref = to;
    }
    if (t > t_last) return;
    if (p.splits > 1) {
        const int64_t row = ((int64_t)blockIdx.y * p.H + h) * p.n_q + t;
#pragma unroll
        for (int dh = 0; dh < 2; ++dh)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4 *>(p.part + row * 64 + dh * 32 + g * 8 + hh * 4) =
                    f32x4{acc[dh][g * 4], acc[dh][g * 4 + 1], acc[dh][g * 4 + 2], acc[dh][g * 4 + 3]};
        if (hh == 0) p.part_row[row] = make_float2(ref, sum);
        return;
    }
    store_row(p.o + h * p.os.head + (int64_t)t * p.os.token, acc, inverse(sum), hh);
    if (LSE && hh == 0) p.lse[(int64_t)h * p.n_q + t] = sum == 0.f ? -INFINITY : r.base2(ref) * kLn2 + logf(sum);
}

// A wave a row, a channel a lane: its parts in order, their weights one a lane first. (All of them
// are on their way with their references: one round trip.)
__global__ void __launch_bounds__(256) join_kernel(const WindowParams p)
{
    const int64_t rows = (int64_t)p.H * p.n_q, row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= rows) return;
    const int lane = threadIdx.x & 63;
    float x[kMaxSplits];
    const float2 r = lane < p.splits ? p.part_row[lane * rows + row] : make_float2(0.f, 0.f);
#pragma unroll
    for (int s0 = 0; s0 < kMaxSplits; s0 += 4)
        if (s0 < p.splits)
#pragma unroll
            for (int s = s0; s < s0 + 4; ++s) x[s] = p.part[(min(s, p.splits - 1) * rows + row) * 64 + lane];
    float top = r.y == 0.f ? -INFINITY : r.x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float w = share(p.refs, r.x, r.y, top);
    float sum = w == 0.f ? 0.f : r.y * w, o = 0.f;
#pragma unroll
    for (int e = 1; e < 64; e <<= 1) sum += __shfl_xor(sum, e);
#pragma unroll
    for (int s = 0; s < kMaxSplits; ++s)
        if (s < p.splits)
            o = fmaf(__builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), s)), x[s], o);
    const int64_t h = row / p.n_q, t = row - h * p.n_q;
    p.o[h * p.os.head + t * p.os.token + lane] = (uint16_t)bf16_bits(o * inverse(sum));
    if (p.lse && lane == 0) p.lse[row] = sum == 0.f ? -INFINITY : p.refs.base2(top) * kLn2 + logf(sum);
}

template <int G>
hipError_t go(const WindowParams &p, hipStream_t s)
{
    const dim3 grid(8u * (unsigned)((p.H * p.n_qb + 7) / 8), (unsigned)p.splits), block(256);
    if (p.lse)
        hipLaunchKernelGGL((window_kernel<true, G>), grid, block, 0, s, p);
    else
        hipLaunchKernelGGL((window_kernel<false, G>), grid, block, 0, s, p);
    if (hipError_t e = hipGetLastError()) return e;
    if (p.splits > 1) {
        hipLaunchKernelGGL(join_kernel, dim3((unsigned)(((int64_t)p.H * p.n_q + 3) / 4)), block, 0, s, p);
        return hipGetLastError();
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_window(const WindowParams &p, int groups, hipStream_t s)
{
    return groups == 1 ? go<1>(p, s) : groups == 2 ? go<2>(p, s) : go<4>(p, s);
}

}  // namespace ress
