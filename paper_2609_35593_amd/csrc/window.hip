// Attention over a sliding window of frames and the first tokens (sinks).
//
// A workgroup owns 128 queries of a head, a wave 32 of them, and walks over the 64-key
// tiles that any of its queries sees: those of the sinks, then those of the window, in
// ascending order and each once. The score tile is formed transposed, S^T = K Q^T (see
// tiles.h), so a lane holds one query's scores, its softmax needs one exchange (with lane
// l^32, which holds the other half of the keys), and the probabilities are the next
// product's operand as they lie. A wave masks only the tiles that some of its queries see
// in part, by two comparisons a score against its lane's range, and passes over those
// that none sees.
//
// Softmax: base 2, against a reference per row that is the row's largest logit in the
// first tile where it sees a key, and moves (O and the sum rescaled) only when a tile's
// sum exceeds 2^50; so a tile costs no maximum, float32 keeps every digit of the sum, and a
// row with a key has a sum of at least 1 against its first reference. The running sum is of
// the float32 probabilities where the logarithm is wanted, else of the bf16-rounded ones
// that the product with V takes (packed dot products, half the instructions).
#include "tiles.h"

namespace ress {
namespace {

using namespace tiles;

constexpr float kSumLimit = 0x1p50f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

template <bool LSE>
__global__ void __launch_bounds__(256, LSE ? 3 : 4) window_kernel(const WindowParams p)
{
    __shared__ __attribute__((aligned(1024))) unsigned char k_0[kTileBytes], k_1[kTileBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char v_0[kTileBytes], v_1[kTileBytes];

    // Contiguous runs of (head, query block) per XCD, whose L2 then holds few heads'
    // windows; last blocks first (a causal row sees the more the later it is).
    const int rows = p.H * p.n_qb, per = (rows + 7) / 8;
    const int at = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || at >= rows) return;
    const int h = at / p.n_qb, i = p.n_qb - 1 - (at - h * p.n_qb);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hh = lane >> 5, ql = lane & 31;

    // The workgroup's tiles: [0, ns) and [w0, w1).
    const int t_first = i * 128, t_last = min(t_first + 128, p.n_q) - 1;
    const Seen s_first = seen_by(p, p.q_offset + t_first), s_last = seen_by(p, p.q_offset + t_last);
    const int ns = (s_last.sk + kTile - 1) / kTile;
    int w0 = s_first.lo / kTile, w1 = (s_last.hi + kTile - 1) / kTile;
    if (s_first.lo >= s_last.hi) w0 = w1 = ns;
    if (w0 < ns) w0 = ns;
    if (w1 < w0) w1 = w0;
    const int tiles_n = ns + w1 - w0;
    auto tile_key = [&](int c) __attribute__((always_inline)) { return (c < ns ? c : c - ns + w0) * kTile; };

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
    const Loader<4> load_k(p.k + (h / p.group) * p.ks.head, p.ks.token, wave, lane);
    const Loader<4> load_v(p.v + (h / p.group) * p.vs.head, p.vs.token, wave, lane);
    const Reader rd(lane);
    // Keys outside every row's sight are not read: [0, sk) and [lo, hi) of the workgroup.
    auto fetch = [&](int c, unsigned char *kd, unsigned char *vd) __attribute__((always_inline)) {
        const int key0 = tile_key(c);
        const bool sinks = key0 < s_last.sk, window = key0 + kTile > s_first.lo && key0 < s_last.hi;
        const int lo = sinks ? 0 : s_first.lo, hi = window ? max(s_last.hi, s_last.sk) : s_last.sk;
        load_k(key0, lo, hi, kd);
        load_v(key0, lo, hi, vd);
    };

    const float c = p.scale_log2;
    float ref = 0.f, sum = 0.f;  // reference (base 2) and the lane's half of the row's sum
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
        if (part) {
            asm volatile("" ::: "memory");  // (a real branch: whole tiles skip the comparisons)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int key = __builtin_amdgcn_readfirstlane(key0 + u * 32 + (v >> 2) * 8 + (v & 3));
                const bool in = (key >= sl.lo && key < sl.hi) || key < sl.sk;
                s[v] = in ? s[v] : -INFINITY;
            }
        }
    };
    // The row's largest logit in the tile.
    auto top = [&](bool part, const unsigned char *kt, int key0) __attribute__((always_inline)) {
        float m = -INFINITY;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f32x16 s;
            scores(part, kt, u, key0, s);
#pragma unroll
            for (int v = 0; v < 16; ++v) m = fmaxf(m, s[v]);
        }
        return fmaxf(m, __shfl_xor(m, 32)) * c;
    };
    // Probabilities against the row's reference, and the lane's part of their sum.
    auto probs = [&](bool part, const unsigned char *kt, int key0, bf16x8 (&pb)[2][2]) __attribute__((always_inline)) {
        float l0 = 0.f, l1 = 0.f;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f32x16 s;
            scores(part, kt, u, key0, s);
#pragma unroll
            for (int v = 0; v < 16; ++v) s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], c, -ref));
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
#pragma nounroll
        for (bool again = false;; again = true) {
            l = probs(part, kt, key0, pb);
            // (Lanes l and l^32 share the row and decide together.)
            const bool far = !(l <= kSumLimit);
            if (again || !__any(far || !has)) break;
            const bool row_far = ((int)far | __shfl_xor((int)far, 32)) != 0;
            const float m = top(part, kt, key0);
            if (has ? row_far : m > -INFINITY) {
                const float to = has ? fmaxf(ref, m) : m;
                const float a = has ? __builtin_amdgcn_exp2f(ref - to) : 0.f;
                sum *= a;
#pragma unroll
                for (int dh = 0; dh < 2; ++dh)
#pragma unroll
                    for (int v = 0; v < 16; ++v) acc[dh][v] *= a;
                ref = to;
                has = true;
            }
        }
        sum += l;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int dh = 0; dh < 2; ++dh) acc[dh] = mfma(rd.cols(vt, u, e, dh), pb[u][e], acc[dh]);
    };
    int ch = 0;
    // Tile ch from (kt, vt), tile ch + 1 on its way into the other slots. (Slots by name: with
    // addresses formed at run time every read takes an addition.)
    auto step = [&](const unsigned char *kt, const unsigned char *vt, unsigned char *kd, unsigned char *vd)
                    __attribute__((always_inline)) -> bool {
        const int key0 = tile_key(ch);
        if (ch + 1 < tiles_n) fetch(ch + 1, kd, vd);
        if (key0 < sb.sk || (key0 + kTile > sa.lo && key0 < sb.hi))
            tile(!(key0 + kTile <= sa.sk || (key0 >= sb.lo && key0 + kTile <= sa.hi)), kt, vt, key0);
        wait_vm_all();
        __syncthreads();
        return ++ch < tiles_n;
    };
    if (tiles_n > 0) {
        fetch(0, k_0, v_0);
        wait_vm_all();
        __syncthreads();
        while (step(k_0, v_0, k_1, v_1) && step(k_1, v_1, k_0, v_0)) {
        }
    }

    sum += __shfl_xor(sum, 32);
    if (t > t_last) return;
    store_row(p.o + h * p.os.head + (int64_t)t * p.os.token, acc, sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum), hh);
    if (LSE && hh == 0) p.lse[(int64_t)h * p.n_q + t] = sum == 0.f ? -INFINITY : ref * kLn2 + logf(sum);
}

}  // namespace

hipError_t launch_window(const WindowParams &p, hipStream_t s)
{
    const dim3 grid(8u * (unsigned)((p.H * p.n_qb + 7) / 8)), block(256);
    if (p.lse)
        hipLaunchKernelGGL(window_kernel<true>, grid, block, 0, s, p);
    else
        hipLaunchKernelGGL(window_kernel<false>, grid, block, 0, s, p);
    return hipGetLastError();
}

}  // namespace ress
