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
__global__ void __launch_bounds__(256, 4) window_kernel(const WindowParams p)
{
    __shared__ __attribute__((aligned(1024))) unsigned char k_s[2][kTileBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char v_s[2][kTileBytes];

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
    int ns = (s_last.sk + kTile - 1) / kTile;
    int w0 = s_first.lo / kTile, w1 = (s_last.hi + kTile - 1) / kTile;
    if (s_first.lo >= s_last.hi) w0 = w1 = ns;
    if (w0 < ns) w0 = ns;
    if (w1 < w0) w1 = w0;
    const int tiles_n = ns + w1 - w0;
    auto tile_key = [&](int c) __attribute__((always_inline)) { return (c < ns ? c : c - ns + w0) * kTile; };

    // What the wave's rows and this lane's row see (rows past the last repeat it).
    const int ta = min(t_first + wave * 32, t_last), tb = min(t_first + wave * 32 + 31, t_last);
    const Seen sa = seen_by(p, p.q_offset + ta), sb = seen_by(p, p.q_offset + tb);
    const int t = t_first + wave * 32 + ql, tq = min(t, t_last);
    const Seen sl = seen_by(p, p.q_offset + tq);

    bf16x8 qf[4];
    {
        const uint16_t *q = p.q + h * p.qs.head + (int64_t)tq * p.qs.token + hh * 8;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) qf[kk] = *reinterpret_cast<const bf16x8 *>(q + kk * 16);
    }
    const uint16_t *kh = p.k + (h / p.group) * p.ks.head, *vh = p.v + (h / p.group) * p.vs.head;
    const Loader<4> load(wave, lane);
    const Reader rd(lane);
    // Keys outside every row's sight are not read: [0, sk) and [lo, hi) of the workgroup.
    auto fetch = [&](int c, int slot) __attribute__((always_inline)) {
        const int key0 = tile_key(c);
        const bool sinks = key0 < s_last.sk, window = key0 + kTile > s_first.lo && key0 < s_last.hi;
        const int lo = sinks ? 0 : s_first.lo, hi = window ? max(s_last.hi, s_last.sk) : s_last.sk;
        load(kh, p.ks.token, key0, lo, hi, k_s[slot]);
        load(vh, p.vs.token, key0, lo, hi, v_s[slot]);
    };

    const float c = p.scale_log2;
    float ref = 0.f, sum = 0.f;  // reference (base 2) and the lane's half of the row's sum
    bool has = false;            // the row has a reference
    f32x16 acc[2];
#pragma unroll
    for (int dh = 0; dh < 2; ++dh)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[dh][v] = 0.f;
    const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};

    auto scores = [&](const unsigned char *kt, int u, int key0, bool part, f32x16 &s) __attribute__((always_inline)) {
#pragma unroll
        for (int v = 0; v < 16; ++v) s[v] = 0.f;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) s = mfma(rd.rows(kt, u, kk), qf[kk], s);
        if (part) {
            asm volatile("" ::: "memory");  // (a real branch: whole tiles skip the comparisons)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int key = key0 + u * 32 + (v >> 2) * 8 + (v & 3) + 4 * hh;
                const bool in = (key >= sl.lo && key < sl.hi) || key < sl.sk;
                s[v] = in ? s[v] : -INFINITY;
            }
        }
    };
    // The lane's half of the row's largest logit in the tile, with the other half's.
    auto top = [&](const unsigned char *kt, int key0, bool part) __attribute__((always_inline)) {
        float m = -INFINITY;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f32x16 s;
            scores(kt, u, key0, part, s);
#pragma unroll
            for (int v = 0; v < 16; ++v) m = fmaxf(m, s[v]);
        }
        return fmaxf(m, __shfl_xor(m, 32)) * c;
    };
    auto probs = [&](const unsigned char *kt, int key0, bool part, bf16x8 (&pb)[2][2]) __attribute__((always_inline)) {
        float l0 = 0.f, l1 = 0.f;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f32x16 s;
            scores(kt, u, key0, part, s);
#pragma unroll
            for (int v = 0; v < 16; ++v) s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], c, -ref));
            pack(s, pb[u]);
            if constexpr (LSE) {
#pragma unroll
                for (int v = 0; v < 16; v += 2) l0 += s[v], l1 += s[v + 1];
            } else {
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int j = 0; j < 8; j += 4) {
                        l0 = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{pb[u][e][j], pb[u][e][j + 1]}, ones, l0, false);
                        l1 = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{pb[u][e][j + 2], pb[u][e][j + 3]}, ones, l1, false);
                    }
            }
        }
        return l0 + l1;
    };

    if (tiles_n > 0) {
        fetch(0, 0);
        wait_vm_all();
        __syncthreads();
    }
    for (int ch = 0; ch < tiles_n; ++ch) {
        const int slot = ch & 1, key0 = tile_key(ch);
        if (ch + 1 < tiles_n) fetch(ch + 1, slot ^ 1);
        const bool none = key0 >= sb.sk && (key0 + kTile <= sa.lo || key0 >= sb.hi);
        if (!none) {
            const bool part = !(key0 + kTile <= sa.sk || (key0 >= sb.lo && key0 + kTile <= sa.hi));
            const unsigned char *kt = k_s[slot], *vt = v_s[slot];
            if (!__all(has)) {
                const float m = top(kt, key0, part);
                if (!has && m > -INFINITY) {
                    ref = m;
                    has = true;
                }
            }
            bf16x8 pb[2][2];
            float l = probs(kt, key0, part, pb);
            if (__any(!(l <= kSumLimit))) {
                const float m = top(kt, key0, part), to = fmaxf(ref, m);
                const float a = __builtin_amdgcn_exp2f(ref - to);
                sum *= a;
#pragma unroll
                for (int dh = 0; dh < 2; ++dh)
#pragma unroll
                    for (int v = 0; v < 16; ++v) acc[dh][v] *= a;
                ref = to;
                l = probs(kt, key0, part, pb);
            }
            sum += l;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int dh = 0; dh < 2; ++dh) acc[dh] = mfma(rd.cols(vt, u, e, dh), pb[u][e], acc[dh]);
        }
        wait_vm_all();
        __syncthreads();
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
