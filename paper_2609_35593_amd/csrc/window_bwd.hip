// Gradients of the windowed attention. The probabilities are formed again from the
// logarithms of their sums, once for each of two kernels, so that every gradient is a sum
// in one workgroup's registers, in one order, with no atomics: 7 products of 64 channels
// per visible pair instead of 5.
//
//   delta_kernel  per query -sum_d d_o o, and lse in base 2;
//   dq_kernel     128 queries a workgroup, walking over the key tiles they see:
//                 S^T = K Q^T, dP^T = V dO^T - delta, dQ^T += K^T dS^T. delta off by e leaves
//                 -e (sum P k) in dQ, which for keys with a common part outweighs dQ itself,
//                 and o is rounded to bf16, as dS is for its product; so sum dS = e (0 for the
//                 true delta and unrounded dS) is summed from the rounded values as well,
//                 B^T += K^T P^T beside it, and dQ takes back e B (without it dq was 1-1.5% off
//                 in norm where keys share a mean). The corrected delta goes to the next kernel;
//   dkv_kernel    128 keys a workgroup, walking over the tiles of queries that see them,
//                 query head after query head of those that share the keys:
//                 S = Q K^T, dP = dO V^T - delta, dV^T += dO^T P, dK^T += Q^T dS.
// In both a lane holds one column of the score tile (a query, a key), so P and dS, rounded
// to bf16, are the next products' operands as they lie (tiles.h); -delta enters as the
// initial value of the accumulator.
#include "tiles.h"

namespace ress {
namespace {

using namespace tiles;

constexpr float kLog2e = 1.4426950408889634f;

// 8 lanes a query.
__global__ void __launch_bounds__(256) delta_kernel(const WindowBwdParams b)
{
    const WindowParams &p = b.w;
    const int64_t row = (int64_t)blockIdx.x * 32 + (threadIdx.x >> 3);
    if (row >= (int64_t)p.H * p.n_q) return;
    const int h = (int)(row / p.n_q), t = (int)(row - (int64_t)h * p.n_q), l = threadIdx.x & 7;
    const bf16x8 x = *reinterpret_cast<const bf16x8 *>(b.d_o + h * b.dos.head + (int64_t)t * b.dos.token + l * 8);
    const bf16x8 y = *reinterpret_cast<const bf16x8 *>(p.o + h * p.os.head + (int64_t)t * p.os.token + l * 8);
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf((float)x[e], (float)y[e], s);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) s += __shfl_xor(s, o);
    if (l == 0) {
        const float lse = p.lse[row];
        b.ndelta[row] = -s;
        b.lse2[row] = lse == -INFINITY ? INFINITY : lse * kLog2e;  // (a query that sees nothing: P = 0)
    }
}

__global__ void __launch_bounds__(256, 2) dq_kernel(const WindowBwdParams b)
{
    __shared__ __attribute__((aligned(1024))) unsigned char k_s[2][kTileBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char v_s[2][kTileBytes];
    const WindowParams &p = b.w;
    const int rows = p.H * p.n_qb, per = (rows + 7) / 8;
    const int at = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || at >= rows) return;
    const int h = at / p.n_qb, i = p.n_qb - 1 - (at - h * p.n_qb);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hh = lane >> 5, ql = lane & 31;

    // Tiles and ranges as in the forward pass (window.hip).
    const int t_first = i * 128, t_last = min(t_first + 128, p.n_q) - 1;
    const Seen s_first = seen_by(p, p.q_offset + t_first), s_last = seen_by(p, p.q_offset + t_last);
    const int ns = (s_last.sk + kTile - 1) / kTile;
    int w0 = s_first.lo / kTile, w1 = (s_last.hi + kTile - 1) / kTile;
    if (s_first.lo >= s_last.hi) w0 = w1 = ns;
    if (w0 < ns) w0 = ns;
    if (w1 < w0) w1 = w0;
    const int tiles_n = ns + w1 - w0;
    auto tile_key = [&](int c) __attribute__((always_inline)) { return (c < ns ? c : c - ns + w0) * kTile; };
    const int ta = min(t_first + wave * 32, t_last), tb = min(t_first + wave * 32 + 31, t_last);
    const Seen sa = seen_by(p, p.q_offset + ta), sb = seen_by(p, p.q_offset + tb);
    const int t = t_first + wave * 32 + ql, tq = min(t, t_last);
    const Seen sl = seen_by(p, p.q_offset + tq);

    bf16x8 qf[4], df[4];
    {
        const uint16_t *q = p.q + h * p.qs.head + (int64_t)tq * p.qs.token + hh * 8;
        const uint16_t *d = b.d_o + h * b.dos.head + (int64_t)tq * b.dos.token + hh * 8;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            qf[kk] = *reinterpret_cast<const bf16x8 *>(q + kk * 16);
            df[kk] = *reinterpret_cast<const bf16x8 *>(d + kk * 16);
        }
    }
    const float lse2 = b.lse2[(int64_t)h * p.n_q + tq], nd = b.ndelta[(int64_t)h * p.n_q + tq];
    const Loader<4> load_k(p.k + (h / p.group) * p.ks.head, p.ks.token, wave, lane);
    const Loader<4> load_v(p.v + (h / p.group) * p.vs.head, p.vs.token, wave, lane);
    const Reader rd(lane);
    auto fetch = [&](int c, int slot) __attribute__((always_inline)) {
        const int key0 = tile_key(c);
        const bool sinks = key0 < s_last.sk, window = key0 + kTile > s_first.lo && key0 < s_last.hi;
        const int lo = sinks ? 0 : s_first.lo, hi = window ? max(s_last.hi, s_last.sk) : s_last.sk;
        load_k(key0, lo, hi, k_s[slot]);
        load_v(key0, lo, hi, v_s[slot]);
    };
    const float c = p.scale_log2;
    f32x16 acc[2], mean[2];  // sum dS k, sum P k
    float off = 0.f;         // the lane's half of sum dS
#pragma unroll
    for (int dh = 0; dh < 2; ++dh)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[dh][v] = mean[dh][v] = 0.f;

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
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                f32x16 s, d;
#pragma unroll
                for (int v = 0; v < 16; ++v) s[v] = 0.f, d[v] = nd;
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) s = mfma(rd.rows(kt, u, kk), qf[kk], s);
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) d = mfma(rd.rows(vt, u, kk), df[kk], d);
                if (part) {
                    asm volatile("" ::: "memory");
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const int key = key0 + u * 32 + (v >> 2) * 8 + (v & 3) + 4 * hh;
                        const bool in = (key >= sl.lo && key < sl.hi) || key < sl.sk;
                        s[v] = in ? s[v] : -INFINITY;
                    }
                }
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], c, -lse2));
                    d[v] *= s[v];
                }
                bf16x8 pb[2], db[2];
                pack(s, pb);
                pack(d, db);
                off = add_up(db, off);
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int dh = 0; dh < 2; ++dh) {
                        const bf16x8 kc = rd.cols(kt, u, e, dh);
                        acc[dh] = mfma(kc, db[e], acc[dh]);
                        mean[dh] = mfma(kc, pb[e], mean[dh]);
                    }
            }
        }
        wait_vm_all();
        __syncthreads();
    }
    off += __shfl_xor(off, 32);
#pragma unroll
    for (int dh = 0; dh < 2; ++dh)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[dh][v] = fmaf(-off, mean[dh][v], acc[dh][v]);
    if (t > t_last) return;
    if (hh == 0) b.ndelta[(int64_t)h * p.n_q + t] = nd - off;
    store_row(b.dq + h * b.dqs.head + (int64_t)t * b.dqs.token, acc, p.scale, hh);
}

__global__ void __launch_bounds__(256, 2) dkv_kernel(const WindowBwdParams b)
{
    __shared__ __attribute__((aligned(1024))) unsigned char q_s[2][kTileBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char d_s[2][kTileBytes];
    __shared__ __attribute__((aligned(256))) float row_s[2][2][kTile];  // lse2, ndelta of the tile's queries
    const WindowParams &p = b.w;
    const int blocks = p.H_kv * p.n_kb, per = (blocks + 7) / 8;
    const int at = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || at >= blocks) return;
    const int hk = at / p.n_kb, j = at - hk * p.n_kb;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hh = lane >> 5, kl = lane & 31;

    const int s_first = j * 128, s_last = min(s_first + 128, p.n_k) - 1;
    // Queries that see any of the workgroup's keys; of the wave's (none outside [wlo, whi), all
    // inside [alo, ahi)); of the lane's. (The first key's range starts first; sinks are seen
    // to the end, and from keys behind them the last one's range ends last.)
    const int q_lo = queries_of(p, s_first).lo, q_hi = s_first < p.n_sink ? p.n_q : queries_of(p, s_last).hi;
    const int ka = min(s_first + wave * 32, s_last), kb = min(s_first + wave * 32 + 31, s_last);
    const SeenBy qb = queries_of(p, kb);
    const int wlo = queries_of(p, ka).lo, whi = ka < p.n_sink ? p.n_q : qb.hi;
    const int alo = qb.lo, ahi = kb < p.n_sink ? p.n_q : queries_of(p, max(ka, p.n_sink)).hi;
    const int key = s_first + wave * 32 + kl, kq = min(key, s_last);
    const SeenBy ql = queries_of(p, kq);

    bf16x8 kf[4], vf[4];
    {
        const uint16_t *k = p.k + hk * p.ks.head + (int64_t)kq * p.ks.token + hh * 8;
        const uint16_t *v = p.v + hk * p.vs.head + (int64_t)kq * p.vs.token + hh * 8;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            kf[kk] = *reinterpret_cast<const bf16x8 *>(k + kk * 16);
            vf[kk] = *reinterpret_cast<const bf16x8 *>(v + kk * 16);
        }
    }
    Loader<4> load_q(p.q, p.qs.token, wave, lane), load_d(b.d_o, b.dos.token, wave, lane);
    const Reader rd(lane);
    const int first = q_lo / kTile, per_head = q_hi > q_lo ? (q_hi + kTile - 1) / kTile - first : 0;
    const int tiles_n = per_head * p.group;
    // Tile n: query head hk group + n / per_head, queries 64 (first + n % per_head) ..; kept
    // as running counters of the next tile to fetch and the one to compute.
    int fh = hk * p.group, ft = first;
    auto fetch = [&](int slot) __attribute__((always_inline)) {
        const int t0 = ft * kTile;
        load_q.base = p.q + fh * p.qs.head;
        load_d.base = b.d_o + fh * b.dos.head;
        load_q(t0, 0, p.n_q, q_s[slot]);
        load_d(t0, 0, p.n_q, d_s[slot]);
        if (wave < 2) {
            const float *src = (wave == 0 ? b.lse2 : b.ndelta) + (int64_t)fh * p.n_q + t0;
            const int last = min(kTile, p.n_q - t0) - 1;
            const __amdgpu_buffer_rsrc_t rs =
                __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(src), 0, 4 * (last + 1), 0x00020000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void *)row_s[slot][wave], 4, 4 * min(lane, last), 0, 0, 0);
        }
        if (++ft == first + per_head) {
            ft = first;
            ++fh;
        }
    };
    const float c = p.scale_log2;
    f32x16 dk[2], dv[2];
#pragma unroll
    for (int dh = 0; dh < 2; ++dh)
#pragma unroll
        for (int v = 0; v < 16; ++v) dk[dh][v] = 0.f, dv[dh][v] = 0.f;

    if (tiles_n > 0) {
        fetch(0);
        wait_vm_all();
        __syncthreads();
    }
    int t0 = first * kTile;
    for (int n = 0; n < tiles_n; ++n) {
        const int slot = n & 1;
        if (n + 1 < tiles_n) fetch(slot ^ 1);
        if (t0 < whi && t0 + kTile > wlo) {
            const bool part = !(t0 >= alo && t0 + kTile <= ahi);
            const unsigned char *qt = q_s[slot], *dt = d_s[slot];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                f32x16 s, d, l;
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x4 a = *reinterpret_cast<const f32x4 *>(&row_s[slot][0][u * 32 + g * 8 + hh * 4]);
                    const f32x4 e = *reinterpret_cast<const f32x4 *>(&row_s[slot][1][u * 32 + g * 8 + hh * 4]);
#pragma unroll
                    for (int v = 0; v < 4; ++v) s[g * 4 + v] = 0.f, l[g * 4 + v] = a[v], d[g * 4 + v] = e[v];
                }
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) s = mfma(rd.rows(qt, u, kk), kf[kk], s);
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) d = mfma(rd.rows(dt, u, kk), vf[kk], d);
                if (part) {
                    asm volatile("" ::: "memory");
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const int t = t0 + u * 32 + (v >> 2) * 8 + (v & 3) + 4 * hh;
                        s[v] = t >= ql.lo && t < ql.hi ? s[v] : -INFINITY;
                    }
                }
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], c, -l[v]));
                    d[v] *= s[v];
                }
                bf16x8 pb[2], db[2];
                pack(s, pb);
                pack(d, db);
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int dh = 0; dh < 2; ++dh) {
                        dv[dh] = mfma(rd.cols(dt, u, e, dh), pb[e], dv[dh]);
                        dk[dh] = mfma(rd.cols(qt, u, e, dh), db[e], dk[dh]);
                    }
            }
        }
        t0 += kTile;
        if (t0 == (first + per_head) * kTile) t0 = first * kTile;
        wait_vm_all();
        __syncthreads();
    }
    if (key <= s_last) {
        store_row(b.dk + hk * b.dks.head + (int64_t)key * b.dks.token, dk, p.scale, hh);
        store_row(b.dv + hk * b.dvs.head + (int64_t)key * b.dvs.token, dv, 1.f, hh);
    }
}

}  // namespace

hipError_t launch_window_bwd(const WindowBwdParams &b, hipStream_t s)
{
    const WindowParams &p = b.w;
    if (p.n_q > 0) {
        const int64_t rows = (int64_t)p.H * p.n_q;
        hipLaunchKernelGGL(delta_kernel, dim3((unsigned)((rows + 31) / 32)), dim3(256), 0, s, b);
        if (hipError_t e = hipGetLastError()) return e;
        hipLaunchKernelGGL(dq_kernel, dim3(8u * (unsigned)((p.H * p.n_qb + 7) / 8)), dim3(256), 0, s, b);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (p.n_k > 0) {
        hipLaunchKernelGGL(dkv_kernel, dim3(8u * (unsigned)((p.H_kv * p.n_kb + 7) / 8)), dim3(256), 0, s, b);
        return hipGetLastError();
    }
    return hipSuccess;
}

}  // namespace ress
