// Gradients of the windowed attention. The probabilities are formed again from the
// logarithms of their sums, once for each of two kernels, so that every gradient is a sum
// in one workgroup's registers, in one order, with no atomics: 8 products of 64 channels
// per visible pair instead of 5.
//
//   dq_kernel     128 queries a workgroup, walking over the key tiles they see, with
//                 delta = sum_d d_o o of its rows:
//                 S^T = K Q^T, dP^T = V dO^T - delta, dQ^T += K^T dS^T. delta off by e leaves
//                 -e (sum P k) in dQ, which for keys with a common part outweighs dQ itself,
//                 and o is rounded to bf16, as dS is for its product; so sum dS = e (0 for the
//                 true delta and unrounded dS) is summed from the rounded values as well,
//                 B^T += K^T P^T beside it, and dQ takes back e B (without it dq was 1-1.5% off
//                 in norm where keys share a mean). The corrected delta and lse in base 2 go to the
//                 next kernel;
//   dkv_kernel    128 keys a workgroup, walking over the tiles of queries that see them,
//                 query head after query head of those that share the keys:
//                 S = Q K^T, dP = dO V^T - delta, dV^T += dO^T P, dK^T += Q^T dS. Keys of
//                 sinks are seen by all later queries, and small calls have few blocks of keys,
//                 so a block's list may be cut over several workgroups (`slices`), whose float32
//                 sums join_kernel adds in order.
// In both a lane holds one column of the score tile (a query, a key), so P and dS, rounded
// to bf16, are the next products' operands as they lie (tiles.h); -delta enters as the
// initial value of the accumulator.
//
// Bound by issue slots beside the matrix unit, as the forward pass: 16 heads of 8 frames of 1,374
// tokens, window 3 and a frame of sinks, 833-855 us, dq and dkv about half each (the 8 products at 941-966
// TFLOP/s, 79-81% of a large library product's rate; matrix unit busy 51%, vector unit 46 and 42%). 3,001
// tokens, 12 heads for 4, 5 sinks: 56-60 us in three launches of short lists. P and dS are rounded to
// bf16 for the matrix unit: gradients are 2.3e-3 off in norm, 1.7e-3 by their own rounding alone.
#include "tiles.h"

namespace ress {
namespace {

using namespace tiles;

constexpr float kLog2e = 1.4426950408889634f;

template <int G>
__global__ void __launch_bounds__(256, 2) dq_kernel(const WindowBwdParams b)
{
    constexpr int QW = 4 / G, ROWS = 32 * QW;  // waves and queries of a key group (window.hip)
    // (Arrays of their own: of one array's parts the compiler does not see that a read of one
    // slot need not wait for the load into another.)
    __shared__ __attribute__((aligned(1024))) unsigned char k_a0[G * kTileBytes], k_a1[G * kTileBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char v_a0[G * kTileBytes], v_a1[G * kTileBytes];
    const WindowParams &p = b.w;
    const int rows = p.H * p.n_qb, per = (rows + 7) / 8;
    const int at = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || at >= rows) return;
    const int h = p.q_blocks(at), i = p.n_qb - 1 - (at - h * p.n_qb), hk = p.groups(h);
    const int lane = threadIdx.x & 63, wave_wg = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int grp = wave_wg / QW, wave = wave_wg % QW;
    const int hh = lane >> 5, ql = lane & 31;
    unsigned char *const k_0 = k_a0 + grp * kTileBytes, *const k_1 = k_a1 + grp * kTileBytes;
    unsigned char *const v_0 = v_a0 + grp * kTileBytes, *const v_1 = v_a1 + grp * kTileBytes;

    // Tiles and ranges as in the forward pass (window.hip).
    const int t_first = i * ROWS, t_last = min(t_first + ROWS, p.n_q) - 1;
    const Seen s_first = seen_by(p, p.q_offset + t_first), s_last = seen_by(p, p.q_offset + t_last);
    const int ns = (s_last.sk + kTile - 1) / kTile;
    int w0 = s_first.lo / kTile, w1 = (s_last.hi + kTile - 1) / kTile;
    if (s_first.lo >= s_last.hi) w0 = w1 = ns;
    if (w0 < ns) w0 = ns;
    if (w1 < w0) w1 = w0;
    const int tiles_n = ns + w1 - w0, turns = (tiles_n + G - 1) / G;
    auto tile_key = [&](int n) __attribute__((always_inline)) {
        const int c = n * G + grp;
        return (c < ns ? c : c - ns + w0) * kTile;
    };
    const int ta = min(t_first + wave * 32, t_last), tb = min(t_first + wave * 32 + 31, t_last);
    const Seen sa = seen_by(p, p.q_offset + ta), sb = seen_by(p, p.q_offset + tb);
    const int t = t_first + wave * 32 + ql, tq = min(t, t_last);
    Seen sl = seen_by(p, p.q_offset + tq);
    sl.lo -= 4 * hh;
    sl.hi -= 4 * hh;
    sl.sk -= 4 * hh;

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
    float nd = 0.f;
    {
        const uint16_t *o = p.o + h * p.os.head + (int64_t)tq * p.os.token + hh * 8;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            const bf16x8 x = *reinterpret_cast<const bf16x8 *>(o + kk * 16);
#pragma unroll
            for (int e = 0; e < 8; ++e) nd = fmaf(-(float)df[kk][e], (float)x[e], nd);
        }
        nd += __shfl_xor(nd, 32);
    }
    // (A query that sees nothing: P = 0.)
    const float lse = p.lse[(int64_t)h * p.n_q + tq], lse2 = lse == -INFINITY ? INFINITY : lse * kLog2e;
    const Loader<QW> load_k(p.k + hk * p.ks.head, p.ks.token, wave, lane);
    const Loader<QW> load_v(p.v + hk * p.vs.head, p.vs.token, wave, lane);
    const Reader rd(lane);
    auto fetch = [&](int n, unsigned char *kd, unsigned char *vd) __attribute__((always_inline)) {
        if (n * G + grp >= tiles_n) return;
        const int key0 = tile_key(n);
        const bool sinks = key0 < s_last.sk, window = s_first.lo < s_last.hi && key0 + kTile > s_first.lo && key0 < s_last.hi;
        const int lo = sinks ? 0 : s_first.lo, hi = window ? max(s_last.hi, s_last.sk) : s_last.sk;
        const int end = sinks && window ? s_first.lo : 0;  // a tile of both: what lies between them
        load_k(key0, lo, hi, s_last.sk, end, kd);
        load_v(key0, lo, hi, s_last.sk, end, vd);
    };
    const float c = p.scale_log2;
    f32x16 acc[2], mean[2];  // sum dS k, sum P k
    f32x16 nd16;
    float off = 0.f;         // the lane's half of sum dS
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[0][v] = acc[1][v] = mean[0][v] = mean[1][v] = 0.f, nd16[v] = nd;

    auto tile = [&](bool part, const unsigned char *kt, const unsigned char *vt, int key0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f32x16 s, d = nd16;
#pragma unroll
            for (int v = 0; v < 16; ++v) s[v] = 0.f;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) s = mfma(rd.rows(kt, u, kk), qf[kk], s);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) d = mfma(rd.rows(vt, u, kk), df[kk], d);
            if (part) hide(s, key0 + u * 32, sl.lo, (unsigned int)(sl.hi - sl.lo), key0 < sb.sk, sl.sk);
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
    };
    int n = 0;
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
    if constexpr (G > 1) {
        // The groups behind the first leave their sums in the slots (65 floats a lane), in two
        // rounds: the slots hold one 32-channel half of all of them.
        constexpr int PER = 33 * 64;
        constexpr int FIT = G * kTileBytes / (PER * 4);  // waves per slot array
        static_assert((G - 1) * QW <= 2 * FIT, "a round's parts fit the key slots");
        auto area = [&](int w) __attribute__((always_inline)) -> float * {
            return reinterpret_cast<float *>(w < FIT ? k_a0 : k_a1) + w % FIT * PER + lane;
        };
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            if (r) __syncthreads();
            if (grp > 0) {
                float *m = area((grp - 1) * QW + wave);
#pragma unroll
                for (int v = 0; v < 16; ++v) m[v * 64] = acc[r][v], m[(16 + v) * 64] = mean[r][v];
                m[32 * 64] = off;
            }
            __syncthreads();
            if (grp == 0) {
#pragma unroll
                for (int g = 1; g < G; ++g) {
                    const float *m = area((g - 1) * QW + wave);
#pragma unroll
                    for (int v = 0; v < 16; ++v) acc[r][v] += m[v * 64], mean[r][v] += m[(16 + v) * 64];
                    if (r == 0) off += m[32 * 64];
                }
            }
        }
        if (grp > 0) return;
    }
    off += __shfl_xor(off, 32);
#pragma unroll
    for (int dh = 0; dh < 2; ++dh)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[dh][v] = fmaf(-off, mean[dh][v], acc[dh][v]);
    if (t > t_last) return;
    if (hh == 0) {
        b.ndelta[(int64_t)h * p.n_q + t] = nd - off;
        b.lse2[(int64_t)h * p.n_q + t] = lse2;
    }
    store_row(b.dq + h * b.dqs.head + (int64_t)t * b.dqs.token, acc, p.scale, hh);
}

// Item `at` of the keys' pass: a slice of a block of keys. Sink blocks' items come first.
struct Item {
    int hk, block, slice, slices;
};
__device__ __forceinline__ Item item_of(const WindowBwdParams &b, int at)
{
    Item r;
    r.hk = at / b.items;
    int x = at - r.hk * b.items;
    const int sinks = b.sink_blocks * b.sink_slices;
    r.slices = x < sinks ? b.sink_slices : b.slices;
    if (x >= sinks) x -= sinks;
    r.block = x / r.slices;
    r.slice = x - r.block * r.slices;
    if (at - r.hk * b.items >= sinks) r.block += b.sink_blocks;
    return r;
}

__global__ void __launch_bounds__(256, 2) dkv_kernel(const WindowBwdParams b)
{
    __shared__ __attribute__((aligned(1024))) unsigned char q_0[kTileBytes], q_1[kTileBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char d_0[kTileBytes], d_1[kTileBytes];
    __shared__ __attribute__((aligned(256))) float row_0[2][kTile], row_1[2][kTile];  // lse2, ndelta of the tile's queries
    const WindowParams &p = b.w;
    const int items = p.H_kv * b.items, per = (items + 7) / 8;
    const int at = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || at >= items) return;
    const Item item = item_of(b, at);
    const int hk = item.hk;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hh = lane >> 5, kl = lane & 31;

    const int s_first = item.block * 128, s_last = min(s_first + 128, p.n_k) - 1;
    // Queries that see any of the workgroup's keys; of the wave's (none outside [wlo, whi), all
    // inside [alo, ahi)); of the lane's. (The first key's range starts first; sinks are seen
    // to the end, and from keys behind them the last one's range ends last.)
    const int q_lo = queries_of(p, s_first).lo, q_hi = s_first < p.n_sink ? p.n_q : queries_of(p, s_last).hi;
    const int ka = min(s_first + wave * 32, s_last), kb = min(s_first + wave * 32 + 31, s_last);
    const SeenBy qb = queries_of(p, kb);
    const int wlo = queries_of(p, ka).lo, whi = ka < p.n_sink ? p.n_q : qb.hi;
    const int alo = qb.lo, ahi = kb < p.n_sink ? p.n_q : queries_of(p, max(ka, p.n_sink)).hi;
    const int key = s_first + wave * 32 + kl, kq = min(key, s_last);
    SeenBy ql = queries_of(p, kq);
    ql.lo -= 4 * hh;
    ql.hi -= 4 * hh;

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
    // The block's list, query head after query head, and this slice's part of it: [n, end).
    const int first = q_lo / kTile, per_head = q_hi > q_lo ? (q_hi + kTile - 1) / kTile - first : 0;
    const int64_t all = (int64_t)per_head * p.group;
    int n = (int)(all * item.slice / item.slices);
    const int end = (int)(all * (item.slice + 1) / item.slices);
    // Query head and first query of the next tile to fetch, and the latter of the one to compute.
    int fh = 0, ft = 0, t0 = 0;
    if (n < end) {
        fh = hk * p.group + n / per_head;
        ft = (first + n % per_head) * kTile;
        t0 = ft;
    }
    const int t_end = (first + per_head) * kTile;
    auto fetch = [&](unsigned char *qd, unsigned char *dd, float (&rows)[2][kTile]) __attribute__((always_inline)) {
        load_q.base = p.q + fh * p.qs.head;
        load_d.base = b.d_o + fh * b.dos.head;
        // (Queries that see none of the keys are not read.)
        load_q(ft, q_lo, q_hi, 0, 0, qd);
        load_d(ft, q_lo, q_hi, 0, 0, dd);
        if (wave < 2) {
            const int t_a = max(ft, q_lo), last = min(ft + kTile, q_hi) - 1 - t_a;
            const float *src = (wave == 0 ? b.lse2 : b.ndelta) + (int64_t)fh * p.n_q + t_a;
            const __amdgpu_buffer_rsrc_t rs =
                __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(src), 0, 4 * (last + 1), 0x00020000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void *)rows[wave], 4, 4 * min(max(lane + ft - t_a, 0), last), 0,
                                                     0, 0);
        }
        ft += kTile;
        if (ft == t_end) {
            ft = first * kTile;
            ++fh;
        }
    };
    const float c = p.scale_log2;
    f32x16 dk[2], dv[2];
#pragma unroll
    for (int dh = 0; dh < 2; ++dh)
#pragma unroll
        for (int v = 0; v < 16; ++v) dk[dh][v] = 0.f, dv[dh][v] = 0.f;

    auto tile = [&](bool part, const unsigned char *qt, const unsigned char *dt, const float (&rows)[2][kTile])
                    __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f32x16 s, d, l;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 a = *reinterpret_cast<const f32x4 *>(&rows[0][u * 32 + g * 8 + hh * 4]);
                const f32x4 e = *reinterpret_cast<const f32x4 *>(&rows[1][u * 32 + g * 8 + hh * 4]);
#pragma unroll
                for (int v = 0; v < 4; ++v) s[g * 4 + v] = 0.f, l[g * 4 + v] = a[v], d[g * 4 + v] = e[v];
            }
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) s = mfma(rd.rows(qt, u, kk), kf[kk], s);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) d = mfma(rd.rows(dt, u, kk), vf[kk], d);
            if (part) hide(s, t0 + u * 32, ql.lo, (unsigned int)(ql.hi - ql.lo), false, 0);
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
    };
    auto step = [&](const unsigned char *qt, const unsigned char *dt, const float (&rt)[2][kTile], unsigned char *qd,
                    unsigned char *dd, float (&rd_)[2][kTile]) __attribute__((always_inline)) -> bool {
        if (n + 1 < end) fetch(qd, dd, rd_);
        if (t0 < whi && t0 + kTile > wlo) tile(!(t0 >= alo && t0 + kTile <= ahi), qt, dt, rt);
        t0 += kTile;
        if (t0 == t_end) t0 = first * kTile;
        wait_vm_all();
        __syncthreads();
        return ++n < end;
    };
    if (n < end) {
        fetch(q_0, d_0, row_0);
        wait_vm_all();
        __syncthreads();
        while (step(q_0, d_0, row_0, q_1, d_1, row_1) && step(q_1, d_1, row_1, q_0, d_0, row_0)) {
        }
    }
    if (item.slices > 1) {
        float *part = b.part + ((int64_t)at * 2 * 128 + wave * 32 + kl) * 64;
#pragma unroll
        for (int dh = 0; dh < 2; ++dh)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float *at_c = part + dh * 32 + g * 8 + hh * 4;
                *reinterpret_cast<f32x4 *>(at_c) = f32x4{dk[dh][g * 4], dk[dh][g * 4 + 1], dk[dh][g * 4 + 2], dk[dh][g * 4 + 3]};
                *reinterpret_cast<f32x4 *>(at_c + 128 * 64) =
                    f32x4{dv[dh][g * 4], dv[dh][g * 4 + 1], dv[dh][g * 4 + 2], dv[dh][g * 4 + 3]};
            }
    } else if (key <= s_last) {
        store_row(b.dk + hk * b.dks.head + (int64_t)key * b.dks.token, dk, p.scale, hh);
        store_row(b.dv + hk * b.dvs.head + (int64_t)key * b.dvs.token, dv, 1.f, hh);
    }
}

// Blocks of keys whose list was cut: a workgroup 32 keys of dk (even) or dv, 2 x 4 channels a
// thread, the slices in order. blockIdx.y counts the cut blocks of all heads, `cut` of a head from `first` on.
__global__ void __launch_bounds__(256) join_kernel(const WindowBwdParams b, int first, int cut)
{
    const WindowParams &p = b.w;
    const int hk = blockIdx.y / cut, block = first + blockIdx.y % cut;
    const int slices = block < b.sink_blocks ? b.sink_slices : b.slices;
    const int at = hk * b.items + (block < b.sink_blocks
                                       ? block * b.sink_slices
                                       : b.sink_blocks * b.sink_slices + (block - b.sink_blocks) * b.slices);
    const int tensor = blockIdx.x & 1, row = (blockIdx.x >> 1) * 32 + (threadIdx.x >> 3), c = (threadIdx.x & 7) * 8;
    const int key = block * 128 + row;
    if (key >= p.n_k) return;
    const float *part = b.part + (((int64_t)at * 2 + tensor) * 128 + row) * 64 + c;
    f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
#pragma unroll 4
    for (int s = 0; s < slices; ++s) {
        x += *reinterpret_cast<const f32x4 *>(part + (int64_t)s * 2 * 128 * 64);
        y += *reinterpret_cast<const f32x4 *>(part + (int64_t)s * 2 * 128 * 64 + 4);
    }
    const float f = tensor ? 1.f : p.scale;
    uint16_t *out = tensor ? b.dv + hk * b.dvs.head + (int64_t)key * b.dvs.token : b.dk + hk * b.dks.head + (int64_t)key * b.dks.token;
    bf16x8 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (__bf16)(x[e] * f), o[e + 4] = (__bf16)(y[e] * f);
    *reinterpret_cast<bf16x8 *>(out + c) = o;
}

}  // namespace

hipError_t launch_window_bwd(const WindowBwdParams &b, int groups, hipStream_t s)
{
    const WindowParams &p = b.w;
    if (p.n_q > 0) {
        const dim3 grid(8u * (unsigned)((p.H * p.n_qb + 7) / 8)), block(256);
        if (groups == 1)
            hipLaunchKernelGGL(dq_kernel<1>, grid, block, 0, s, b);
        else if (groups == 2)
            hipLaunchKernelGGL(dq_kernel<2>, grid, block, 0, s, b);
        else
            hipLaunchKernelGGL(dq_kernel<4>, grid, block, 0, s, b);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (p.n_k > 0) {
        hipLaunchKernelGGL(dkv_kernel, dim3(8u * (unsigned)((p.H_kv * b.items + 7) / 8)), dim3(256), 0, s, b);
        if (hipError_t e = hipGetLastError()) return e;
        int first = 0;
        const int cut = window_bwd_joined({groups, b.sink_blocks, b.sink_slices, b.slices, b.items}, p.n_kb, first);
        if (cut > 0) {
            hipLaunchKernelGGL(join_kernel, dim3(8, (unsigned)(p.H_kv * cut)), dim3(256), 0, s, b, first, cut);
            return hipGetLastError();
        }
    }
    return hipSuccess;
}

}  // namespace ress
