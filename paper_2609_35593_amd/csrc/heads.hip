// Norm of every head of Q and K with the rotary positions, forward, backward and into pages.
//
// Memory bound: an element is read and written once (backward: two reads, one write). As in
// rope.hip a thread owns one chunk of a token's channels and walks over the heads, the angles
// formed once; a head's chunks lie in `lanes` neighbouring lanes of a wave, which add up the row's sums among
// themselves. Norm and turn are one step: with xc = x - mean an output is
//   rstd (xc_own A + xc_other B) + C,  A = gamma_own cos, B = -+ gamma_other sin, C = beta_own cos -+ beta_other sin,
// so that the three coefficients are kept over a token's heads in place of six values. The chunk that
// a chunk's pairs meet is read a second time, from the L1. Where halves, strides or addresses allow no
// chunks of 16 or 8 bytes a thread owns pairs of channels instead.
//
// Backward: the gradients of gamma and beta stay in registers over all tokens of a workgroup, which
// leaves one row of partial sums; join_kernel adds the rows in order.
#include "pages_internal.h"

namespace ress {
namespace {

constexpr int kThreads = 256;

template <typename T, int V>
struct alignas(sizeof(T) * V) Chunk {
    T e[V];
};

__device__ __forceinline__ float get(float x) { return x; }
__device__ __forceinline__ float get(uint16_t x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }
__device__ __forceinline__ void put(float &d, float x) { d = x; }
__device__ __forceinline__ void put(uint16_t &d, float x) { d = __builtin_bit_cast(uint16_t, (__bf16)x); }

// cos and sin of `turns` turns a position, in float64 up to the fraction of a turn (as in rope.hip).
__device__ __forceinline__ void angle(const RopeParams &p, const int32_t *pos, int pair, float &c, float &s)
{
    const double t = (double)pos[p.axis[pair]] * p.turns[pair];
    sincospif((float)(2.0 * (t - rint(t))), &s, &c);
}

template <int CTRL>
__device__ __forceinline__ float add_from(float x)
{
    return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}

// Sums over 1 << log2 neighbouring lanes, the same in each of them. (All of a wave's lanes take part.)
template <int M>
__device__ __forceinline__ void add_lanes(float (&x)[M], int log2)
{
    if (log2 >= 1)
#pragma unroll
        for (int j = 0; j < M; ++j) x[j] = add_from<0xB1>(x[j]);  // lanes 1 0 3 2
    if (log2 >= 2)
#pragma unroll
        for (int j = 0; j < M; ++j) x[j] = add_from<0x4E>(x[j]);  // lanes 2 3 0 1
    if (log2 >= 3)
#pragma unroll
        for (int j = 0; j < M; ++j) x[j] = add_from<0x141>(x[j]);  // mirrored in 8 lanes
    if (log2 >= 4)
#pragma unroll
        for (int j = 0; j < M; ++j) x[j] = add_from<0x140>(x[j]);  // mirrored in 16 lanes
    if (log2 >= 5)
#pragma unroll
        for (int j = 0; j < M; ++j) x[j] += __shfl_xor(x[j], 16);
    if (log2 >= 6)
#pragma unroll
        for (int j = 0; j < M; ++j) x[j] += __shfl_xor(x[j], 32);
}

// A chunk's coefficients (turn forward): own and other channel's of a pair.
template <int V>
struct Coefs {
    float a[V], b[V], c[V];
};

// A thread's place: its token, its chunk, and what that chunk's pairs are.
struct Place {
    int64_t t;     // (the last token again behind it)
    int c, other;  // own chunk; the chunk that its pairs meet
    int pair;      // its first pair
    bool there;    // the token and the chunk exist
    bool copy;     // channels that do not turn
    bool second;   // (halves) the pairs' second side
};

template <int V>
__device__ __forceinline__ Place place_of(const RopeParams &p, int64_t i, int lanes_log2)
{
    Place x;
    const int64_t t = i >> lanes_log2;
    const int c = (int)i & ((1 << lanes_log2) - 1);
    x.there = t < p.N && c * V < p.D;
    x.t = t < p.N ? t : p.N - 1;
    x.c = c * V < p.D ? c : 0;
    x.copy = x.c * V >= p.turned;
    x.other = p.other[x.c];
    x.pair = p.pair_of[x.c];
    x.second = x.other < x.c;
    return x;
}

// cos and sin of a chunk's entries: cs, and sn with the sign of the entry's other channel in the
// forward turn (own' = own cs + other sn). A pair of halves shares its angles: the first side's
// thread forms the first half of them, the second side's the rest.
template <int V, bool INTERLEAVED>
__device__ __forceinline__ void chunk_angles(const RopeParams &p, const Place &x, float (&cs)[V], float (&sn)[V])
{
    const int32_t *pos = p.pos + x.t * p.n_axes;
    if constexpr (INTERLEAVED) {
#pragma unroll
        for (int e = 0; e < V / 2; ++e) {
            float c = 1.f, s = 0.f;
            if (!x.copy) angle(p, pos, x.pair + e, c, s);
            cs[2 * e] = cs[2 * e + 1] = c;
            sn[2 * e] = -s;
            sn[2 * e + 1] = s;
        }
    } else {
        const int lane = threadIdx.x & 63, mate = lane - x.c + x.other;
#pragma unroll
        for (int e = 0; e < V / 2; ++e) {
            float c0 = 1.f, s0 = 0.f;
            if (!x.copy) angle(p, pos, x.pair + e + (x.second ? V / 2 : 0), c0, s0);
            const float c1 = __shfl(c0, mate), s1 = __shfl(s0, mate);
            cs[e] = x.second ? c1 : c0;
            sn[e] = x.second ? s1 : -s0;
            cs[e + V / 2] = x.second ? c0 : c1;
            sn[e + V / 2] = x.second ? s0 : -s1;
        }
    }
}

__device__ __forceinline__ float weight(const float *w, int i, float none) { return w ? w[i] : none; }

// Where head h of q, k and v together reads and writes token t: q first, then k, then v.
template <typename T>
struct Rows {
    const T *in;
    T *out;
    int64_t in_step, out_step;  // between heads
    int n;                      // heads
};
template <typename T>
__device__ __forceinline__ Rows<T> rows_of(const HeadNormParams &p, int role, int64_t t, int slot)
{
    const RopeParams &r = p.r;
    Rows<T> x;
    if (role == 0) {
        x.in = static_cast<const T *>(r.q_in) + t * r.qi.token;
        x.out = static_cast<T *>(r.q_out) + t * r.qo.token;
        x.in_step = r.qi.head;
        x.out_step = r.qo.head;
        x.n = r.H;
        return x;
    }
    x.n = r.H_all - r.H;
    const bool v = role == 2;
    x.in = v ? static_cast<const T *>(p.v_in) + t * p.vi.token : static_cast<const T *>(r.k_in) + t * r.ki.token;
    x.in_step = v ? p.vi.head : r.ki.head;
    if (p.slots) {
        const int page = p.pages(slot);
        const ress_page_strides &s = v ? p.vp : p.kp;
        x.out = static_cast<T *>(v ? p.v_out : r.k_out) + page * s.page + (int64_t)(slot - page * p.page) * s.token;
        x.out_step = s.head;
    } else {
        x.out = static_cast<T *>(r.k_out) + t * r.ko.token;
        x.out_step = r.ko.head;
    }
    return x;
}

// The part of heads [h0, h1) of q, k and v together that a role has: its own [a, b).
__device__ __forceinline__ void role_heads(const RopeParams &r, int role, int h0, int h1, int &a, int &b)
{
    const int kv = r.H_all - r.H, base = role == 0 ? 0 : role == 1 ? r.H : r.H_all, n = role == 0 ? r.H : kv;
    a = max(h0 - base, 0);
    b = min(h1 - base, n);
}

// A thread: token i >> lanes_log2, chunk of V channels; heads blockIdx.y * heads ..., B of them in flight. (A token's lanes
// lie in one wave: its loads are ahead of its stores, also where an output is its input.)
template <typename T, int V, int B, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads) chunk_kernel(const HeadNormParams p, int lanes_log2, int heads)
{
    using Chunk = Chunk<T, V>;
    const RopeParams &r = p.r;
    const Place x = place_of<V>(r, (int64_t)blockIdx.x * kThreads + threadIdx.x, lanes_log2);
    const int slot = p.slots ? p.slots[x.t] : 0;
    const bool cached = !p.slots || (unsigned int)slot < (unsigned int)p.n_slots;
    const int h_all = r.H_all + (p.slots ? r.H_all - r.H : 0);
    const int h0 = blockIdx.y * heads, h1 = min(h0 + heads, h_all);
    const bool own = (threadIdx.x & ((1 << lanes_log2) - 1)) * V < r.D;  // the chunk exists
    const float width = 1.f / (float)r.D;
    float cs[V], sn[V];
    chunk_angles<V, INTERLEAVED>(r, x, cs, sn);
    for (int role = 0; role < 2; ++role) {
        int a, b;
        role_heads(r, role, h0, h1, a, b);
        if (a >= b) continue;
        const bool store = x.there && (role == 0 || cached);
        const Rows<T> rows = rows_of<T>(p, role, x.t, cached ? slot : 0);
        Coefs<V> f;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int i = x.c * V + e, o = INTERLEAVED ? i ^ 1 : x.other * V + e;
            f.a[e] = weight(p.gamma[role], i, 1.f) * cs[e];
            f.b[e] = weight(p.gamma[role], o, 1.f) * sn[e];
            f.c[e] = weight(p.beta[role], i, 0.f) * cs[e] + weight(p.beta[role], o, 0.f) * sn[e];
        }
        for (int hb = a; hb < b; hb += B) {
            Chunk xo[B], xp[B];
#pragma unroll
            for (int j = 0; j < B; ++j) {
                const T *in = rows.in + min(hb + j, b - 1) * rows.in_step;
                xo[j] = *reinterpret_cast<const Chunk *>(in + x.c * V);
                if constexpr (!INTERLEAVED) xp[j] = *reinterpret_cast<const Chunk *>(in + x.other * V);
            }
            float m[B], q[B];
#pragma unroll
            for (int j = 0; j < B; ++j) {
                m[j] = 0.f;
                if (p.layer && own)
#pragma unroll
                    for (int e = 0; e < V; ++e) m[j] += get(xo[j].e[e]);
            }
            if (p.layer) add_lanes(m, lanes_log2);
#pragma unroll
            for (int j = 0; j < B; ++j) {
                m[j] *= width;
                q[j] = 0.f;
                if (own)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float d = get(xo[j].e[e]) - m[j];
                        q[j] = fmaf(d, d, q[j]);
                    }
            }
            add_lanes(q, lanes_log2);
#pragma unroll
            for (int j = 0; j < B; ++j) {
                if (hb + j >= b || !store) break;
                const float rstd = 1.f / sqrtf(fmaf(q[j], width, p.eps));
                Chunk y;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float d = (get(xo[j].e[e]) - m[j]) * rstd;
                    const float z = (get(INTERLEAVED ? xo[j].e[e ^ 1] : xp[j].e[e]) - m[j]) * rstd;
                    put(y.e[e], fmaf(d, f.a[e], fmaf(z, f.b[e], f.c[e])));
                }
                *reinterpret_cast<Chunk *>(rows.out + (hb + j) * rows.out_step + x.c * V) = y;
            }
        }
    }
    int a, b;
    role_heads(r, 2, h0, h1, a, b);
    if (!p.slots || !cached || !x.there || a >= b) return;
    const Rows<T> rows = rows_of<T>(p, 2, x.t, slot);
    for (int h = a; h < b; ++h)
        *reinterpret_cast<Chunk *>(rows.out + h * rows.out_step + x.c * V) =
            *reinterpret_cast<const Chunk *>(rows.in + h * rows.in_step + x.c * V);
}

// A thread's pairs of a row where there are no chunks: pairs c, c + 64 of token i >> lanes_log2.
template <int U>
struct Pairs {
    int64_t t;
    bool there;
    int ca[U], cb[U];
    bool on[U];
    float cs[U], sn[U];
};
template <int U>
__device__ __forceinline__ Pairs<U> pairs_of(const RopeParams &p, int64_t i, int lanes_log2)
{
    Pairs<U> x;
    const int64_t t = i >> lanes_log2;
    x.there = t < p.N;
    x.t = x.there ? t : p.N - 1;
    const int c = (int)i & ((1 << lanes_log2) - 1);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        x.on[u] = c + 64 * u < p.n_pairs;
        const int pr = x.on[u] ? c + 64 * u : 0;
        x.ca[u] = p.ca[pr];
        x.cb[u] = p.cb[pr];
        x.cs[u] = 1.f;
        x.sn[u] = 0.f;
        if (!(p.turns[pr] < 0.0)) angle(p, p.pos + x.t * p.n_axes, pr, x.cs[u], x.sn[u]);
    }
    return x;
}

template <typename T, int B, int U>
__global__ void __launch_bounds__(kThreads) pair_kernel(const HeadNormParams p, int lanes_log2, int heads)
{
    const RopeParams &r = p.r;
    const Pairs<U> x = pairs_of<U>(r, (int64_t)blockIdx.x * kThreads + threadIdx.x, lanes_log2);
    const int slot = p.slots ? p.slots[x.t] : 0;
    const bool cached = !p.slots || (unsigned int)slot < (unsigned int)p.n_slots;
    const int h_all = r.H_all + (p.slots ? r.H_all - r.H : 0);
    const int h0 = blockIdx.y * heads, h1 = min(h0 + heads, h_all);
    const float width = 1.f / (float)r.D;
    for (int role = 0; role < 2; ++role) {
        int a, b;
        role_heads(r, role, h0, h1, a, b);
        if (a >= b) continue;
        const bool store = x.there && (role == 0 || cached);
        const Rows<T> rows = rows_of<T>(p, role, x.t, cached ? slot : 0);
        float ga[U], gb[U], ba[U], bb[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            ga[u] = weight(p.gamma[role], x.ca[u], 1.f);
            gb[u] = weight(p.gamma[role], x.cb[u], 1.f);
            ba[u] = weight(p.beta[role], x.ca[u], 0.f);
            bb[u] = weight(p.beta[role], x.cb[u], 0.f);
        }
        for (int hb = a; hb < b; hb += B) {
            float xa[B][U], xb[B][U], m[B], q[B];
#pragma unroll
            for (int j = 0; j < B; ++j) {
                const T *in = rows.in + min(hb + j, b - 1) * rows.in_step;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    xa[j][u] = get(in[x.ca[u]]);
                    xb[j][u] = get(in[x.cb[u]]);
                }
            }
#pragma unroll
            for (int j = 0; j < B; ++j) {
                m[j] = 0.f;
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (p.layer && x.on[u]) m[j] += xa[j][u] + xb[j][u];
            }
            if (p.layer) add_lanes(m, lanes_log2);
#pragma unroll
            for (int j = 0; j < B; ++j) {
                m[j] *= width;
                q[j] = 0.f;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    xa[j][u] -= m[j];
                    xb[j][u] -= m[j];
                    if (x.on[u]) q[j] = fmaf(xa[j][u], xa[j][u], fmaf(xb[j][u], xb[j][u], q[j]));
                }
            }
            add_lanes(q, lanes_log2);
#pragma unroll
            for (int j = 0; j < B; ++j) {
                if (hb + j >= b || !store) break;
                const float rstd = 1.f / sqrtf(fmaf(q[j], width, p.eps));
                T *out = rows.out + (hb + j) * rows.out_step;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (!x.on[u]) continue;
                    const float ya = fmaf(xa[j][u] * rstd, ga[u], ba[u]), yb = fmaf(xb[j][u] * rstd, gb[u], bb[u]);
                    put(out[x.ca[u]], fmaf(ya, x.cs[u], -(yb * x.sn[u])));
                    put(out[x.cb[u]], fmaf(yb, x.cs[u], ya * x.sn[u]));
                }
            }
        }
    }
    int a, b;
    role_heads(r, 2, h0, h1, a, b);
    if (!p.slots || !cached || !x.there || a >= b) return;
    const Rows<T> rows = rows_of<T>(p, 2, x.t, slot);
    for (int h = a; h < b; ++h) {
        const T *in = rows.in + h * rows.in_step;
        T *out = rows.out + h * rows.out_step;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (x.on[u]) out[x.ca[u]] = in[x.ca[u]], out[x.cb[u]] = in[x.cb[u]];
    }
}

// Lanes of a token: chunks of V channels, or (V = 0) pairs, up to a wave's.
int lanes_of(int D, int V)
{
    int log2 = 0;
    while (log2 < 6 && (V > 0 ? V : 2) << log2 < D) ++log2;
    return log2;
}

template <typename T, int V, int B>
hipError_t go(const HeadNormParams &p, hipStream_t s)
{
    const RopeParams &r = p.r;
    const int lanes_log2 = lanes_of(r.D, V), h_all = r.H_all + (p.slots ? r.H_all - r.H : 0);
    const int64_t blocks = (((int64_t)r.N << lanes_log2) + kThreads - 1) / kThreads;
    // Heads per thread: all that leave 2,048 workgroups, at least one batch.
    int heads = h_all;
    while (heads > B && blocks * ((h_all + heads - 1) / heads) < 2048) heads = (heads + 1) / 2;
    const dim3 grid((unsigned)blocks, (unsigned)((h_all + heads - 1) / heads)), block(kThreads);
    if constexpr (V > 0) {
        if (r.interleaved)
            hipLaunchKernelGGL((chunk_kernel<T, V, B, true>), grid, block, 0, s, p, lanes_log2, heads);
        else
            hipLaunchKernelGGL((chunk_kernel<T, V, B, false>), grid, block, 0, s, p, lanes_log2, heads);
    } else if (r.n_pairs <= 64) {
        hipLaunchKernelGGL((pair_kernel<T, B, 1>), grid, block, 0, s, p, lanes_log2, heads);
    } else {
        hipLaunchKernelGGL((pair_kernel<T, B, 2>), grid, block, 0, s, p, lanes_log2, heads);
    }
    return hipGetLastError();
}

template <typename T>
hipError_t by_chunk(const HeadNormParams &p, hipStream_t s)
{
    constexpr int V = 16 / sizeof(T);
    return p.r.chunk == V ? go<T, V, 4>(p, s) : p.r.chunk == V / 2 ? go<T, V / 2, 4>(p, s) : go<T, 0, 4>(p, s);
}

// ---------------------------------------------------------------- backward

// The rows of one of q and k in the backward pass: gradients of the outputs, inputs, gradients of
// the inputs.
template <typename T>
struct BwdRows {
    const T *dy, *x;
    T *dx;
    int64_t dy_step, x_step, dx_step;
};
template <typename T>
__device__ __forceinline__ BwdRows<T> bwd_rows(const HeadNormBwdParams &p, int role, int64_t t)
{
    const RopeParams &r = p.r;
    const ress_strides &yi = role ? r.ki : r.qi, &xo = role ? r.ko : r.qo, &xs = p.xs[role];
    return {static_cast<const T *>(role ? r.k_in : r.q_in) + t * yi.token, static_cast<const T *>(p.x[role]) + t * xs.token,
            static_cast<T *>(role ? r.k_out : r.q_out) + t * xo.token, yi.head, xs.head, xo.head};
}

// A workgroup's sums of a channel over its rows: every thread leaves its M values (channels
// first(e) of row `row`), 4 kinds of them; then a thread a column adds up the rows in order.
template <int M, typename F>
__device__ __forceinline__ void leave_sums(const HeadNormBwdParams &p, float *lds, int rows, int row, int part, float (&s)[4][M],
                                           F channel)
{
    const int D = p.r.D;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < M; ++e) {
            const int c = channel(e);
            if (c >= 0) lds[row * D + c] = s[k][e];
        }
        __syncthreads();
        for (int c = threadIdx.x; c < D; c += kThreads) {
            float a = 0.f;
            for (int i = 0; i < rows; ++i) a += lds[i * D + c];
            p.part[((int64_t)part * 4 + k) * D + c] = a;
        }
    }
}

// A workgroup: heads blockIdx.y * heads ... of 256 / lanes tokens at a time, every gridDim.x-th of them.
template <typename T, int V, int B, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads) chunk_bwd_kernel(const HeadNormBwdParams p, int lanes_log2, int heads)
{
    using Chunk = Chunk<T, V>;
    __shared__ float lds[kThreads * V];
    const RopeParams &r = p.r;
    const int h0 = blockIdx.y * heads, h1 = min(h0 + heads, r.H_all);
    const bool own = (threadIdx.x & ((1 << lanes_log2) - 1)) * V < r.D;
    const float width = 1.f / (float)r.D;
    float s[4][V];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) s[k][e] = 0.f;
    const int64_t all = (int64_t)r.N << lanes_log2, step = (int64_t)gridDim.x * kThreads;
    for (int64_t i0 = (int64_t)blockIdx.x * kThreads; i0 < all; i0 += step) {
        const Place x = place_of<V>(r, i0 + threadIdx.x, lanes_log2);
        float cs[V], sn[V];
        chunk_angles<V, INTERLEAVED>(r, x, cs, sn);
#pragma unroll
        for (int role = 0; role < 2; ++role) {
            int a, b;
            role_heads(r, role, h0, h1, a, b);
            if (a >= b) continue;
            const BwdRows<T> rows = bwd_rows<T>(p, role, x.t);
            float ga[V];
#pragma unroll
            for (int e = 0; e < V; ++e) ga[e] = weight(p.gamma[role], x.c * V + e, 1.f);
            for (int hb = a; hb < b; hb += B) {
                Chunk yo[B], yp[B], xo[B];
#pragma unroll
                for (int j = 0; j < B; ++j) {
                    const int h = min(hb + j, b - 1);
                    const T *dy = rows.dy + h * rows.dy_step;
                    yo[j] = *reinterpret_cast<const Chunk *>(dy + x.c * V);
                    if constexpr (!INTERLEAVED) yp[j] = *reinterpret_cast<const Chunk *>(dy + x.other * V);
                    xo[j] = *reinterpret_cast<const Chunk *>(rows.x + h * rows.x_step + x.c * V);
                }
                float m[B], t[3 * B];
#pragma unroll
                for (int j = 0; j < B; ++j) {
                    m[j] = 0.f;
                    if (p.layer && own)
#pragma unroll
                        for (int e = 0; e < V; ++e) m[j] += get(xo[j].e[e]);
                }
                if (p.layer) add_lanes(m, lanes_log2);
#pragma unroll
                for (int j = 0; j < B; ++j) {
                    m[j] *= width;
                    float qq = 0.f, sg = 0.f, sx = 0.f;
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float d = get(xo[j].e[e]) - m[j];
                        // (The turn back: the sines change sign.)
                        const float z = get(INTERLEAVED ? yo[j].e[e ^ 1] : yp[j].e[e]);
                        const float g = fmaf(get(yo[j].e[e]), cs[e], -(z * sn[e])) * ga[e];
                        qq = fmaf(d, d, qq);
                        sg += g;
                        sx = fmaf(g, d, sx);
                    }
                    t[3 * j] = own ? qq : 0.f;
                    t[3 * j + 1] = own ? sg : 0.f;
                    t[3 * j + 2] = own ? sx : 0.f;
                }
                add_lanes(t, lanes_log2);
#pragma unroll
                for (int j = 0; j < B; ++j) {
                    if (hb + j >= b || !x.there) break;
                    const float rstd = 1.f / sqrtf(fmaf(t[3 * j], width, p.eps));
                    const float mg = p.layer ? t[3 * j + 1] * width : 0.f, mx = t[3 * j + 2] * rstd * width;
                    Chunk y;
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float xh = (get(xo[j].e[e]) - m[j]) * rstd;
                        const float z = get(INTERLEAVED ? yo[j].e[e ^ 1] : yp[j].e[e]);
                        const float u = fmaf(get(yo[j].e[e]), cs[e], -(z * sn[e]));
                        put(y.e[e], rstd * (fmaf(u, ga[e], -mg) - xh * mx));
                        s[2 * role][e] = fmaf(u, xh, s[2 * role][e]);
                        s[2 * role + 1][e] += u;
                    }
                    *reinterpret_cast<Chunk *>(rows.dx + (hb + j) * rows.dx_step + x.c * V) = y;
                }
            }
        }
    }
    if (!p.part) return;
    const int c = threadIdx.x & ((1 << lanes_log2) - 1);
    leave_sums<V>(p, lds, kThreads >> lanes_log2, threadIdx.x >> lanes_log2, blockIdx.y * gridDim.x + blockIdx.x, s,
                  [&](int e) { return own ? c * V + e : -1; });
}

template <typename T, int U>
__global__ void __launch_bounds__(kThreads) pair_bwd_kernel(const HeadNormBwdParams p, int lanes_log2, int heads)
{
    __shared__ float lds[kThreads * 2 * U];
    const RopeParams &r = p.r;
    const int h0 = blockIdx.y * heads, h1 = min(h0 + heads, r.H_all);
    const float width = 1.f / (float)r.D;
    float s[4][2 * U];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < 2 * U; ++e) s[k][e] = 0.f;
    const int64_t all = (int64_t)r.N << lanes_log2, step = (int64_t)gridDim.x * kThreads;
    Pairs<U> x;
    for (int64_t i0 = (int64_t)blockIdx.x * kThreads; i0 < all; i0 += step) {
        x = pairs_of<U>(r, i0 + threadIdx.x, lanes_log2);
#pragma unroll
        for (int role = 0; role < 2; ++role) {
            int a, b;
            role_heads(r, role, h0, h1, a, b);
            if (a >= b) continue;
            const BwdRows<T> rows = bwd_rows<T>(p, role, x.t);
            for (int h = a; h < b; ++h) {
                const T *dy = rows.dy + h * rows.dy_step, *in = rows.x + h * rows.x_step;
                float m[1] = {0.f}, t[3] = {0.f, 0.f, 0.f}, xa[U], xb[U], ua[U], ub[U], ga[U], gb[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const float ya = get(dy[x.ca[u]]), yb = get(dy[x.cb[u]]);
                    ga[u] = weight(p.gamma[role], x.ca[u], 1.f);
                    gb[u] = weight(p.gamma[role], x.cb[u], 1.f);
                    xa[u] = get(in[x.ca[u]]);
                    xb[u] = get(in[x.cb[u]]);
                    ua[u] = fmaf(ya, x.cs[u], yb * x.sn[u]);
                    ub[u] = fmaf(yb, x.cs[u], -(ya * x.sn[u]));
                    if (p.layer && x.on[u]) m[0] += xa[u] + xb[u];
                }
                if (p.layer) add_lanes(m, lanes_log2);
                m[0] *= width;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    xa[u] -= m[0];
                    xb[u] -= m[0];
                    if (!x.on[u]) continue;
                    t[0] = fmaf(xa[u], xa[u], fmaf(xb[u], xb[u], t[0]));
                    t[1] += ua[u] * ga[u] + ub[u] * gb[u];
                    t[2] = fmaf(ua[u] * ga[u], xa[u], fmaf(ub[u] * gb[u], xb[u], t[2]));
                }
                add_lanes(t, lanes_log2);
                if (!x.there) continue;
                const float rstd = 1.f / sqrtf(fmaf(t[0], width, p.eps));
                const float mg = p.layer ? t[1] * width : 0.f, mx = t[2] * rstd * width;
                T *dx = rows.dx + h * rows.dx_step;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (!x.on[u]) continue;
                    const float ha = xa[u] * rstd, hb = xb[u] * rstd;
                    put(dx[x.ca[u]], rstd * (fmaf(ua[u], ga[u], -mg) - ha * mx));
                    put(dx[x.cb[u]], rstd * (fmaf(ub[u], gb[u], -mg) - hb * mx));
                    s[2 * role][2 * u] = fmaf(ua[u], ha, s[2 * role][2 * u]);
                    s[2 * role][2 * u + 1] = fmaf(ub[u], hb, s[2 * role][2 * u + 1]);
                    s[2 * role + 1][2 * u] += ua[u];
                    s[2 * role + 1][2 * u + 1] += ub[u];
                }
            }
        }
    }
    if (!p.part) return;
    x = pairs_of<U>(r, threadIdx.x, lanes_log2);  // (the thread's pairs, whatever its tokens)
    leave_sums<2 * U>(p, lds, kThreads >> lanes_log2, threadIdx.x >> lanes_log2, blockIdx.y * gridDim.x + blockIdx.x, s,
                      [&](int e) { return x.on[e >> 1] ? (e & 1 ? x.cb[e >> 1] : x.ca[e >> 1]) : -1; });
}

// 4 columns of the partial sums' rows a workgroup, 64 runs of rows each, joined in order.
__global__ void __launch_bounds__(kThreads) join_kernel(const HeadNormBwdParams p)
{
    __shared__ float lds[kThreads];
    const int columns = 4 * p.r.D, c = blockIdx.x * 4 + (threadIdx.x & 3), run = threadIdx.x >> 2;
    float a = 0.f;
    if (c < columns)
        for (int i = run; i < p.parts; i += 64) a += p.part[(int64_t)i * columns + c];
    lds[threadIdx.x] = a;
    __syncthreads();
    if (run > 0 || c >= columns) return;
    a = 0.f;
    for (int i = 0; i < 64; ++i) a += lds[i * 4 + (threadIdx.x & 3)];
    float *out = p.sums[c / p.r.D];
    if (out) out[c % p.r.D] = a;
}

template <typename T, int V, int B>
hipError_t go_bwd(const HeadNormBwdParams &p, hipStream_t s)
{
    const RopeParams &r = p.r;
    const int lanes_log2 = lanes_of(r.D, V);
    const HeadBwdPlan plan = head_bwd_plan(r.H_all, r.N, r.D);
    if (plan.parts > 0) {
        const dim3 grid((unsigned)plan.tokens, (unsigned)((r.H_all + plan.heads - 1) / plan.heads)), block(kThreads);
        if constexpr (V > 0) {
            if (r.interleaved)
                hipLaunchKernelGGL((chunk_bwd_kernel<T, V, B, true>), grid, block, 0, s, p, lanes_log2, plan.heads);
            else
                hipLaunchKernelGGL((chunk_bwd_kernel<T, V, B, false>), grid, block, 0, s, p, lanes_log2, plan.heads);
        } else if (r.n_pairs <= 64) {
            hipLaunchKernelGGL((pair_bwd_kernel<T, 1>), grid, block, 0, s, p, lanes_log2, plan.heads);
        } else {
            hipLaunchKernelGGL((pair_bwd_kernel<T, 2>), grid, block, 0, s, p, lanes_log2, plan.heads);
        }
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (!p.part) return hipSuccess;
    hipLaunchKernelGGL(join_kernel, dim3((unsigned)r.D), dim3(kThreads), 0, s, p);
    return hipGetLastError();
}

template <typename T>
hipError_t bwd_by_chunk(const HeadNormBwdParams &p, hipStream_t s)
{
    constexpr int V = 16 / sizeof(T);
    return p.r.chunk == V ? go_bwd<T, V, 2>(p, s) : p.r.chunk == V / 2 ? go_bwd<T, V / 2, 2>(p, s) : go_bwd<T, 0, 1>(p, s);
}

}  // namespace

hipError_t launch_head_norm(const HeadNormParams &p, hipStream_t s)
{
    return p.r.f32 ? by_chunk<float>(p, s) : by_chunk<uint16_t>(p, s);
}

hipError_t launch_head_norm_bwd(const HeadNormBwdParams &p, hipStream_t s)
{
    return p.r.f32 ? bwd_by_chunk<float>(p, s) : bwd_by_chunk<uint16_t>(p, s);
}

}  // namespace ress
