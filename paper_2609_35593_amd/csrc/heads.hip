// Norm of every head of Q and K with the rotary positions, forward, backward and into pages.
//
// Memory bound: an element is read and written once (backward: two reads, one write). As in
// rope.hip a thread owns one chunk of a token's channels and walks over the heads, the angles
// formed once; a head's chunks lie in `lanes` neighbouring lanes of a wave, which add up the row's sums among
// themselves. Norm and turn are one step: an output is
//   rstd ((x_own - mean) A + (x_other - mean) B) + C,
//   A = gamma_own cos, B = -+ gamma_other sin, C = beta_own cos -+ beta_other sin,
// with coefficients that are kept over a token's heads; the weights they are formed from lie in LDS (read from
// memory a value at a time they took longer than 4 heads of a token). The chunk that a chunk's pairs meet is
// read a second time, from the L1. Where halves, strides or addresses allow no chunks of 16 or 8 bytes a
// thread owns pairs of channels instead.
//
// Backward: the gradients of gamma and beta stay in registers over all tokens of a workgroup, which
// leaves one row of partial sums; join_kernel adds the rows in order.
//
// Measured (a copy on this card moves 5.2 TB/s): 43,968 tokens of 16 + 16 bf16 heads, layer norm, two axes 80 us, 4.5 TB/s
// (root mean square 77: the mean is a second chain of sums over lanes), float32 143 us, 5.0 TB/s; with axes of 20, 20 and 24
// channels, by pairs, bf16 97 us, 3.7 TB/s, gradients of 21,984 tokens 97 where chunks take 62. 11,264 rows of 16 + 4 heads into
// pages, V with them, 16.6 us, 4.2 TB/s (704 workgroups, each with its angles to form and its last stores to wait for). Kernels
// alone: backward 21,984 tokens 51 us, 5.3 TB/s with some of it from the caches, and the join 4; 1,374 tokens, 12 + 4 float32 heads
// 10 us and the join 3: 688 workgroups of one trip, which waits for positions, angles in float64, loads, and sums in turn; 24
// tokens forward 5.9 us, the same chain.
#include "pages_internal.h"

namespace ress {
namespace {

constexpr int kThreads = 256;

template <typename T, int V>
struct alignas(sizeof(T) * V) Chunk {
    T e[V];
};

// The chunk's words as they are, unknown to the compiler from here on: values converted from them are converted again
// behind this, not kept beside them (which spilled).
template <typename T, int V>
__device__ __forceinline__ void forget(Chunk<T, V> &c)
{
    constexpr int n = sizeof(T) * V / 4;
    uint32_t w[n];
    __builtin_memcpy(w, &c, sizeof w);
#pragma unroll
    for (int i = 0; i < n; ++i) asm volatile("" : "+v"(w[i]));
    __builtin_memcpy(&c, w, sizeof w);
}

__device__ __forceinline__ float get(float x) { return x; }
__device__ __forceinline__ float get(uint16_t x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }
__device__ __forceinline__ void put(float &d, float x) { d = x; }
__device__ __forceinline__ void put(uint16_t &d, float x) { d = __builtin_bit_cast(uint16_t, (__bf16)x); }

// cos and sin of `turns` turns a position, in float64 up to the fraction of a turn (as in rope.hip).
__device__ __forceinline__ void angle(double turns, int32_t pos, float &c, float &s)
{
    const double t = (double)pos * turns;
    sincospif((float)(2.0 * (t - rint(t))), &s, &c);
}

// A workgroup's tables in LDS: gamma and beta of Q and of K ([4][D]), and the pairs' turns and axes. (Read a value at a
// time from memory and from the kernel's arguments, and one behind the other, they took longer than four heads of a
// token.)
struct Tables {
    __attribute__((aligned(16))) float weights[4 * RESS_MAX_ROPE_D];
    double turns[kMaxPairs];
    int axis[kMaxPairs];
};
// (Callers wait for the workgroup.)
__device__ __forceinline__ void load_tables(Tables &t, const RopeParams &r, const float *const (&gamma)[2],
                                            const float *const (&beta)[2])
{
    const int D = r.D;
    for (int i = threadIdx.x; i < D; i += kThreads)
#pragma unroll
        for (int role = 0; role < 2; ++role) {
            t.weights[2 * role * D + i] = gamma[role] ? gamma[role][i] : 1.f;
            t.weights[(2 * role + 1) * D + i] = beta[role] ? beta[role][i] : 0.f;
        }
    // (From the last threads on: others than those of narrow weights.)
    const int i = kThreads - 1 - threadIdx.x;
    if (i < r.n_pairs) {
        t.turns[i] = r.turns[i];
        t.axis[i] = r.axis[i];
    }
}

// A token's positions.
struct Positions {
    int32_t p[RESS_MAX_ROPE_AXES];
    __device__ __forceinline__ Positions(const RopeParams &r, int64_t t)
    {
#pragma unroll
        for (int a = 0; a < RESS_MAX_ROPE_AXES; ++a) p[a] = a < r.n_axes ? r.pos[t * r.n_axes + a] : 0;
    }
    __device__ __forceinline__ int32_t operator[](int axis) const
    {
        const int32_t lo = axis & 1 ? p[1] : p[0], hi = axis & 1 ? p[3] : p[2];
        return axis & 2 ? hi : lo;
    }
};

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
__device__ __forceinline__ Place place_of(const RopeParams &p, const ChunkRuns &runs, int64_t i, int lanes_log2)
{
    Place x;
    const int64_t t = i >> lanes_log2;
    const int c = (int)i & ((1 << lanes_log2) - 1);
    x.there = t < p.N && c * V < p.D;
    x.t = t < p.N ? t : p.N - 1;
    x.c = c * V < p.D ? c : 0;
    x.copy = x.c * V >= p.turned;
    x.other = x.c;
    x.pair = 0;
#pragma unroll
    for (int a = 0; a < RESS_MAX_ROPE_AXES; ++a) {
        const int at = x.c - runs.first[a], half = runs.half[a];
        if (a < runs.n && at >= 0 && at < runs.count[a]) {
            const bool second = half > 0 && at >= half;
            x.other = second ? x.c - half : x.c + half;
            x.pair = runs.pair[a] + (half > 0 ? (second ? at - half : at) * V : at * (V / 2));
        }
    }
    x.second = x.other < x.c;
    return x;
}

// cos and sin of a chunk's entries: cs, and sn with the sign of the entry's other channel in the
// forward turn (own' = own cs + other sn). A pair of halves shares its angles: the first side's
// thread forms the first half of them, the second side's the rest.
template <int V, bool INTERLEAVED>
__device__ __forceinline__ void chunk_angles(const Tables &t, const Positions &pos, const Place &x, float (&cs)[V], float (&sn)[V])
{
    if constexpr (INTERLEAVED) {
#pragma unroll
        for (int e = 0; e < V / 2; ++e) {
            float c = 1.f, s = 0.f;
            if (!x.copy) angle(t.turns[x.pair + e], pos[t.axis[x.pair + e]], c, s);
            cs[2 * e] = cs[2 * e + 1] = c;
            sn[2 * e] = -s;
            sn[2 * e + 1] = s;
        }
    } else {
        const int lane = threadIdx.x & 63, mate = lane - x.c + x.other;
#pragma unroll
        for (int e = 0; e < V / 2; ++e) {
            float c0 = 1.f, s0 = 0.f;
            const int pair = x.pair + e + (x.second ? V / 2 : 0);
            if (!x.copy) angle(t.turns[pair], pos[t.axis[pair]], c0, s0);
            const float c1 = __shfl(c0, mate), s1 = __shfl(s0, mate);
            cs[e] = x.second ? c1 : c0;
            sn[e] = x.second ? s1 : -s0;
            cs[e + V / 2] = x.second ? c0 : c1;
            sn[e + V / 2] = x.second ? s0 : -s1;
        }
    }
}

template <int V>
__device__ __forceinline__ void take(float (&x)[V], const float *lds)
{
    if constexpr (V % 4 == 0) {
#pragma unroll
        for (int e = 0; e < V; e += 4) {
            const float4 y = *reinterpret_cast<const float4 *>(lds + e);
            x[e] = y.x, x[e + 1] = y.y, x[e + 2] = y.z, x[e + 3] = y.w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = lds[e];
    }
}

// Where a role (0: q, 1: k, 2: v) reads and writes token t. Inputs as a scalar address (of the workgroup's first token t0)
// and bytes from there, which fit 32 bits: with an address a lane and head they spilled.
template <typename T>
struct Rows {
    const char *in;
    uint32_t from;
    T *out;
    int64_t in_step, out_step;  // between heads, of the input in bytes
    template <typename C>
    __device__ __forceinline__ C load(int h, int element) const
    {
        return *reinterpret_cast<const C *>(in + h * in_step + (from + (uint32_t)element * (uint32_t)sizeof(T)));
    }
};
template <typename T>
__device__ __forceinline__ Rows<T> rows_of(const HeadNormParams &p, int role, int64_t t0, int64_t t, int slot)
{
    const RopeParams &r = p.r;
    const ress_strides &s = role == 0 ? r.qi : role == 1 ? r.ki : p.vi;
    Rows<T> x;
    x.in = static_cast<const char *>(role == 0 ? r.q_in : role == 1 ? r.k_in : p.v_in) + t0 * s.token * (int64_t)sizeof(T);
    x.from = (uint32_t)(t - t0) * (uint32_t)s.token * (uint32_t)sizeof(T);
    x.in_step = s.head * (int64_t)sizeof(T);
    if (role > 0 && p.slots) {
        const int page = p.pages(slot);
        const ress_page_strides &to = role == 2 ? p.vp : p.kp;
        x.out = static_cast<T *>(role == 2 ? p.v_out : r.k_out) + page * to.page + (int64_t)(slot - page * p.page) * to.token;
        x.out_step = to.head;
    } else {
        const ress_strides &to = role == 0 ? r.qo : r.ko;
        x.out = static_cast<T *>(role == 0 ? r.q_out : r.k_out) + t * to.token;
        x.out_step = to.head;
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

// NB heads of a row of chunks from `h` on: loads, sums, and the outputs.
template <typename T, int V, int NB, bool INTERLEAVED>
struct Batch {
    Chunk<T, V> xo[NB], xp[NB];
    __device__ __forceinline__ void load(const Rows<T> &rows, const Place &x, int h)
    {
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            xo[j] = rows.template load<Chunk<T, V>>(h + j, x.c * V);
            if constexpr (!INTERLEAVED) xp[j] = rows.template load<Chunk<T, V>>(h + j, x.other * V);
        }
    }
    template <bool LAYER>
    __device__ __forceinline__ void turn(const Rows<T> &rows, const Place &x, int h, int lanes_log2, bool own, bool store, float width,
                                         float eps, const float (&a)[V], const float (&b)[V], const float (&c)[V])
    {
        float m[NB], q[NB];
        if constexpr (LAYER) {
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                m[j] = 0.f;
                if (own)
#pragma unroll
                    for (int e = 0; e < V; ++e) m[j] += get(xo[j].e[e]);
            }
            add_lanes(m, lanes_log2);
        }
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            if (LAYER) forget(xo[j]);
            m[j] = LAYER ? m[j] * width : 0.f;
            q[j] = 0.f;
            if (own)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float d = LAYER ? get(xo[j].e[e]) - m[j] : get(xo[j].e[e]);
                    q[j] = fmaf(d, d, q[j]);
                }
        }
        add_lanes(q, lanes_log2);
        if (!store) return;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const float rstd = 1.f / sqrtf(fmaf(q[j], width, eps));
            forget(xo[j]);
            Chunk<T, V> y;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                // (Centred before the products: behind them, mean (A + B) would take away the digits of rows far from zero.)
                const float z = get(INTERLEAVED ? xo[j].e[e ^ 1] : xp[j].e[e]) - (LAYER ? m[j] : 0.f);
                const float x_own = get(xo[j].e[e]) - (LAYER ? m[j] : 0.f);
                put(y.e[e], fmaf(fmaf(z, b[e], x_own * a[e]), rstd, c[e]));
            }
            *reinterpret_cast<Chunk<T, V> *>(rows.out + (h + j) * rows.out_step + x.c * V) = y;
            __builtin_amdgcn_sched_barrier(0);  // (one head's values at a time)
        }
    }
};

// A thread: token i >> lanes_log2, chunk of V channels; heads blockIdx.y * heads ..., four of them in flight, behind them one at a
// time. (A token's lanes lie in one wave: its loads are ahead of its stores, also where an output is its input.)
template <typename T, int V, bool INTERLEAVED, bool LAYER>
__global__ void __launch_bounds__(kThreads, V * sizeof(T) == 16 ? 3 : 4) chunk_kernel(const HeadNormParams p, int lanes_log2, int heads)
{
    __shared__ Tables tables;
    const RopeParams &r = p.r;
    const Place x = place_of<V>(r, p.runs, (int64_t)blockIdx.x * kThreads + threadIdx.x, lanes_log2);
    const Positions pos(r, x.t);
    const int slot = p.slots ? p.slots[x.t] : 0;
    const int h_all = r.H_all + (p.slots ? r.H_all - r.H : 0);
    const int h0 = blockIdx.y * heads, h1 = min(h0 + heads, h_all);
    const bool own = (threadIdx.x & ((1 << lanes_log2) - 1)) * V < r.D;  // the chunk exists
    const float width = 1.f / (float)r.D;
    const int64_t t0 = (int64_t)blockIdx.x * kThreads >> lanes_log2;
    const bool cached = !p.slots || (unsigned int)slot < (unsigned int)p.n_slots;
    // The first heads are on their way while the tables and the coefficients are formed.
    Batch<T, V, 4, INTERLEAVED> four;
    Rows<T> rows;
    int h, end;
    auto begin = [&](int role) __attribute__((always_inline)) {
        role_heads(r, role, h0, h1, h, end);
        if (h >= end) return;
        rows = rows_of<T>(p, role, t0, x.t, cached ? slot : 0);
        if (h + 4 <= end) four.load(rows, x, h);
    };
    begin(0);
    load_tables(tables, r, p.gamma, p.beta);
    __syncthreads();
    float cs[V], sn[V];
    chunk_angles<V, INTERLEAVED>(tables, pos, x, cs, sn);
#pragma nounroll
    for (int role = 0; role < 2; ++role) {
        if (role == 1) begin(1);
        if (h >= end) continue;
        const bool store = x.there && (role == 0 || cached);
        float a[V], b[V], c[V];
        const float *const w = tables.weights + 2 * role * r.D;
        constexpr int Q = V < 4 ? V : 4;
#pragma unroll
        for (int e0 = 0; e0 < V; e0 += Q) {
            float g[Q], be[Q], go[Q], bo[Q];
            take(g, w + x.c * V + e0);
            take(be, w + r.D + x.c * V + e0);
            if constexpr (!INTERLEAVED) {
                take(go, w + x.other * V + e0);
                take(bo, w + r.D + x.other * V + e0);
            }
#pragma unroll
            for (int i = 0; i < Q; ++i) {
                const int e = e0 + i;
                a[e] = g[i] * cs[e];
                b[e] = (INTERLEAVED ? g[i ^ 1] : go[i]) * sn[e];
                c[e] = be[i] * cs[e] + (INTERLEAVED ? be[i ^ 1] : bo[i]) * sn[e];
            }
            __builtin_amdgcn_sched_barrier(0);  // (else all weights are held at once: spills)
        }
        if (h + 4 <= end)
            for (;;) {
                four.template turn<LAYER>(rows, x, h, lanes_log2, own, store, width, p.eps, a, b, c);
                h += 4;
                if (h + 4 > end) break;
                four.load(rows, x, h);
            }
        for (; h < end; ++h) {
            Batch<T, V, 1, INTERLEAVED> one;
            one.load(rows, x, h);
            one.template turn<LAYER>(rows, x, h, lanes_log2, own, store, width, p.eps, a, b, c);
        }
    }
    int a, b;
    role_heads(r, 2, h0, h1, a, b);
    if (!p.slots || !cached || !x.there || a >= b) return;
    rows = rows_of<T>(p, 2, t0, x.t, slot);
    for (; a + 4 <= b; a += 4) {
        Chunk<T, V> y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = rows.template load<Chunk<T, V>>(a + j, x.c * V);
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<Chunk<T, V> *>(rows.out + (a + j) * rows.out_step + x.c * V) = y[j];
    }
    for (; a < b; ++a)
        *reinterpret_cast<Chunk<T, V> *>(rows.out + a * rows.out_step + x.c * V) =
            rows.template load<Chunk<T, V>>(a, x.c * V);
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
__device__ __forceinline__ Pairs<U> pairs_of(const RopeParams &p, const Tables &tables, int64_t i, int lanes_log2)
{
    Pairs<U> x;
    const int64_t t = i >> lanes_log2;
    x.there = t < p.N;
    x.t = x.there ? t : p.N - 1;
    const int c = (int)i & ((1 << lanes_log2) - 1);
    const Positions pos(p, x.t);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        x.on[u] = c + 64 * u < p.n_pairs;
        const int pr = x.on[u] ? c + 64 * u : 0;
        x.ca[u] = p.ca[pr];
        x.cb[u] = p.cb[pr];
        x.cs[u] = 1.f;
        x.sn[u] = 0.f;
        const double turns = tables.turns[pr];
        if (!(turns < 0.0)) angle(turns, pos[tables.axis[pr]], x.cs[u], x.sn[u]);
    }
    return x;
}

template <typename T, int B, int U>
__global__ void __launch_bounds__(kThreads) pair_kernel(const HeadNormParams p, int lanes_log2, int heads)
{
    __shared__ Tables tables;
    const RopeParams &r = p.r;
    const int64_t t0 = (int64_t)blockIdx.x * kThreads >> lanes_log2;
    load_tables(tables, r, p.gamma, p.beta);
    __syncthreads();
    const Pairs<U> x = pairs_of<U>(r, tables, (int64_t)blockIdx.x * kThreads + threadIdx.x, lanes_log2);
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
        const Rows<T> rows = rows_of<T>(p, role, t0, x.t, cached ? slot : 0);
        float ga[U], gb[U], ba[U], bb[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float *const w = tables.weights + 2 * role * r.D;
            ga[u] = w[x.ca[u]];
            gb[u] = w[x.cb[u]];
            ba[u] = w[r.D + x.ca[u]];
            bb[u] = w[r.D + x.cb[u]];
        }
        for (int hb = a; hb < b; hb += B) {
            float xa[B][U], xb[B][U], m[B], q[B];
#pragma unroll
            for (int j = 0; j < B; ++j) {
                const int h = min(hb + j, b - 1);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    xa[j][u] = get(rows.template load<T>(h, x.ca[u]));
                    xb[j][u] = get(rows.template load<T>(h, x.cb[u]));
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
    const Rows<T> rows = rows_of<T>(p, 2, t0, x.t, slot);
    for (int h = a; h < b; ++h) {
        T *out = rows.out + h * rows.out_step;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (x.on[u]) out[x.ca[u]] = rows.template load<T>(h, x.ca[u]), out[x.cb[u]] = rows.template load<T>(h, x.cb[u]);
    }
}

// Lanes of a token: chunks of V channels, or (V = 0) pairs, up to a wave's.
int lanes_of(int D, int V)
{
    int log2 = 0;
    while (log2 < 6 && (V > 0 ? V : 2) << log2 < D) ++log2;
    return log2;
}

template <typename T, int V>
hipError_t go(const HeadNormParams &p, hipStream_t s)
{
    const RopeParams &r = p.r;
    const int lanes_log2 = lanes_of(r.D, V), h_all = r.H_all + (p.slots ? r.H_all - r.H : 0);
    const int64_t blocks = (((int64_t)r.N << lanes_log2) + kThreads - 1) / kThreads;
    // Heads per thread: all that leave 512 workgroups, in fours, so that few calls fill the CUs' three or four places of a workgroup
    // more than once and not twice. (us where 256 / 512 / 1,024 are left: 5,496 bf16 tokens of 16 + 16 heads 17.2 / 14.9 / 18.0,
    // 10,992 29.6 / 24.0 / 26.1; 11,264 of 16 + 4 into pages 21.2 / 17.8 / 19.6; 5,496 float32 tokens of 12 + 4 14.4 / 12.4 / 14.3.)
    int heads = (h_all + 3) / 4 * 4;
    while (heads > 4 && blocks * ((h_all + heads - 1) / heads) < 512) heads = (heads / 2 + 3) / 4 * 4;
    const dim3 grid((unsigned)blocks, (unsigned)((h_all + heads - 1) / heads)), block(kThreads);
    if constexpr (V > 0) {
        if (r.interleaved && p.layer)
            hipLaunchKernelGGL((chunk_kernel<T, V, true, true>), grid, block, 0, s, p, lanes_log2, heads);
        else if (r.interleaved)
            hipLaunchKernelGGL((chunk_kernel<T, V, true, false>), grid, block, 0, s, p, lanes_log2, heads);
        else if (p.layer)
            hipLaunchKernelGGL((chunk_kernel<T, V, false, true>), grid, block, 0, s, p, lanes_log2, heads);
        else
            hipLaunchKernelGGL((chunk_kernel<T, V, false, false>), grid, block, 0, s, p, lanes_log2, heads);
    } else if (r.n_pairs <= 64) {
        hipLaunchKernelGGL((pair_kernel<T, 4, 1>), grid, block, 0, s, p, lanes_log2, heads);
    } else {
        hipLaunchKernelGGL((pair_kernel<T, 4, 2>), grid, block, 0, s, p, lanes_log2, heads);
    }
    return hipGetLastError();
}

template <typename T>
hipError_t by_chunk(const HeadNormParams &p, hipStream_t s)
{
    constexpr int V = 16 / sizeof(T);
    return p.r.chunk == V ? go<T, V>(p, s) : p.r.chunk == V / 2 ? go<T, V / 2>(p, s) : go<T, 0>(p, s);
}

// ---------------------------------------------------------------- backward

// The rows of one of q and k in the backward pass: gradients of the outputs, inputs, gradients of
// the inputs; each as a scalar address of the workgroup's first token t0 and bytes from there, as in Rows.
template <typename T>
struct BwdRows {
    const char *dy, *x;
    char *dx;
    int64_t dy_step, x_step, dx_step;  // between heads, in bytes
    uint32_t dy_from, x_from, dx_from;
    template <typename C>
    __device__ __forceinline__ C load_dy(int h, int element) const
    {
        return *reinterpret_cast<const C *>(dy + h * dy_step + (dy_from + (uint32_t)element * (uint32_t)sizeof(T)));
    }
    template <typename C>
    __device__ __forceinline__ C load_x(int h, int element) const
    {
        return *reinterpret_cast<const C *>(x + h * x_step + (x_from + (uint32_t)element * (uint32_t)sizeof(T)));
    }
    template <typename C>
    __device__ __forceinline__ void store(int h, int element, const C &c) const
    {
        *reinterpret_cast<C *>(dx + h * dx_step + (dx_from + (uint32_t)element * (uint32_t)sizeof(T))) = c;
    }
};
template <typename T>
__device__ __forceinline__ BwdRows<T> bwd_rows(const HeadNormBwdParams &p, int role, int64_t t0, int64_t t)
{
    constexpr int64_t size = sizeof(T);
    const RopeParams &r = p.r;
    const ress_strides &dy = role ? r.ki : r.qi, &dx = role ? r.ko : r.qo, &xs = p.xs[role];
    const uint32_t n = (uint32_t)(t - t0) * (uint32_t)size;
    return {static_cast<const char *>(role ? r.k_in : r.q_in) + t0 * dy.token * size,
            static_cast<const char *>(p.x[role]) + t0 * xs.token * size,
            static_cast<char *>(role ? r.k_out : r.q_out) + t0 * dx.token * size,
            dy.head * size, xs.head * size, dx.head * size,
            n * (uint32_t)dy.token, n * (uint32_t)xs.token, n * (uint32_t)dx.token};
}

// A workgroup's sums of a channel over its rows: every thread leaves its M values (channel channel(e) of row
// `row`) of 4 kinds; then a thread a column adds up the rows in order. lds: [4][rows][D].
template <int M, typename F>
__device__ __forceinline__ void leave_sums(const HeadNormBwdParams &p, float *lds, int rows, int row, int part, const float (&s)[4][M],
                                           F channel)
{
    const int D = p.r.D;
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < M; ++e) {
            const int c = channel(e);
            if (c >= 0) lds[(k * rows + row) * D + c] = s[k][e];
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 4 * D; i += kThreads) {
        const int k = i / D;
        const float *x = lds + k * rows * D + (i - k * D);
        float a = 0.f;
#pragma unroll 8
        for (int j = 0; j < rows; ++j) a += x[j * D];
        p.part[(int64_t)part * 4 * D + i] = a;
    }
}

// A workgroup: heads blockIdx.y * heads ... of 256 / lanes tokens at a time, every gridDim.x-th of them.
template <typename T, int V, int B, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads, V == 8 ? 3 : 4) chunk_bwd_kernel(const HeadNormBwdParams p, int lanes_log2, int heads)
{
    using Chunk = Chunk<T, V>;
    __shared__ float lds[4 * kThreads * V];
    __shared__ Tables tables;
    const RopeParams &r = p.r;
    load_tables(tables, r, p.gamma, {nullptr, nullptr});
    const int h0 = blockIdx.y * heads, h1 = min(h0 + heads, r.H_all);
    const bool own = (threadIdx.x & ((1 << lanes_log2) - 1)) * V < r.D;
    const float width = 1.f / (float)r.D;
    float s[4][V];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) s[k][e] = 0.f;
    bool waited = false;  // for the tables
    const int64_t all = (int64_t)r.N << lanes_log2, step = (int64_t)gridDim.x * kThreads;
    for (int64_t i0 = (int64_t)blockIdx.x * kThreads; i0 < all; i0 += step) {
        const Place x = place_of<V>(r, p.runs, i0 + threadIdx.x, lanes_log2);
        const Positions pos(r, x.t);
        // (The first heads' loads are on their way while the tables come and the angles are formed.)
        Chunk yo[B], yp[B], xo[B];
        BwdRows<T> rows;
        int a, b;
        auto load = [&](int h) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < B; ++j) {
                if (j > 0 && h + j >= b) break;
                yo[j] = rows.template load_dy<Chunk>(h + j, x.c * V);
                if constexpr (!INTERLEAVED) yp[j] = rows.template load_dy<Chunk>(h + j, x.other * V);
                xo[j] = rows.template load_x<Chunk>(h + j, x.c * V);
            }
        };
        auto begin = [&](int role) __attribute__((always_inline)) {
            role_heads(r, role, h0, h1, a, b);
            if (a >= b) return;
            rows = bwd_rows<T>(p, role, i0 >> lanes_log2, x.t);
            load(a);
        };
        begin(0);
        if (!waited) __syncthreads();
        waited = true;
        float cs[V], sn[V];
        chunk_angles<V, INTERLEAVED>(tables, pos, x, cs, sn);
#pragma unroll
        for (int role = 0; role < 2; ++role) {
            if (role == 1) begin(1);
            if (a >= b) continue;
            float ga[V];
            take(ga, tables.weights + 2 * role * r.D + x.c * V);
            for (int hb = a; hb < b; hb += B) {
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
                    rows.store(hb + j, x.c * V, y);
                }
                if (hb + B < b) load(hb + B);
            }
        }
    }
    if (!p.part) return;
    const int c = threadIdx.x & ((1 << lanes_log2) - 1);
    leave_sums<V>(p, lds, kThreads >> lanes_log2, threadIdx.x >> lanes_log2, blockIdx.y * gridDim.x + blockIdx.x, s,
                  [&](int e) { return own ? c * V + e : -1; });
}

template <typename T, int B, int U>
__global__ void __launch_bounds__(kThreads) pair_bwd_kernel(const HeadNormBwdParams p, int lanes_log2, int heads)
{
    __shared__ float lds[4 * kThreads * 2 * U];
    __shared__ Tables tables;
    const RopeParams &r = p.r;
    load_tables(tables, r, p.gamma, {nullptr, nullptr});
    __syncthreads();
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
        x = pairs_of<U>(r, tables, i0 + threadIdx.x, lanes_log2);
#pragma unroll
        for (int role = 0; role < 2; ++role) {
            int a, b;
            role_heads(r, role, h0, h1, a, b);
            if (a >= b) continue;
            const BwdRows<T> rows = bwd_rows<T>(p, role, i0 >> lanes_log2, x.t);
            float ga[U], gb[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                ga[u] = tables.weights[2 * role * r.D + x.ca[u]];
                gb[u] = tables.weights[2 * role * r.D + x.cb[u]];
            }
            for (int hb = a; hb < b; hb += B) {
                float xa[B][U], xb[B][U], ua[B][U], ub[B][U], m[B], t[3 * B];
#pragma unroll
                for (int j = 0; j < B; ++j) {
                    const int h = min(hb + j, b - 1);
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        xa[j][u] = get(rows.template load_x<T>(h, x.ca[u]));
                        xb[j][u] = get(rows.template load_x<T>(h, x.cb[u]));
                        ua[j][u] = get(rows.template load_dy<T>(h, x.ca[u]));
                        ub[j][u] = get(rows.template load_dy<T>(h, x.cb[u]));
                    }
                }
#pragma unroll
                for (int j = 0; j < B; ++j) {
                    m[j] = 0.f;
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const float ya = ua[j][u], yb = ub[j][u];
                        ua[j][u] = fmaf(ya, x.cs[u], yb * x.sn[u]);
                        ub[j][u] = fmaf(yb, x.cs[u], -(ya * x.sn[u]));
                        if (p.layer && x.on[u]) m[j] += xa[j][u] + xb[j][u];
                    }
                }
                if (p.layer) add_lanes(m, lanes_log2);
#pragma unroll
                for (int j = 0; j < B; ++j) {
                    float qq = 0.f, sg = 0.f, sx = 0.f;
                    m[j] *= width;
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        xa[j][u] -= m[j];
                        xb[j][u] -= m[j];
                        if (!x.on[u]) continue;
                        const float g = ua[j][u] * ga[u], k = ub[j][u] * gb[u];
                        qq = fmaf(xa[j][u], xa[j][u], fmaf(xb[j][u], xb[j][u], qq));
                        sg += g + k;
                        sx = fmaf(g, xa[j][u], fmaf(k, xb[j][u], sx));
                    }
                    t[3 * j] = qq;
                    t[3 * j + 1] = sg;
                    t[3 * j + 2] = sx;
                }
                add_lanes(t, lanes_log2);
#pragma unroll
                for (int j = 0; j < B; ++j) {
                    if (hb + j >= b || !x.there) break;
                    const float rstd = 1.f / sqrtf(fmaf(t[3 * j], width, p.eps));
                    const float mg = p.layer ? t[3 * j + 1] * width : 0.f, mx = t[3 * j + 2] * rstd * width;
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        if (!x.on[u]) continue;
                        const float ha = xa[j][u] * rstd, hc = xb[j][u] * rstd;
                        T da, db;
                        put(da, rstd * (fmaf(ua[j][u], ga[u], -mg) - ha * mx));
                        put(db, rstd * (fmaf(ub[j][u], gb[u], -mg) - hc * mx));
                        rows.store(hb + j, x.ca[u], da);
                        rows.store(hb + j, x.cb[u], db);
                        s[2 * role][2 * u] = fmaf(ua[j][u], ha, s[2 * role][2 * u]);
                        s[2 * role][2 * u + 1] = fmaf(ub[j][u], hc, s[2 * role][2 * u + 1]);
                        s[2 * role + 1][2 * u] += ua[j][u];
                        s[2 * role + 1][2 * u + 1] += ub[j][u];
                    }
                }
            }
        }
    }
    if (!p.part) return;
    x = pairs_of<U>(r, tables, threadIdx.x, lanes_log2);  // (the thread's pairs, whatever its tokens)
    leave_sums<2 * U>(p, lds, kThreads >> lanes_log2, threadIdx.x >> lanes_log2, blockIdx.y * gridDim.x + blockIdx.x, s,
                      [&](int e) { return x.on[e >> 1] ? (e & 1 ? x.cb[e >> 1] : x.ca[e >> 1]) : -1; });
}

// 4 columns of the partial sums' rows a workgroup, 64 runs of rows each, 12 rows of a run on their way at once; joined in a fixed
// order, by lanes and then by waves.
__global__ void __launch_bounds__(kThreads) join_kernel(const HeadNormBwdParams p, int parts)
{
    __shared__ float lds[4][4];
    const int columns = 4 * p.r.D, c = blockIdx.x * 4 + (threadIdx.x & 3), run = threadIdx.x >> 2;
    float a = 0.f;
    for (int i0 = 0; i0 < parts; i0 += 64 * 12) {
        float x[12];
#pragma unroll
        for (int i = 0; i < 12; ++i) {
            const int part = i0 + i * 64 + run;
            x[i] = p.part[(int64_t)min(part, parts - 1) * columns + c];
            if (part >= parts) x[i] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < 12; ++i) a += x[i];
    }
#pragma unroll
    for (int o = 4; o < 64; o <<= 1) a += __shfl_xor(a, o);
    if ((threadIdx.x & 63) < 4) lds[threadIdx.x >> 6][threadIdx.x & 3] = a;
    __syncthreads();
    if (run > 0) return;
    a = 0.f;
    for (int w = 0; w < 4; ++w) a += lds[w][threadIdx.x & 3];
    float *out = p.sums[c / p.r.D];
    if (out) out[c % p.r.D] = a;
}

template <typename T, int V, int B>
hipError_t go_bwd(const HeadNormBwdParams &p, hipStream_t s)
{
    const RopeParams &r = p.r;
    const int lanes_log2 = lanes_of(r.D, V);
    const HeadBwdPlan plan = head_bwd_plan(r.H_all, r.N, kThreads >> lanes_log2);
    if (plan.parts > 0) {
        const dim3 grid((unsigned)plan.tokens, (unsigned)((r.H_all + plan.heads - 1) / plan.heads)), block(kThreads);
        if constexpr (V > 0) {
            if (r.interleaved)
                hipLaunchKernelGGL((chunk_bwd_kernel<T, V, B, true>), grid, block, 0, s, p, lanes_log2, plan.heads);
            else
                hipLaunchKernelGGL((chunk_bwd_kernel<T, V, B, false>), grid, block, 0, s, p, lanes_log2, plan.heads);
        } else if (r.n_pairs <= 64) {
            hipLaunchKernelGGL((pair_bwd_kernel<T, 4, 1>), grid, block, 0, s, p, lanes_log2, plan.heads);
        } else {
            hipLaunchKernelGGL((pair_bwd_kernel<T, 2, 2>), grid, block, 0, s, p, lanes_log2, plan.heads);
        }
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (!p.part) return hipSuccess;
    hipLaunchKernelGGL(join_kernel, dim3((unsigned)r.D), dim3(kThreads), 0, s, p, plan.parts);
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
