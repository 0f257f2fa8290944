// Layer norm over the channels of a row, forward and backward.
//
// Both passes are memory bound: a row is read into registers once, its sums are
// taken there (the variance from centred values, so that a large mean costs no
// digits), and the result is written from the same registers. A row belongs to LPR
// lanes, each with K chunks of VEC neighbouring channels: narrow rows share a wave
// (8 rows of 64 bf16 channels), ordinary ones take a wave, wide ones a workgroup.
// VEC is what fills 16 bytes of the wider of the two types; rows whose width, strides
// or addresses are not multiples of that take pairs of channels or one at a time.
//
// float32 rows of 1,024 channels, bf16 out: 43,968 forward 50.5 us (5.35 TB/s, a large copy's
// rate), 21,984 backward 48.6 (4.6 TB/s, 4-5 us of it the join of the weights' gradients);
// 175,872 bf16 rows of 64 channels backward 18.5 (3.65 TB/s).
#include <type_traits>

#include "layer_internal.h"

namespace ress {
namespace {

__device__ __forceinline__ float from_bf16(uint16_t b) { return __builtin_bit_cast(float, (uint32_t)b << 16); }
__device__ __forceinline__ uint16_t to_bf16(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

template <typename T, int V>
struct alignas(sizeof(T) * V) Pack {
    T e[V];
};

template <int V>
__device__ __forceinline__ void load(const float *p, float (&x)[V])
{
    const Pack<float, V> t = *reinterpret_cast<const Pack<float, V> *>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = t.e[i];
}
template <int V>
__device__ __forceinline__ void load(const uint16_t *p, float (&x)[V])
{
    const Pack<uint16_t, V> t = *reinterpret_cast<const Pack<uint16_t, V> *>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = from_bf16(t.e[i]);
}
template <int V>
__device__ __forceinline__ void store(float *p, const float (&x)[V])
{
    Pack<float, V> t;
#pragma unroll
    for (int i = 0; i < V; ++i) t.e[i] = x[i];
    *reinterpret_cast<Pack<float, V> *>(p) = t;
}
template <int V>
__device__ __forceinline__ void store(uint16_t *p, const float (&x)[V])
{
    Pack<uint16_t, V> t;
#pragma unroll
    for (int i = 0; i < V; ++i) t.e[i] = to_bf16(x[i]);
    *reinterpret_cast<Pack<uint16_t, V> *>(p) = t;
}

// Sum over the LPR lanes of a row, the same in each of them. Rows of several waves exchange
// through LDS; `buf` alternates, so that one barrier a sum is enough.
template <int LPR, int WAVES>
__device__ __forceinline__ float row_sum(float x, float (&lds)[2][WAVES], int &buf)
{
#pragma unroll
    for (int o = 1; o < (LPR < 64 ? LPR : 64); o <<= 1) x += __shfl_xor(x, o);
    if constexpr (LPR > 64) {
        const int wave = threadIdx.x >> 6, w0 = wave / (LPR / 64) * (LPR / 64);
        if ((threadIdx.x & 63) == 0) lds[buf][wave] = x;
        __syncthreads();
        x = (lds[buf][w0] + lds[buf][w0 + 1]) + (lds[buf][w0 + 2] + lds[buf][w0 + 3]);
        if constexpr (LPR == 512) x += (lds[buf][4] + lds[buf][5]) + (lds[buf][6] + lds[buf][7]);
        buf ^= 1;
    }
    return x;
}

// `reps` times RU rows per group of LPR lanes share one load of the weights.
template <typename XT, typename YT, int VEC, int LPR, int K, int RU>
__global__ void __launch_bounds__(256) norm_kernel(const NormParams p, int reps)
{
    constexpr int RPW = 256 / LPR;  // rows of a workgroup side by side
    __shared__ float lds[2][4];
    int buf = 0;
    const int l = threadIdx.x % LPR, w = p.width;
    const float inv_w = 1.f / (float)w;
    float g[K][VEC], b[K][VEC];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (k * LPR + l) * VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i) g[k][i] = 1.f, b[k][i] = 0.f;
        if (c < w) {
            if (p.gamma) load<VEC>(p.gamma + c, g[k]);
            if (p.beta) load<VEC>(p.beta + c, b[k]);
        }
    }
    int64_t r0 = (int64_t)blockIdx.x * reps * RU * RPW;
    for (int rep = 0; rep < reps && r0 < p.rows; ++rep, r0 += RU * RPW) {
        float v[RU][K][VEC], mean[RU], rstd[RU];
#pragma unroll
        for (int j = 0; j < RU; ++j) {
            // (Lanes of a row that is past the end run along with the last row: its sums need them.)
            const int64_t r = min(r0 + j * RPW + threadIdx.x / LPR, p.rows - 1);
            const XT *x = static_cast<const XT *>(p.x) + r * p.x_stride;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = (k * LPR + l) * VEC;
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[j][k][i] = 0.f;
                if (c < w) load<VEC>(x + c, v[j][k]);
            }
        }
#pragma unroll
        for (int j = 0; j < RU; ++j) {
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < VEC; ++i) s += v[j][k][i];
            mean[j] = row_sum<LPR>(s, lds, buf) * inv_w;
        }
#pragma unroll
        for (int j = 0; j < RU; ++j) {
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const bool in = (k * LPR + l) * VEC < w;
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    v[j][k][i] = in ? v[j][k][i] - mean[j] : 0.f;
                    s = fmaf(v[j][k][i], v[j][k][i], s);
                }
            }
            rstd[j] = 1.f / sqrtf(row_sum<LPR>(s, lds, buf) * inv_w + p.eps);
        }
#pragma unroll
        for (int j = 0; j < RU; ++j) {
            const int64_t row = r0 + j * RPW + threadIdx.x / LPR;
            if (row >= p.rows) break;
            YT *y = static_cast<YT *>(p.y) + row * p.y_stride;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = (k * LPR + l) * VEC;
                if (c < w) {
                    float o[VEC];
#pragma unroll
                    for (int i = 0; i < VEC; ++i) o[i] = fmaf(v[j][k][i] * rstd[j], g[k][i], b[k][i]);
                    store<VEC>(y + c, o);
                }
            }
            if (l == 0 && p.mean) {
                p.mean[row] = mean[j];
                p.rstd[row] = rstd[j];
            }
        }
    }
}

// Backward. Each group of LPR lanes walks over its rows and keeps its channels' sums of dy xh
// and dy in registers; at the end the workgroup adds its groups' sums in a fixed order and
// leaves them as one row of `part`, or as the result where it is the only one.
constexpr int kBwdThreads = 512, kBwdWaves = kBwdThreads / 64;

// Rows that a group of lanes has in flight: two where that keeps a lane's values of a tensor at
// 16 (400,000 rows of 64 channels 50.6 -> 47.7 us; 175,872 bf16 ones level), or at 8 for a group of
// several waves (7,457 float32 rows of 1,341 59 us with 16, 36 with 8).
constexpr int bwd_rows(int values, int lanes) { return values <= (lanes > 64 ? 4 : 8) ? 2 : 1; }

template <typename XT, typename YT, int VEC, int LPR, int K>
__global__ void __launch_bounds__(kBwdThreads) norm_bwd_kernel(const NormBwdParams p)
{
    constexpr int RPW = kBwdThreads / LPR, RU = bwd_rows(K * VEC, LPR);
    constexpr int SUMS = LPR <= 64 ? kBwdWaves : kBwdThreads / LPR;  // sums of a channel to add up
    constexpr int COLS = (LPR <= 64 ? 64 : LPR) * VEC;
    __shared__ float lds[2][kBwdWaves];
    __shared__ float sums[SUMS][COLS];
    int buf = 0;
    const int l = threadIdx.x % LPR, w = p.width;
    const float inv_w = 1.f / (float)w;
    float g[K][VEC], dg[K][VEC], db[K][VEC];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (k * LPR + l) * VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i) g[k][i] = 1.f, dg[k][i] = 0.f, db[k][i] = 0.f;
        if (c < w && p.gamma) load<VEC>(p.gamma + c, g[k]);
    }
    // (The loop's count is the workgroup's: a workgroup's lanes meet at its barriers.)
    const int64_t step = (int64_t)gridDim.x * RU * RPW;
    for (int64_t r0 = (int64_t)blockIdx.x * RU * RPW; r0 < p.rows; r0 += step) {
        float xh[RU][K][VEC], d[RU][K][VEC], s1[RU], s2[RU], mean[RU], rstd[RU];
#pragma unroll
        for (int j = 0; j < RU; ++j) {
            const int64_t r = min(r0 + j * RPW + threadIdx.x / LPR, p.rows - 1);
            const XT *x = static_cast<const XT *>(p.x) + r * p.x_stride;
            const YT *dy = static_cast<const YT *>(p.dy) + r * p.y_stride;
            mean[j] = p.mean[r];
            rstd[j] = p.rstd[r];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = (k * LPR + l) * VEC;
#pragma unroll
                for (int i = 0; i < VEC; ++i) xh[j][k][i] = mean[j], d[j][k][i] = 0.f;
                if (c < w) {
                    load<VEC>(x + c, xh[j][k]);
                    load<VEC>(dy + c, d[j][k]);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < RU; ++j) {
            const bool real = r0 + j * RPW + threadIdx.x / LPR < p.rows;
            s1[j] = s2[j] = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    xh[j][k][i] = (xh[j][k][i] - mean[j]) * rstd[j];
                    if (real) {
                        dg[k][i] = fmaf(d[j][k][i], xh[j][k][i], dg[k][i]);
                        db[k][i] += d[j][k][i];
                    }
                    d[j][k][i] *= g[k][i];
                    s1[j] += d[j][k][i];
                    s2[j] = fmaf(d[j][k][i], xh[j][k][i], s2[j]);
                }
        }
#pragma unroll
        for (int j = 0; j < RU; ++j) {
            s1[j] = row_sum<LPR>(s1[j], lds, buf) * inv_w;
            s2[j] = row_sum<LPR>(s2[j], lds, buf) * inv_w;
        }
#pragma unroll
        for (int j = 0; j < RU; ++j) {
            const int64_t row = r0 + j * RPW + threadIdx.x / LPR;
            if (row >= p.rows) break;
            XT *dx = static_cast<XT *>(p.dx) + row * p.x_stride;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = (k * LPR + l) * VEC;
                if (c < w) {
                    float o[VEC];
#pragma unroll
                    for (int i = 0; i < VEC; ++i) o[i] = rstd[j] * (d[j][k][i] - s1[j] - xh[j][k][i] * s2[j]);
                    store<VEC>(dx + c, o);
                }
            }
        }
    }
    if (!p.part) return;
    const bool only = gridDim.x == 1;
    float *part = p.part + (size_t)blockIdx.x * 2 * w;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (k * LPR + l) * VEC;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float *to = only ? (t ? p.dbeta : p.dgamma) : part + t * w;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                float a = t ? db[k][i] : dg[k][i];
#pragma unroll
                for (int o = LPR; o < 64; o <<= 1) a += __shfl_xor(a, o);  // rows that share the wave
                if (LPR > 64 || (threadIdx.x & 63) < LPR) sums[threadIdx.x / (LPR > 64 ? LPR : 64)][l * VEC + i] = a;
            }
            __syncthreads();
            if (threadIdx.x < LPR && c < w && to)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    float a = 0.f;
#pragma unroll
                    for (int n = 0; n < SUMS; ++n) a += sums[n][l * VEC + i];
                    to[c + i] = a;
                }
        }
    }
}

// The rows of `part` added in order: 16 columns by 64 row groups a workgroup.
__global__ void __launch_bounds__(1024) norm_join_kernel(const float *part, int parts, int width, float *dgamma,
                                                         float *dbeta)
{
    __shared__ float lds[64][17];
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), gr = threadIdx.x >> 4;
    float s = 0.f;
    if (c < 2 * width)
#pragma unroll 8
        for (int r = gr; r < parts; r += 64) s += part[(size_t)r * 2 * width + c];
    lds[gr][threadIdx.x & 15] = s;
    __syncthreads();
    if (gr < 8) {
        s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += lds[gr * 8 + i][threadIdx.x & 15];
    }
    __syncthreads();
    if (gr < 8) lds[gr][threadIdx.x & 15] = s;
    __syncthreads();
    if (gr == 0 && c < 2 * width) {
        s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += lds[i][threadIdx.x];
        if (c < width) {
            if (dgamma) dgamma[c] = s;
        } else if (dbeta) {
            dbeta[c - width] = s;
        }
    }
}

bool multiple(const void *p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

template <typename XT, typename YT, int VEC, int LPR, int K, int RU>
hipError_t go_rows(const NormParams &p, hipStream_t s)
{
    constexpr int64_t SET = 256 / LPR * RU;  // rows a workgroup has in flight
    // Turns per load of the weights: as many as leave 2,048 workgroups, 8 a CU, up to 8 (more
    // only to keep the grid below 2^23 workgroups).
    const int64_t sets = (p.rows + SET - 1) / SET;
    const int64_t even = sets / 2048, least = (sets + (1 << 23) - 1) >> 23;
    int64_t reps = even < 1 ? 1 : even > 8 ? 8 : even;
    if (reps < least) reps = least;
    const int64_t grid = (sets + reps - 1) / reps;
    hipLaunchKernelGGL((norm_kernel<XT, YT, VEC, LPR, K, RU>), dim3((unsigned)grid), dim3(256), 0, s, p, (int)reps);
    return hipGetLastError();
}

// Two rows of float32 in flight where that still leaves workgroups for two fillings of the chip
// (43,968 rows of 1,024 channels 55.0 -> 52.1 us; 100,000 bf16 ones 88.8 -> 100.3).
template <typename XT, typename YT, int VEC, int LPR, int K>
hipError_t go(const NormParams &p, hipStream_t s)
{
    if constexpr (sizeof(XT) == 4 && K * VEC <= 16) {
        if (p.rows >= (int64_t)256 / LPR * 2 * 4096) return go_rows<XT, YT, VEC, LPR, K, 2>(p, s);
    }
    return go_rows<XT, YT, VEC, LPR, K, 1>(p, s);
}

template <typename XT, typename YT, int VEC, int LPR, int K>
hipError_t go(const NormBwdParams &p, hipStream_t s)
{
    constexpr int64_t SET = kBwdThreads / LPR * bwd_rows(K * VEC, LPR);
    const int64_t sets = (p.rows + SET - 1) / SET;
    const int grid = (int)(sets < p.parts ? sets : p.parts);
    hipLaunchKernelGGL((norm_bwd_kernel<XT, YT, VEC, LPR, K>), dim3(grid), dim3(kBwdThreads), 0, s, p);
    if (hipError_t e = hipGetLastError()) return e;
    if (p.part && grid > 1) {
        hipLaunchKernelGGL(norm_join_kernel, dim3((2 * p.width + 15) / 16), dim3(1024), 0, s, p.part, grid, p.width,
                           p.dgamma, p.dbeta);
        return hipGetLastError();
    }
    return hipSuccess;
}

// Rows of K chunks in 256 lanes, or backward in 512 where a lane would hold 32 values and more of
// each tensor (10 million float32 channels: rows of 16,384 202 -> 54 us, of 16,383 303 -> 130, of 8,179
// 85 -> 59), or 16 and more with rows enough for a few a workgroup (4,878 rows of 2,050 44 -> 34, but
// 487 14 -> 18: twice the partial sums).
template <typename XT, typename YT, int VEC, int K, typename P>
hipError_t wide(const P &p, hipStream_t s)
{
    if constexpr (std::is_same<P, NormBwdParams>::value && K * VEC >= 32) {
        return go<XT, YT, VEC, 512, K / 2>(p, s);
    } else {
        if constexpr (std::is_same<P, NormBwdParams>::value && K * VEC >= 16)
            if (p.rows >= 2048) return go<XT, YT, VEC, 512, K / 2>(p, s);
        return go<XT, YT, VEC, 256, K>(p, s);
    }
}

// The lanes and chunks that hold a row: few lanes left over, and several chunks a lane, which
// keep more loads in flight and add up in fewer steps; narrow chunks want more of them (10 million
// float32 channels, forward / backward us: rows of 257 in 256 lanes of 2 40 / 67, in 64 of 5
// 15 / 33; of 41 in 64 lanes of 1 42 / 60, in 16 of 3 16 / 33; of 701 in 256 of 4 20 / 39, in 64 of 12
// 15 / 31; but of 1,001 in 256 of 4 16 / 35, in 64 of 16 - / 48: the registers leave few waves).
template <typename XT, typename YT, int VEC, typename P>
hipError_t by_width(const P &p, hipStream_t s)
{
    const int n = (p.width + VEC - 1) / VEC;
    if (n <= 8) return go<XT, YT, VEC, 8, 1>(p, s);
    if (n <= 16) return go<XT, YT, VEC, 16, 1>(p, s);
    if constexpr (VEC <= 2) {
        if (n <= 24) return go<XT, YT, VEC, 8, 3>(p, s);
        if (n <= 32) return go<XT, YT, VEC, 8, 4>(p, s);
        if (n <= 48) return go<XT, YT, VEC, 16, 3>(p, s);
        if (n <= 64) return go<XT, YT, VEC, 16, 4>(p, s);
        if (n <= 96) return go<XT, YT, VEC, 32, 3>(p, s);
        if (n <= 128) return go<XT, YT, VEC, 32, 4>(p, s);
        if (n <= 160) return go<XT, YT, VEC, 32, 5>(p, s);
        if (n <= 192) return go<XT, YT, VEC, 32, 6>(p, s);
        if (n <= 256) return go<XT, YT, VEC, 64, 4>(p, s);
        if (n <= 320) return go<XT, YT, VEC, 64, 5>(p, s);
        if (n <= 384) return go<XT, YT, VEC, 64, 6>(p, s);
        if (n <= 512) return go<XT, YT, VEC, 64, 8>(p, s);
        if constexpr (VEC == 1) {
            if (n <= 768) return go<XT, YT, VEC, 64, 12>(p, s);
        }
    } else {
        if (n <= 32) return go<XT, YT, VEC, 32, 1>(p, s);
        if (n <= 64) return go<XT, YT, VEC, 64, 1>(p, s);
        if (n <= 96) return go<XT, YT, VEC, 32, 3>(p, s);
        if (n <= 128) return go<XT, YT, VEC, 64, 2>(p, s);
        if (n <= 192) return go<XT, YT, VEC, 64, 3>(p, s);
        if (n <= 256) return go<XT, YT, VEC, 64, 4>(p, s);
        if (n <= 512) return go<XT, YT, VEC, 256, 2>(p, s);
    }
    if (n <= 1024) return go<XT, YT, VEC, 256, 4>(p, s);
    if (n <= 2048) return wide<XT, YT, VEC, 8>(p, s);
    if constexpr (VEC <= 4) {
        if (n <= 4096) return wide<XT, YT, VEC, 16>(p, s);
    }
    if constexpr (VEC <= 2) {
        if (n <= 8192) return wide<XT, YT, VEC, 32>(p, s);
    }
    if constexpr (VEC == 1) return wide<XT, YT, VEC, 64>(p, s);
    return hipErrorInvalidValue;  // (not reached: RESS_MAX_NORM_WIDTH)
}

// Whole 16-byte chunks of the wider type everywhere, or pairs, or single channels (10,992 rows
// of 770 bf16 channels 27 us as singles).
template <typename XT, typename YT, typename P>
hipError_t by_alignment(const P &p, const void *xs, const void *xs2, const void *ys, const float *w1, const float *w2,
                        hipStream_t s)
{
    constexpr int V = 16 / (sizeof(XT) > sizeof(YT) ? sizeof(XT) : sizeof(YT));
    auto whole = [&](size_t v) {
        return p.width % v == 0 && p.x_stride % v == 0 && p.y_stride % v == 0 && multiple(xs, v * sizeof(XT)) &&
               multiple(xs2, v * sizeof(XT)) && multiple(ys, v * sizeof(YT)) && multiple(w1, v * sizeof(float)) &&
               multiple(w2, v * sizeof(float));
    };
    return whole(V) ? by_width<XT, YT, V>(p, s) : whole(2) ? by_width<XT, YT, 2>(p, s) : by_width<XT, YT, 1>(p, s);
}

template <typename P>
hipError_t by_type(const P &p, const void *xs, const void *xs2, const void *ys, const float *w1, const float *w2,
                   hipStream_t s)
{
    if (p.x_f32)
        return p.y_f32 ? by_alignment<float, float>(p, xs, xs2, ys, w1, w2, s)
                       : by_alignment<float, uint16_t>(p, xs, xs2, ys, w1, w2, s);
    return p.y_f32 ? by_alignment<uint16_t, float>(p, xs, xs2, ys, w1, w2, s)
                   : by_alignment<uint16_t, uint16_t>(p, xs, xs2, ys, w1, w2, s);
}

}  // namespace

hipError_t launch_norm(const NormParams &p, hipStream_t s) { return by_type(p, p.x, p.x, p.y, p.gamma, p.beta, s); }

hipError_t launch_norm_bwd(const NormBwdParams &p, hipStream_t s)
{
    if (p.rows == 0) {  // no row has a part in the sums
        hipLaunchKernelGGL(norm_join_kernel, dim3((2 * p.width + 15) / 16), dim3(1024), 0, s, p.part, 0, p.width, p.dgamma,
                           p.dbeta);
        return hipGetLastError();
    }
    return by_type(p, p.x, p.dx, p.dy, p.gamma, p.gamma, s);
}

}  // namespace ress
