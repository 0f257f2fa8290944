// Layer norm over the channels of a row, forward and backward.
//
// Both passes are memory bound: a row is read into registers once, its sums are
// taken there (the variance from centred values, so that a large mean costs no
// digits), and the result is written from the same registers. A row belongs to LPR
// lanes, each with K chunks of VEC neighbouring channels: narrow rows share a wave
// (8 rows of 64 bf16 channels), ordinary ones take a wave, wide ones a workgroup.
// VEC is what fills 16 bytes of the wider of the two types; rows whose width, strides
// or addresses are not multiples of that take one channel at a time.
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

constexpr int kThreads = 256;

// Sum over the LPR lanes of a row, the same in each of them. Rows of a workgroup
// exchange through LDS; `buf` alternates, so that one barrier a sum is enough.
template <int LPR>
__device__ __forceinline__ float row_sum(float x, float (&lds)[2][4], int &buf)
{
#pragma unroll
    for (int o = 1; o < (LPR < 64 ? LPR : 64); o <<= 1) x += __shfl_xor(x, o);
    if constexpr (LPR > 64) {
        if ((threadIdx.x & 63) == 0) lds[buf][threadIdx.x >> 6] = x;
        __syncthreads();
        x = (lds[buf][0] + lds[buf][1]) + (lds[buf][2] + lds[buf][3]);
        buf ^= 1;
    }
    return x;
}

// `reps` rows per group of LPR lanes share one load of the weights.
template <typename XT, typename YT, int VEC, int LPR, int K>
__global__ void __launch_bounds__(kThreads) norm_kernel(const NormParams p, int reps)
{
    constexpr int RPW = kThreads / LPR;  // rows of a workgroup at a time
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
    int64_t r = (int64_t)blockIdx.x * reps * RPW + threadIdx.x / LPR;
    for (int rep = 0; rep < reps; ++rep, r += RPW) {
        // (Lanes of a row that is past the end run along with the last row: its sums need them.)
        if (r - threadIdx.x / LPR >= p.rows) break;
        const bool real = r < p.rows;
        const int64_t row = real ? r : p.rows - 1;
        const XT *x = static_cast<const XT *>(p.x) + row * p.x_stride;
        float v[K][VEC];
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * LPR + l) * VEC;
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[k][i] = 0.f;
            if (c < w) load<VEC>(x + c, v[k]);
        }
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < VEC; ++i) s += v[k][i];
        const float mean = row_sum<LPR>(s, lds, buf) * inv_w;
        float s2 = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const bool in = (k * LPR + l) * VEC < w;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                v[k][i] = in ? v[k][i] - mean : 0.f;
                s2 = fmaf(v[k][i], v[k][i], s2);
            }
        }
        const float rstd = 1.f / sqrtf(row_sum<LPR>(s2, lds, buf) * inv_w + p.eps);
        if (!real) continue;
        YT *y = static_cast<YT *>(p.y) + row * p.y_stride;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * LPR + l) * VEC;
            if (c < w) {
                float o[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) o[i] = fmaf(v[k][i] * rstd, g[k][i], b[k][i]);
                store<VEC>(y + c, o);
            }
        }
        if (l == 0 && p.mean) {
            p.mean[row] = mean;
            p.rstd[row] = rstd;
        }
    }
}

// Backward. Each group of LPR lanes walks over its rows (row, row + parts RPW, ...) and
// keeps its channels' sums of dy xh and dy in registers; at the end the workgroup adds
// its groups' sums in a fixed order and leaves them as one row of `part`.
template <typename XT, typename YT, int VEC, int LPR, int K>
__global__ void __launch_bounds__(kThreads) norm_bwd_kernel(const NormBwdParams p)
{
    constexpr int RPW = kThreads / LPR;
    __shared__ float lds[2][4];
    __shared__ float sums[4][64 * VEC];
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
    const int64_t step = (int64_t)gridDim.x * RPW;
    for (int64_t r0 = (int64_t)blockIdx.x * RPW; r0 < p.rows; r0 += step) {
        const int64_t r = r0 + threadIdx.x / LPR;
        const bool real = r < p.rows;
        const int64_t row = real ? r : p.rows - 1;
        const XT *x = static_cast<const XT *>(p.x) + row * p.x_stride;
        const YT *dy = static_cast<const YT *>(p.dy) + row * p.y_stride;
        const float mean = p.mean[row], rstd = p.rstd[row];
        float xh[K][VEC], d[K][VEC];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * LPR + l) * VEC;
#pragma unroll
            for (int i = 0; i < VEC; ++i) xh[k][i] = mean, d[k][i] = 0.f;
            if (c < w) {
                load<VEC>(x + c, xh[k]);
                load<VEC>(dy + c, d[k]);
            }
        }
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                xh[k][i] = (xh[k][i] - mean) * rstd;
                if (real) {
                    dg[k][i] = fmaf(d[k][i], xh[k][i], dg[k][i]);
                    db[k][i] += d[k][i];
                }
                d[k][i] *= g[k][i];
                s1 += d[k][i];
                s2 = fmaf(d[k][i], xh[k][i], s2);
            }
        s1 = row_sum<LPR>(s1, lds, buf) * inv_w;
        s2 = row_sum<LPR>(s2, lds, buf) * inv_w;
        if (!real) continue;
        XT *dx = static_cast<XT *>(p.dx) + row * p.x_stride;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * LPR + l) * VEC;
            if (c < w) {
                float o[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) o[i] = rstd * (d[k][i] - s1 - xh[k][i] * s2);
                store<VEC>(dx + c, o);
            }
        }
    }
    if (!p.part) return;
    float *part = p.part + (size_t)blockIdx.x * 2 * w;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (k * LPR + l) * VEC;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float a[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                a[i] = t ? db[k][i] : dg[k][i];
#pragma unroll
                for (int o = LPR; o < 64; o <<= 1) a[i] += __shfl_xor(a[i], o);  // rows that share the wave
            }
            if constexpr (LPR <= 64) {
                __syncthreads();
                if ((threadIdx.x & 63) < LPR)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) sums[threadIdx.x >> 6][l * VEC + i] = a[i];
                __syncthreads();
                if (threadIdx.x < LPR && c < w)
#pragma unroll
                    for (int i = 0; i < VEC; ++i)
                        part[t * w + c + i] = (sums[0][l * VEC + i] + sums[1][l * VEC + i]) +
                                              (sums[2][l * VEC + i] + sums[3][l * VEC + i]);
            } else if (c < w) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) part[t * w + c + i] = a[i];
            }
        }
    }
}

// The rows of `part` added in order: 16 columns by 16 row groups a workgroup.
__global__ void __launch_bounds__(256) norm_join_kernel(const float *part, int parts, int width, float *dgamma,
                                                        float *dbeta)
{
    __shared__ float lds[16][17];
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), gr = threadIdx.x >> 4;
    float s = 0.f;
    if (c < 2 * width)
#pragma unroll 8
        for (int r = gr; r < parts; r += 16) s += part[(size_t)r * 2 * width + c];
    lds[gr][threadIdx.x & 15] = s;
    __syncthreads();
    if (gr == 0 && c < 2 * width) {
        s = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += lds[i][threadIdx.x];
        if (c < width) {
            if (dgamma) dgamma[c] = s;
        } else if (dbeta) {
            dbeta[c - width] = s;
        }
    }
}

bool multiple(const void *p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

template <typename XT, typename YT, int VEC, int LPR, int K>
hipError_t go(const NormParams &p, hipStream_t s)
{
    constexpr int RPW = kThreads / LPR;
    // Rows per load of the weights: as many as leave 2,048 workgroups, 8 a CU, up to 8
    // (more only to keep the grid below 2^23 workgroups).
    const int64_t sets = (p.rows + RPW - 1) / RPW;
    const int64_t even = sets / 2048, least = (sets + (1 << 23) - 1) >> 23;
    int64_t reps = even < 1 ? 1 : even > 8 ? 8 : even;
    if (reps < least) reps = least;
    const int64_t grid = (sets + reps - 1) / reps;
    hipLaunchKernelGGL((norm_kernel<XT, YT, VEC, LPR, K>), dim3((unsigned)grid), dim3(kThreads), 0, s, p, (int)reps);
    return hipGetLastError();
}

template <typename XT, typename YT, int VEC, int LPR, int K>
hipError_t go(const NormBwdParams &p, hipStream_t s)
{
    constexpr int RPW = kThreads / LPR;
    const int64_t sets = (p.rows + RPW - 1) / RPW;
    const int grid = (int)(sets < p.parts ? sets : p.parts);
    hipLaunchKernelGGL((norm_bwd_kernel<XT, YT, VEC, LPR, K>), dim3(grid), dim3(kThreads), 0, s, p);
    if (hipError_t e = hipGetLastError()) return e;
    if (p.part) {
        hipLaunchKernelGGL(norm_join_kernel, dim3((2 * p.width + 15) / 16), dim3(256), 0, s, p.part, grid, p.width,
                           p.dgamma, p.dbeta);
        return hipGetLastError();
    }
    return hipSuccess;
}

// The lanes and chunks that hold a row.
template <typename XT, typename YT, int VEC, typename P>
hipError_t by_width(const P &p, hipStream_t s)
{
    const int n = (p.width + VEC - 1) / VEC;
    if (n <= 8) return go<XT, YT, VEC, 8, 1>(p, s);
    if (n <= 16) return go<XT, YT, VEC, 16, 1>(p, s);
    if (n <= 32) return go<XT, YT, VEC, 32, 1>(p, s);
    if (n <= 64) return go<XT, YT, VEC, 64, 1>(p, s);
    if (n <= 128) return go<XT, YT, VEC, 64, 2>(p, s);
    if (n <= 256) return go<XT, YT, VEC, 64, 4>(p, s);
    if (n <= 512) return go<XT, YT, VEC, 256, 2>(p, s);
    if (n <= 1024) return go<XT, YT, VEC, 256, 4>(p, s);
    if (n <= 2048) return go<XT, YT, VEC, 256, 8>(p, s);
    if constexpr (VEC <= 4) {
        if (n <= 4096) return go<XT, YT, VEC, 256, 16>(p, s);
    }
    if constexpr (VEC == 1) return go<XT, YT, VEC, 256, 64>(p, s);
    return hipErrorInvalidValue;  // (not reached: RESS_MAX_NORM_WIDTH)
}

// Whole 16-byte chunks of the wider type everywhere, or single channels.
template <typename XT, typename YT, typename P>
hipError_t by_alignment(const P &p, const void *xs, const void *xs2, const void *ys, const float *w1, const float *w2,
                        hipStream_t s)
{
    constexpr int V = 16 / (sizeof(XT) > sizeof(YT) ? sizeof(XT) : sizeof(YT));
    const bool whole = p.width % V == 0 && p.x_stride % V == 0 && p.y_stride % V == 0 && multiple(xs, V * sizeof(XT)) &&
                       multiple(xs2, V * sizeof(XT)) && multiple(ys, V * sizeof(YT)) && multiple(w1, V * sizeof(float)) &&
                       multiple(w2, V * sizeof(float));
    return whole ? by_width<XT, YT, V>(p, s) : by_width<XT, YT, 1>(p, s);
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

// 512 rows of partial sums of 1,024 channels are 4 MB; no more than 1,024 rows, no
// fewer than a workgroup a CU.
int norm_bwd_parts(int64_t rows, int width)
{
    const int most = width <= 512 ? 1024 : 512;
    return (int)(rows < most ? (rows < 1 ? 1 : rows) : most);
}

hipError_t launch_norm(const NormParams &p, hipStream_t s) { return by_type(p, p.x, p.x, p.y, p.gamma, p.beta, s); }

hipError_t launch_norm_bwd(const NormBwdParams &p, hipStream_t s)
{
    if (p.rows == 0) {  // no row has a part in the sums
        hipLaunchKernelGGL(norm_join_kernel, dim3((2 * p.width + 15) / 16), dim3(256), 0, s, p.part, 0, p.width, p.dgamma,
                           p.dbeta);
        return hipGetLastError();
    }
    return by_type(p, p.x, p.dx, p.dy, p.gamma, p.gamma, s);
}

}  // namespace ress
