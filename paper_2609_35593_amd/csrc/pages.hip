// Pages of a step: tables, slots and positions from request lengths, and pages given back.
//
// Latency: a step moves kilobytes. What depends on every sequence before it, their sums of
// tokens and of pages, is one pass of one workgroup over the sequences; the lists of tokens
// are written by that workgroup where they are short, else by a second launch that finds a token's
// sequence by bisection in cu_q.
//
// Measured: 256 sequences of one new token 5.4 us (lengths, scan, pages, lists: four trips to memory, five barriers of 16 waves), 47 of 1,374
// tokens each 6.8 and 1.9 for their 65,538 slots and positions. Pages given back by 64 sequences: 3.0 us for the counts, 4.1 for
// the stack (a launch between, because a stack's height depends on every sequence before).
#include "pages_internal.h"
#include "scan.h"

namespace ress {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kMost = 1 << 28;  // sums of tokens, and of pages for them, stop here (more than any N takes, less than 2^31 with one more)

// Tokens and pages, whose sums stop at kMost. (The least of a sum and a bound: associative, so the order of a scan is free.)
struct Need {
    int tokens, pages;
};
__device__ __forceinline__ int sum_of(int a, int b) { return min(a + b, kMost); }
__device__ __forceinline__ Need operator+(Need a, Need b) { return {sum_of(a.tokens, b.tokens), sum_of(a.pages, b.pages)}; }
__device__ __forceinline__ Need scan_needs(Need x) { return {scan_wave(x.tokens, sum_of), scan_wave(x.pages, sum_of)}; }

// The last of [0, n) whose entry of the ascending list is at most x (list[0] <= x).
__device__ __forceinline__ int last_at_most(const int *list, int n, int x)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (list[mid] <= x)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

__device__ __forceinline__ int pages_for(const TableParams &p, int tokens)
{
    return tokens == 0 ? 0 : p.pages(tokens - 1) + 1;
}

// One workgroup, kThreads sequences a turn.
__global__ void __launch_bounds__(kThreads) step_kernel(const TableParams p, bool lists)
{
    __shared__ Need waves[kWaves], ends[kWaves];
    __shared__ int first_token[kThreads], first_page[kThreads], len_of[kThreads];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int capacity = p.max_pages * p.page, n_free = min(max(p.n_free[0], 0), p.n_pages);
    Need before = {0, 0};                    // wanted by all sequences up to this turn's
    int tokens = 0, taken = 0, refused = 0;  // given to them; refused sequences of this thread
    for (int b0 = 0; b0 < p.B; b0 += kThreads) {
        const int b = b0 + threadIdx.x;
        int len = 0, want = 0;
        if (b < p.B) {
            len = min(max(p.lens[b], 0), capacity);
            want = max(p.new_lens[b], 0);
        }
        const bool fits = want <= capacity - len;
        Need own = {0, 0};
        if (fits) own = {want, pages_for(p, len + want) - pages_for(p, len)};
        Need sum = scan_needs(own);
        if (lane == 63) waves[wave] = sum;
        __syncthreads();
        Need head = before;
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) head = head + waves[w];
            before = before + waves[w];
        }
        sum = head + sum;
        // The sums ascend, so sequences within the bounds come first, and the last of them has what was given.
        const bool within = sum.tokens <= p.N && sum.pages <= n_free;
        if (want > 0 && !(fits && within)) ++refused;
        const int n_within = __popcll(__ballot(within));
        if (lane == max(n_within - 1, 0)) ends[wave] = within ? sum : Need{0, 0};
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) {
            tokens = max(tokens, ends[w].tokens);
            taken = max(taken, ends[w].pages);
        }
        if (!within) {
            sum = {tokens, taken};
            own = {0, 0};
        }
        if (b < p.B) {
            p.cu_q[b] = sum.tokens - own.tokens;
            p.lens_out[b] = len + own.tokens;
        }
        first_token[threadIdx.x] = sum.tokens - own.tokens;
        first_page[threadIdx.x] = sum.pages - own.pages;
        len_of[threadIdx.x] = len;
        __syncthreads();
        // The turn's pages and tokens, by whoever is free.
        const int n = min(kThreads, p.B - b0);
        for (int j = first_page[0] + (int)threadIdx.x; j < taken; j += kThreads) {
            const int i = last_at_most(first_page, n, j);
            const int entry = pages_for(p, len_of[i]) + j - first_page[i];
            p.tables[(int64_t)(b0 + i) * p.stride + entry] = p.free_pages[n_free - 1 - j];
        }
        if (lists)
            for (int t = first_token[0] + (int)threadIdx.x; t < tokens; t += kThreads) {
                const int i = last_at_most(first_token, n, t);
                const int at = len_of[i] + t - first_token[i], idx = p.pages(at), had_i = pages_for(p, len_of[i]);
                const int page = idx >= had_i ? p.free_pages[n_free - 1 - (first_page[i] + idx - had_i)]
                                              : p.tables[(int64_t)(b0 + i) * p.stride + idx];
                p.pos[t] = at;
                p.slots[t] = (unsigned int)page < (unsigned int)p.n_pages ? page * p.page + (at - idx * p.page) : -1;
            }
        __syncthreads();
    }
    if (lists)
        for (int t = tokens + (int)threadIdx.x; t < p.N; t += kThreads) {
            p.pos[t] = 0;
            p.slots[t] = -1;
        }
    if (p.n_refused) {
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) refused += __shfl_xor(refused, o);
        if (lane == 0) first_token[wave] = refused;
        __syncthreads();
    }
    if (threadIdx.x > 0) return;
    p.cu_q[p.B] = tokens;
    p.n_free_out[0] = n_free - taken;
    if (p.n_refused) {
        int all = 0;
        for (int w = 0; w < kWaves; ++w) all += first_token[w];
        p.n_refused[0] = all;
    }
}

constexpr int kListThreads = 256, kInLds = 4096;

// The lists of tokens behind step_kernel: cu_q, the lengths after the step, and the tables are there.
__global__ void __launch_bounds__(kListThreads) lists_kernel(const TableParams p)
{
    __shared__ int cu[kInLds];
    const bool in_lds = p.B <= kInLds;
    if (in_lds)
        for (int b = threadIdx.x; b < p.B; b += kListThreads) cu[b] = p.cu_q[b];
    const int tokens = p.cu_q[p.B];
    __syncthreads();
    const int t = blockIdx.x * kListThreads + threadIdx.x;
    if (t >= p.N) return;
    if (t >= tokens) {
        p.pos[t] = 0;
        p.slots[t] = -1;
        return;
    }
    const int b = in_lds ? last_at_most(cu, p.B, t) : last_at_most(p.cu_q, p.B, t);
    // (The sequence's last token is at lens_out[b] - 1.)
    const int at = p.lens_out[b] - (p.cu_q[b + 1] - t), idx = p.pages(at);
    const int page = p.tables[(int64_t)b * p.stride + idx];
    p.pos[t] = at;
    p.slots[t] = (unsigned int)page < (unsigned int)p.n_pages ? page * p.page + (at - idx * p.page) : -1;
}

// ----------------------------------------------------------------- release

constexpr int kScan = 1024;  // sequences up to which every workgroup adds up the counts before its own

// Heights of the stack, which stop at 2^31 - 1 (no n_pages is more).
__device__ __forceinline__ uint32_t higher(uint32_t a, uint32_t b) { return min(a + b, 0x7fffffffu); }

__device__ __forceinline__ bool valid(const ReleaseParams &p, int page) { return (unsigned int)page < (unsigned int)p.n_pages; }

// A workgroup a sequence: how many of its entries go back. (The stack's height is kept beside the
// counts: the next launch may write it where it was read.)
__global__ void __launch_bounds__(256) count_kernel(const ReleaseParams p)
{
    __shared__ int waves[4];
    const int b = blockIdx.x;
    const int first = min(max(p.first[b], 0), p.max_pages), last = min(max(p.last[b], 0), p.max_pages);
    const int32_t *row = p.tables + (int64_t)b * p.stride;
    int n = 0;
    for (int i = first + (int)threadIdx.x; i < last; i += 256) n += valid(p, row[i]);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) n += __shfl_xor(n, o);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = n;
    __syncthreads();
    if (threadIdx.x == 0) p.counts[b] = waves[0] + waves[1] + waves[2] + waves[3];
    if (b == 0 && threadIdx.x == 0) p.counts[p.B] = min(max(p.n_free[0], 0), p.n_pages);
}

// Many sequences: counts become the sums before them, by one workgroup.
__global__ void __launch_bounds__(kThreads) sums_kernel(const ReleaseParams p)
{
    __shared__ uint32_t waves[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t before = 0;
    for (int b0 = 0; b0 < p.B; b0 += kThreads) {
        const int b = b0 + threadIdx.x;
        const uint32_t own = b < p.B ? p.counts[b] : 0;
        const uint32_t sum = scan_wave((int)own, [](int a, int b) { return (int)higher(a, b); });
        if (lane == 63) waves[wave] = sum;
        const uint32_t up = __shfl_up(sum, 1);  // (of the lanes before: a sum that stopped tells nothing of what it is without one's own)
        uint32_t head = higher(before, lane ? up : 0);
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) head = higher(head, waves[w]);
            before = higher(before, waves[w]);
        }
        if (b < p.B) p.counts[b] = (int32_t)head;
        __syncthreads();
    }
}

// A workgroup a sequence: its entries onto the stack, in order.
__global__ void __launch_bounds__(256) push_kernel(const ReleaseParams p, bool summed)
{
    __shared__ uint32_t waves[4];
    const int b = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int first = min(max(p.first[b], 0), p.max_pages), last = min(max(p.last[b], 0), p.max_pages);
    int32_t *row = p.tables + (int64_t)b * p.stride;
    uint32_t at = summed && threadIdx.x == 0 ? p.counts[b] : 0;
    if (!summed)
        for (int i = threadIdx.x; i < b; i += 256) at = higher(at, p.counts[i]);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) at = higher(at, __shfl_xor(at, o));
    if (lane == 0) waves[wave] = at;
    __syncthreads();
    at = p.counts[p.B];
    for (int w = 0; w < 4; ++w) at = higher(at, waves[w]);
    for (int i0 = first; i0 < last; i0 += 256) {
        const int i = i0 + (int)threadIdx.x;
        const int page = i < last ? row[i] : -1;
        const bool back = valid(p, page);
        const unsigned long long in_wave = __ballot(back);
        __syncthreads();
        if (lane == 0) waves[wave] = __popcll(in_wave);
        __syncthreads();
        uint32_t to = at + __popcll(in_wave & ((1ull << lane) - 1));
        for (int w = 0; w < 4; ++w) {
            if (w < wave) to += waves[w];
            at = higher(at, waves[w]);
        }
        if (back) {
            if (to < (uint32_t)p.n_pages) p.free_pages[to] = page;
            if (p.clear) row[i] = -1;
        }
    }
    if (b == p.B - 1 && threadIdx.x == 0) p.n_free_out[0] = (int32_t)min(at, (uint32_t)p.n_pages);
}

// No sequences: the stack stays as it is.
__global__ void keep_kernel(const ReleaseParams p) { p.n_free_out[0] = min(max(p.n_free[0], 0), p.n_pages); }

}  // namespace

hipError_t launch_tables(const TableParams &p, hipStream_t s)
{
    const bool lists = p.N <= 4096;
    hipLaunchKernelGGL(step_kernel, dim3(1), dim3(kThreads), 0, s, p, lists);
    if (hipError_t e = hipGetLastError()) return e;
    if (lists) return hipSuccess;
    hipLaunchKernelGGL(lists_kernel, dim3((unsigned)((p.N + kListThreads - 1) / kListThreads)), dim3(kListThreads), 0, s, p);
    return hipGetLastError();
}

hipError_t launch_release(const ReleaseParams &p, hipStream_t s)
{
    if (p.B == 0) {
        hipLaunchKernelGGL(keep_kernel, dim3(1), dim3(1), 0, s, p);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(count_kernel, dim3((unsigned)p.B), dim3(256), 0, s, p);
    if (hipError_t e = hipGetLastError()) return e;
    if (p.B > kScan) {
        hipLaunchKernelGGL(sums_kernel, dim3(1), dim3(kThreads), 0, s, p);
        if (hipError_t e = hipGetLastError()) return e;
    }
    hipLaunchKernelGGL(push_kernel, dim3((unsigned)p.B), dim3(256), 0, s, p, p.B > kScan);
    return hipGetLastError();
}

}  // namespace ress
