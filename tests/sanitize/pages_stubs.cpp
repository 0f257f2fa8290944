// Launchers that do nothing, for the CPU tests of ress_pages.h's C ABI and plans (pages_api.cpp and pages_plan.cpp, linked
// with them as they are), and the plans by C names. A call that passes every check ends in a launcher here, whose
// error it returns; what the kernels take for granted of their parameters is looked at on the way.
#include <stdlib.h>

#include "pages_internal.h"

namespace ress {
namespace {
void must(bool ok)
{
    if (!ok) abort();
}
// Every chunk's pairs and the chunk that they meet, as the tables of single pairs have them.
void check_runs(const RopeParams &r, const ChunkRuns &runs)
{
    if (r.chunk == 0) return;
    must(r.D % r.chunk == 0 && r.D / r.chunk <= kMaxChunks && runs.n >= 1 && runs.n <= RESS_MAX_ROPE_AXES);
    for (int c = 0; c * r.chunk < r.D; ++c) {
        int other = c, pair = 0;
        for (int a = 0; a < runs.n; ++a) {
            const int at = c - runs.first[a], half = runs.half[a];
            if (at < 0 || at >= runs.count[a]) continue;
            const bool second = half > 0 && at >= half;
            other = second ? c - half : c + half;
            pair = runs.pair[a] + (half > 0 ? (second ? at - half : at) * r.chunk : at * (r.chunk / 2));
        }
        if (c * r.chunk >= r.turned) {
            must(other == c);
            continue;
        }
        must(other >= 0 && other * r.chunk < r.turned && pair >= 0);
        for (int e = 0; e < (r.interleaved ? r.chunk / 2 : r.chunk); ++e) {
            const int a = r.ca[pair + e], b = r.cb[pair + e];
            must(r.turns[pair + e] >= 0.0);
            if (r.interleaved)
                must(a == c * r.chunk + 2 * e && b == a + 1 && other == c);
            else
                must((other > c ? a : b) == c * r.chunk + e && (other > c ? b : a) == other * r.chunk + e);
        }
    }
}
}  // namespace

hipError_t launch_head_norm(const HeadNormParams &p, hipStream_t)
{
    check_runs(p.r, p.runs);
    must(p.r.N > 0 && p.r.H_all > 0 && (!p.slots || (p.page >= 1 && p.n_slots >= 0)));
    return hipErrorInvalidValue;
}
hipError_t launch_head_norm_bwd(const HeadNormBwdParams &p, hipStream_t)
{
    check_runs(p.r, p.runs);
    return hipErrorInvalidValue;
}
hipError_t launch_tables(const TableParams &p, hipStream_t)
{
    must(p.page >= 1 && (int64_t)p.max_pages * p.page <= RESS_MAX_TOKENS && (int64_t)p.n_pages * p.page <= 0x7fffffff);
    return hipErrorInvalidValue;
}
hipError_t launch_release(const ReleaseParams &, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_paged(const PagedParams &p, int rows, hipStream_t)
{
    const int64_t all = (int64_t)p.N * p.group, some = p.B < p.N ? p.B : p.N;
    must(rows == 32 || rows == 128);
    must(p.blocks >= (all + rows - 1) / rows && p.blocks <= all / rows + some + 1);
    // Grids: below 2^32 threads in a dimension, and ids that fit 31 bits.
    must(rows == 128 || (int64_t)p.blocks * 256 < ((int64_t)1 << 32));
    must((int64_t)p.H_kv * p.blocks < 0x7ffffff0 && p.splits >= 1 && p.splits <= kMaxPagedSplits && p.H_kv <= 65535);
    must(p.splits == 1 || (p.part && p.part_row && (rows == 128 || p.cuts)));
    must((int64_t)p.window * p.frame < ((int64_t)1 << 28));
    return hipErrorInvalidValue;
}
}  // namespace ress

extern "C" {
void plan_paged(const ress_paged_shape *s, int *out)
{
    const ress::PagedPlan p = ress::paged_plan(s);
    out[0] = p.rows, out[1] = p.blocks, out[2] = p.splits, out[3] = p.parts, out[4] = p.target;
}
void plan_head_bwd(int H_all, int N, int tokens_each, int *out)
{
    const ress::HeadBwdPlan p = ress::head_bwd_plan(H_all, N, tokens_each);
    out[0] = p.tokens, out[1] = p.heads, out[2] = p.parts, out[3] = ress::head_bwd_parts(H_all, N);
}
}
