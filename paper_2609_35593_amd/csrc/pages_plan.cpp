// How the kernels of ress_pages.h spread over the chip: functions of a shape alone. Plain host code,
// apart from the kernels, so that it runs without a GPU.
#include "pages_internal.h"

namespace ress {

HeadBwdPlan head_bwd_plan(int H_all, int N, int tokens_each)
{
    HeadBwdPlan r = {0, 0, 0};
    if (H_all == 0 || N == 0) return r;
    // Workgroups over tokens, and over heads while there are few.
    const int64_t tokens = ((int64_t)N + tokens_each - 1) / tokens_each;
    r.tokens = (int)(tokens < kHeadParts ? tokens : kHeadParts);
    int cuts = kHeadParts / r.tokens;
    if (cuts > H_all) cuts = H_all;
    r.heads = (H_all + cuts - 1) / cuts;
    r.parts = r.tokens * ((H_all + r.heads - 1) / r.heads);
    return r;
}

int head_bwd_parts(int H_all, int N)
{
    const int64_t rows = (int64_t)H_all * N;
    return (int)(rows < 1 ? 1 : rows < kHeadParts ? rows : kHeadParts);
}

PagedPlan paged_plan(const ress_paged_shape *s)
{
    PagedPlan r = {32, 0, 1};
    if (s->B == 0 || s->N == 0 || s->H == 0) return r;
    const int64_t group = s->H / s->H_kv, rows = s->N * group, some = s->B < s->N ? s->B : s->N;
    // Blocks of 128 rows where sequences have more than 32 on average.
    if (rows > 32 * some) r.rows = 128;
    // A sequence leaves at most one block that is not full.
    r.blocks = (int)((rows + some * (r.rows - 1)) / r.rows);
    const int64_t capacity = (int64_t)s->max_pages * s->page;
    int64_t keys = window_tokens(s->frame, s->window) + s->n_sink + r.rows / group;
    if (keys > capacity) keys = capacity;
    // Keys are cut over workgroups, of kTileLeast or kWideLeast tiles at least, while there are few blocks. (us by workgroups that share
    // a block. 128 rows: 176 blocks of 687 tiles 1 / 5 / 8 / 16 793 / 342 / 333 / 313; 512 of up to 64, 1 / 4 / 16 104 / 90 / 93;
    // 128 of 31, 1 / 3 43 / 38; but 176 of 21, 1 / 2 32 / 41. 32 rows: 192 blocks of 47 tiles 1 / 2 / 4 31.7 / 34.9 / 38.0, 384 55 /
    // 58 / 62, 4 of 688, 16 / 32 / 64 33 / 25 / 24.)
    const int64_t tiles = (keys + 63) / 64, blocks = (int64_t)r.blocks * s->H_kv;
    const int64_t most = r.rows == 32 ? tiles / kTileLeast : tiles < 24 ? 1 : tiles / kWideLeast;
    const int64_t want = (r.rows == 32 ? 256 : 2816) / blocks, n = want < most ? want : most;
    r.splits = (int)(n < 1 ? 1 : n > kMaxPagedSplits ? kMaxPagedSplits : n);
    return r;
}

}  // namespace ress
