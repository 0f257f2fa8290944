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
    PagedPlan r = {32, 0, 1, 0, 0};
    if (s->B == 0 || s->N == 0 || s->H == 0) return r;
    const int64_t group = s->H / s->H_kv, rows = s->N * group, some = s->B < s->N ? s->B : s->N;
    // Blocks of 128 rows where sequences have more than 32 on average, rows that pad the batch counted: the host knows no better, and
    // blocks of 128 rows lose little on sequences that have fewer (single tokens of 24 sequences of 5,000 keys, 16 heads for 4, in 24 /
    // 200 / 1,024 / 4,096 rows: 38 / 40 / 41 / 42 us).
    if (rows > 32 * some) r.rows = 128;
    // A sequence leaves at most one block that is not full.
    r.blocks = (int)((rows + some * (r.rows - 1)) / r.rows);
    const int64_t capacity = (int64_t)s->max_pages * s->page;
    int64_t keys = window_tokens(s->frame, s->window) + s->n_sink + r.rows / group;
    if (keys > capacity) keys = capacity;
    const int64_t tiles = (keys + 63) / 64, n = (int64_t)r.blocks * s->H_kv;
    int64_t want, most;
    if (r.rows == 32) {
        // Parts by keys (see find_part), as many as kTileParts workgroups need for one long sequence; of more rows 16, which a wave joins.
        // (us where a block is one part / where parts go by keys: single tokens of 64 sequences of 1 to 30,000 keys on a log scale, 16
        // heads for 4, 242 / 46; 250 of 1 to 6,000 evenly, one K/V head, 56 / 50, all of 3,000 36 / 38; 96 with 4 K/V heads 77 /
        // 75, all of 3,000 55 / 57.) Beyond kMostCut sequences or 1,024 blocks of all K/V heads, none: the longest sequence is then a
        // call's least time (one of 30,000 keys among others of 500, 16 K/V heads: of 64 84 us, of 65 289).
        if (s->B > kMostCut || n > 1024 || tiles < 2 * kTileLeast) return r;
        r.target = kTileParts;
        want = kTileParts / s->H_kv;
        if (want > 8192 / n) want = 8192 / n;
        if (want > 16 && (int64_t)s->H * s->N > 512) want = 16;
        most = tiles / kTileLeast;
    } else if (n >= 1000 || tiles < 24) {
        // 1 / 3: 1,024 blocks of up to 64 tiles, 4 heads a K/V head, 96 / 119 (one head 150 / 128), 2,048 181 / 219, 1,250 of 18
        // 78 / 84; 176 of 21 32.0 / 33.4.
        return r;
    } else {
        // Parts by keys here too, for as many workgroups as fill the chip's 1,024 places once, by 80% at least and not to the last one, else
        // nearly half as many again; long lists are cut further, into parts of 40 tiles. By parts of a block, 1 / 2 / 3 / 4 / 6 / 8 /
        // 16: 440 blocks of up to 66 tiles 107 / 94 / 92 / 92 / 92 / 94 / 92; 880 139 / 160 / 156; 512 of up to 64 102 / 90 / 77 / 77 / 78
        // / 78; 220 of 66 85 / 65 / 59 / 57 / 62; 176 of 86 106 / 81 / 72 / 61 / 68 / 64 / 64; 176 of 687 782 / 523 / 434 / 341 / 370 / 330 /
        // 310; 128 of 64 78 / 48 / 45 / 38 / 37. (As many parts for every block / by keys: 200 tokens each of 16 sequences of 50 to 20,000 on a
        // log scale, 16 heads for 4, 178 / 107; 512 each of 12 of 100 to 8,000, 8 heads, 75 / 62; of 4 of 16,384, 16 for 4, 208 / 194.)
        if (s->B > kMostCut) return r;
        want = 1024 / n;
        if (want * n < 820 || want * n > 1000) want = (1400 + n - 1) / n;
        const int64_t parts = 2816 / n < tiles / 40 ? 2816 / n : tiles / 40;
        if (parts > want) want = parts;
        // (The workspace stays below 100 MB.)
        const int64_t room = 2700 - n - s->H_kv;
        r.target = (int)(want * n < room ? want * n : room);
        want = kMaxPagedSplits;
        most = tiles / kWideLeast;
    }
    const int64_t splits = want < most ? want : most;
    r.splits = (int)(splits < 1 ? 1 : splits > kMaxPagedSplits ? kMaxPagedSplits : splits);
    // (A block's share of the target, rounded, and at least one.)
    r.parts = r.blocks + r.target / s->H_kv + 1;
    return r;
}

}  // namespace ress
