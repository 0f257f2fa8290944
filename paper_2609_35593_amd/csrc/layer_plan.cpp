// How the kernels of ress_layer.h spread over the chip: functions of a shape alone, from measured
// times. Plain host code, apart from the kernels, so that it runs without a GPU.
#include "layer_internal.h"

namespace ress {

// 512 workgroups of 8 waves fill the chip (128 registers a lane), and their partial sums of
// 1,024 channels are 4 MB. (1,024 for narrow rows: 175,872 of 64 bf16 channels 19.9 -> 22.8 us.)
int norm_bwd_parts(int64_t rows) { return (int)(rows < 1 ? 1 : rows < 512 ? rows : 512); }

// ---------------------------------------------------------------- windowed attention, forward

WindowPlan window_plan(const ress_window_shape *s)
{
    // Tiles a block sees at most, and one in the middle of the queries.
    const int64_t window = window_tokens(s->frame, s->window) * (s->causal ? 1 : 2);
    const int64_t sinks = s->n_sink < s->n_k ? s->n_sink : s->n_k;
    const int64_t keys = window + 128 + sinks < s->n_k ? window + 128 + sinks : s->n_k;
    const int64_t middle = (int64_t)s->q_offset + s->n_q / 2, reach = s->causal && middle < s->n_k ? middle : s->n_k;
    const int64_t tiles = (keys + 63) / 64, tiles_mid = (window + sinks < reach ? window + sinks : reach) / 64;
    auto blocks = [&](int g) { return (int64_t)s->H * (((int64_t)s->n_q * g + 127) / 128); };
    const int64_t n = blocks(1);
    // (In the comments, G/S us: with G key groups, blocks cut over S workgroups.)
    WindowPlan plan = {1, 1};
    if (tiles < 2 || n >= 1200) return plan;
    // From 512 workgroups of 128 queries on, two a CU, key groups cost (640 blocks of 18 tiles 1/1 44, 2/1
    // 47; 688 of 172 308 / 354), but where a few blocks see much more than the others and finish late:
    // those on the edge of a large frame, one frame more. For that, edges lie inside blocks (688 blocks,
    // one frame of 1,024 36 / 43, of 1,000 78 / 68), not every key is in reach (688, two of 3,000 and
    // 2,504 158 / 121, both in reach 126 / 143), and the frame is long beside what all the blocks take:
    //   516-528 blocks: one of 776 48-49 / 44-50, of 850 53 / 46-52, of 900 54-56 / 50, of 1,374 93 / 67
    //   784-864: ratios, of 900 1.03-1.11, of 1,000 0.90-0.97, of 1,374 0.83-0.94
    //   992-1,120: of 1,000 0.95-1.09, of 1,200 1.02-1.11, of 1,374 0.79-1.00
    // and from 1,200 blocks on no more (1,264, three of 1,374 212 / 217, 1,632 279 / 287).
    if (n >= 512) {
        const bool edges = s->frame % 128 || s->q_offset % 128;
        const int least = n < 768 ? 850 : n < 896 ? 1000 : 1300;
        if (edges && window + sinks < s->n_k && s->frame >= least) plan.groups = 2;
        return plan;
    }
    plan.groups = 2;  // (352 blocks of 87 1/1 197, 2/1 155, 4/1 243; 18 of 3 13 / 7.3 / 8.5)
    if (n > 64) {
        // Long lists: cut, to balance the load of four workgroups a CU, where that outweighs the partial
        // results (268 blocks of 65 2/1 109, 1/4 83; 176 of 118 96 / 76; 88 of 172 119, 1/8 62; 192 of 58
        // 49, 1/4 49; 142 of 47 42 / 42).
        if (tiles_mid >= 56) plan = {1, n >= 128 ? 4 : 8};
        return plan;
    }
    if (n >= 8 && tiles >= 40) {
        // About a workgroup a CU, of 8 tiles at least (47 blocks of 94 4/1 38, 2/5 25; 22 of 63 4/2 23, 2/8
        // 19; 24 of 47 18, 2/5 15).
        const int64_t want = 240 / n;
        plan.splits = (int)(want < tiles / 8 ? want : tiles / 8);
    } else if (tiles >= 8) {
        // Four groups (one workgroup a CU, by its LDS), with tiles enough for each: 64 blocks of 9 13.4 /
        // 9.4 / 9.2. Few blocks: workgroups to fill the CUs, each with two tiles a group at least: one
        // of 625 203 -> 22 with 32.
        plan.groups = 4;
        if (n > 0) {
            int64_t want = 256 / blocks(4);
            if (want > tiles / 8) want = tiles / 8;
            plan.splits = (int)(want < 1 ? 1 : want > kMaxSplits ? kMaxSplits : want);
        }
    }
    return plan;
}

// ---------------------------------------------------------------- backward

WindowBwdPlan window_bwd_plan(const ress_window_shape *s)
{
    WindowBwdPlan r = {1, 0, 1, 1, 0};
    // dq: four key groups where their workgroups still are one a CU and see 8 tiles, else two while
    // there are fewer blocks than fill the chip four times over (whole pass in us with 1 / 2 / 4 groups:
    // 63 blocks over 2,000 keys 76 / 56 / 52, 128 over 1,000 65 / 53 / 65, 640 over 512 116 / 107 / 173,
    // 1,376 over three frames of 1,374 848 / 850 / 1,183).
    const int64_t window = window_tokens(s->frame, s->window) * (s->causal ? 1 : 2);
    const int64_t q_blocks = (int64_t)s->H * (((int64_t)s->n_q + 127) / 128);
    const int64_t seen = window + 128 + s->n_sink < s->n_k ? window + 128 + s->n_sink : s->n_k;
    r.groups = q_blocks <= 64 && seen > 7 * 64 ? 4 : q_blocks < 1024 ? 2 : 1;
    const int64_t blocks = (s->n_k + 127) / 128;
    if (s->H_kv == 0 || blocks == 0) return r;
    const int64_t sinks = s->n_sink < s->n_k ? s->n_sink : s->n_k, group = s->H / s->H_kv;
    r.sink_blocks = (int)((sinks + 127) / 128);
    // Tiles of queries in a list at most: of sinks, and of other keys.
    const int64_t span = window_tokens(s->frame, s->window) * (s->causal ? 1 : 2) + at_most_2_26(s->frame) + 127;
    const int64_t all = ((int64_t)s->n_q + 63) / 64;
    const int64_t some = span < s->n_q ? (span + 63) / 64 + 1 : all;
    const int64_t t_sink = group * all, t_win = group * (some < all ? some : all);
    const int64_t sb = r.sink_blocks, wb = blocks - sb;
    const double total = (double)s->H_kv * (sb * t_sink + wb * t_win);
    // The slices that the following estimate (us) favours: a tile takes 1.3 in a workgroup that has
    // a CU to itself, 1.8 in one of two, the chip 1 / 290 per tile when full; a slice's sums cost
    // 0.03 to write and add up, the join 4. Measured, whole pass, uncut / as chosen here: 12 heads
    // for 4 of 3,001 tokens, 5 sinks, 225 / 62; 16 for 4 of 5,000, 4 sinks, 474 / 100; 6 for 2 of 700,
    // 20 sinks, 63 / 28; 16 of 1,374, uncut 64, in halves 69.
    double best = 1e30;
    for (int ss = 1; ss <= (sb ? 64 : 1); ss *= 2)
        for (int ws = 1; ws <= (wb ? 16 : 1); ws *= 2) {
            if (ss > t_sink || ws > t_win) continue;
            const double items = (double)s->H_kv * (sb * ss + wb * ws);
            const double cut = (double)s->H_kv * ((ss > 1 ? sb * ss : 0) + (ws > 1 ? wb * ws : 0));
            const int64_t l_sink = sb ? (t_sink + ss - 1) / ss : 0, l_win = wb ? (t_win + ws - 1) / ws : 0;
            const double alone = (double)(l_sink > l_win ? l_sink : l_win) * (items <= 256 ? 1.3 : 1.8);
            const double cost = (alone > total / 290 ? alone : total / 290) + (cut > 0 ? 4 + 0.03 * cut : 0);
            if (cost < best) {
                best = cost;
                r.sink_slices = ss;
                r.slices = ws;
            }
        }
    r.items = (int)(sb * r.sink_slices + wb * r.slices);
    return r;
}

int window_bwd_joined(const WindowBwdPlan &p, int blocks, int &first)
{
    first = p.sink_slices > 1 ? 0 : p.sink_blocks;
    return (p.slices > 1 ? blocks : p.sink_slices > 1 ? p.sink_blocks : first) - first;
}

// ---------------------------------------------------------------- decode

// Workgroups per sequence and K/V head (or 32 of its heads).
int decode_splits(const ress_decode_shape *s)
{
    if (s->B == 0 || s->H == 0 || s->capacity == 0) return 1;
    const int64_t seen = window_tokens(s->frame, s->window) + s->n_sink;
    const int64_t keys = seen < s->capacity ? seen : s->capacity;  // at least 1
    const int group = s->H / s->H_kv;
    const bool one = group == 1;
    const int64_t heads = (int64_t)s->B * s->H_kv * ((group + 31) / 32);
    // One head: enough for 4 workgroups a CU, none with less than 256 keys (us with at least 256 /
    // 512 / 1,024 keys, the join counted: 16 heads of 6,870 9.6 / 9.3 / 10.8; one of 40,000 10.6 with 32
    // splits; 32 heads of 300 7.4 / 5.1 / 5.2). Several: one a CU, of at least a turn a wave (us: 96 of
    // 4,160 keys, 1 / 2 / 5 / 8 splits 29.6 / 23.3 / 23.8 / 25.2; 32 of 4,000, 4 / 8 / 16 14.2 / 11.7 / 12.0;
    // 4 of 8,000, 8 / 16 / 32 12.4 / 10.0 / 8.9). One workgroup up to 512 keys: a join costs more.
    const int64_t turns = one ? (keys + 31) / 32 : (keys + 63) / 64, waves = one ? kHeadWaves : kTileWaves;
    const int64_t want = (one ? 1024 : 256) / heads, most = keys <= 512 ? 1 : (turns + waves - 1) / waves;
    int64_t n = want < most ? want : most;
    n = n < 1 ? 1 : n > kMaxSplits ? kMaxSplits : n;
    // No more than give every wave the same turns: 10 splits of 3.25 turns a wave take as long as 8 of 4.
    const int64_t each = (turns + n * waves - 1) / (n * waves);
    return (int)((turns + each * waves - 1) / (each * waves));
}

}  // namespace ress
