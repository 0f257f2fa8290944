// Internal declarations shared by the kernels and the C ABI layer of ress_pages.h.
#pragma once

#include "layer_internal.h"
#include "ress_pages.h"

namespace ress {

// Runs of chunks whose first `half` ones hold the pairs' first sides, the next `half` the second sides, and from
// `pair` on the pairs (half = 0, interleaved: chunks that hold whole pairs, `count` of them).
struct ChunkRuns {
    int n;
    int first[RESS_MAX_ROPE_AXES], half[RESS_MAX_ROPE_AXES], count[RESS_MAX_ROPE_AXES], pair[RESS_MAX_ROPE_AXES];
};

// The norm of heads with the rotation. r: tables, sizes, pos and strides as in rope.hip (q_in, k_in,
// q_out, k_out are this pass's inputs and outputs; r.chunk: 0 for pairs).
struct HeadNormParams {
    RopeParams r;
    ChunkRuns runs;
    bool layer;  // subtract the mean
    float eps;
    const float *gamma[2], *beta[2];  // of Q and K; null: 1, 0
    // Into pages (slots not null): k_out and v_out are pages, behind K's heads come V's.
    const int32_t *slots;
    int n_slots;
    Divider pages;  // of the tokens of a page
    int page;
    const void *v_in;
    void *v_out;
    ress_strides vi;
    ress_page_strides kp, vp;
};

struct HeadNormBwdParams {
    ChunkRuns runs;
    RopeParams r;  // q_in, k_in: the gradients of the outputs; q_out, k_out: those of the inputs
    bool layer;
    float eps;
    const float *gamma[2];
    const void *x[2];  // the forward pass's inputs
    ress_strides xs[2];
    float *part;    // [parts][4][D]: gamma and beta of Q, of K; null: not wanted
    float *sums[4]; // outputs, each may be null
};

// Workgroups of the backward pass, which take `tokens_each` tokens at a time: over tokens, over heads.
// At most, each with a row of partial sums: three a CU, which 16-byte chunks have places for. (us with 344 / 512 / 768 / 1,024: 2,748 bf16
// tokens of 16 + 16 heads 19.6 / 20.2 / 19.8 / 24.2, 5,496 25.1 / 25.5 / 23.9 / 27.3, 21,984 76 / 68 / 58 / 58; 10,992 float32 tokens of
// 12 + 4 36.4 / 35.8 / 32.7 / 32.0.)
constexpr int kHeadParts = 768;
struct HeadBwdPlan {
    int tokens, heads;  // workgroups over tokens; heads a workgroup
    int parts;
};
HeadBwdPlan head_bwd_plan(int H_all, int N, int tokens_each);
// Rows of partial sums that any of its plans needs at most.
int head_bwd_parts(int H_all, int N);

struct TableParams {
    int B, N, page, n_pages, max_pages;
    Divider pages;  // of page
    int64_t stride;
    const int32_t *lens, *new_lens, *free_pages, *n_free;
    int32_t *tables, *lens_out, *n_free_out, *cu_q, *slots, *pos, *n_refused;
};

struct ReleaseParams {
    int B, n_pages, max_pages;
    int64_t stride;
    bool clear;
    const int32_t *first, *last, *n_free;
    int32_t *tables, *free_pages, *n_free_out;
    int32_t *counts;  // [B + 1]: entries given back, then the stack's height
};

// Attention over pages. A block is `rows` rows (new token, query head of a K/V head) of one
// sequence, computed together: 128 by paged_wide.hip's kernel, 32 by paged_tile.hip's.
struct PagedParams {
    int B, N, H, H_kv, group;
    int page, n_pages, max_pages, capacity;  // capacity: tokens that a table holds
    int frame, window, n_sink;               // (frame, window: see sights)
    Divider frames, pages, groups;           // of frame, page, group
    int64_t table_stride;
    int blocks;  // of all sequences, at most
    int splits;  // workgroups that share a block's keys, at most
    int parts;      // splits > 1: of all blocks of a K/V head, at most
    float share;    // splits > 1: of all sequences' keys of a K/V head, what a workgroup takes
    int most_keys;  // that a token sees
    References refs;
    float scale, scale_log2;
    ress_strides qs, os;
    ress_page_strides ks, vs;
    // Pages of multiples of 8 tokens whose strides, and whose rows' offsets in a page, fit 32 bits in steps of 16 bytes:
    // those steps, and whether K's and V's are the same.
    bool eights, alike;
    uint32_t k_page16, k_token16, v_page16, v_token16;
    const uint16_t *q, *k, *v;
    const int32_t *cu_q, *lens, *tables;
    uint16_t *o;
    float *lse;
    // splits > 1: unnormalised outputs, and references and sums. 32 rows: [splits][H][N] of 64 floats, and [H][N], the
    // workgroups that share a row's keys. 128 rows: [H_kv][parts] of 128 x 64, as the lanes hold them, and [blocks], the first part, how
    // far the next ones are, and how many.
    float *part;
    float2 *part_row;
    int32_t *cuts;
    int4 *cut;
    int32_t *starts;  // [B + 1], of more than kMostScanned sequences: blocks before each one's, and all
};

constexpr int kMostScanned = 512;  // (see find_block)
struct PagedPlan {
    int rows;    // of a block
    int blocks, splits;
    int target, parts;  // splits > 1: workgroups that keys are cut for, parts of a K/V head at most
};
PagedPlan paged_plan(const ress_paged_shape *s);
constexpr int kMaxPagedSplits = 64;
constexpr int kMostCut = 256;    // sequences up to which keys are cut
constexpr int kTileParts = 256;  // workgroups that blocks of 32 rows are cut for
constexpr int kTileLeast = 4, kWideLeast = 10;  // tiles of a workgroup at least where keys are cut (a wave one; see paged_plan)

hipError_t launch_head_norm(const HeadNormParams &p, hipStream_t s);
hipError_t launch_head_norm_bwd(const HeadNormBwdParams &p, hipStream_t s);
hipError_t launch_tables(const TableParams &p, hipStream_t s);
hipError_t launch_release(const ReleaseParams &p, hipStream_t s);
hipError_t launch_paged(const PagedParams &p, int rows, hipStream_t s);
hipError_t launch_paged_wide(const PagedParams &p, hipStream_t s);

}  // namespace ress
