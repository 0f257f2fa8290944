/*
 * ress_pages.h - steps of a layer over keys and values that live in pages: the norm
 * of every head of Q and K with the position rotation in the same pass (forward,
 * backward, and with K and V written into pages), the tables and slots of a step from
 * request lengths, and attention of a chunk of new tokens of several sequences over
 * their pages. Status codes and limits are those of ress.h, conventions those of
 * ress_layer.h.
 *
 * A cache in pages
 *  - K and V are [n_pages][H_kv][page][64] by strides, `page` tokens of one sequence a
 *    page. The row `tables + b * table_stride` holds sequence b's pages in the order of
 *    its tokens: token t is row t % page of page tables[b][t / page]. The slot of a token
 *    is that page times `page` plus that row.
 *  - Lengths, tables, slots and offsets are on the device and read by the kernels, so a
 *    captured call follows their changes. They are never trusted with an address: a
 *    length outside what a table holds is clamped, and a page outside [0, n_pages) or a slot
 *    outside [0, n_pages * page) is not touched.
 */
#ifndef RESS_PAGES_H
#define RESS_PAGES_H

#include "ress_layer.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element strides of [pages][heads][tokens][channels]. */
typedef struct {
    int64_t page, head, token;
} ress_page_strides;

/* ----------------------------------- norm of heads with rotary positions */

/* RMS: the mean is taken as 0. */
#define RESS_HEAD_NORM_LAYER 0
#define RESS_HEAD_NORM_RMS 1

typedef struct {
    ress_rope_shape rope; /* heads, tokens, channels, the rotation, the type and strides (inverse must be 0) */
    int norm;             /* RESS_HEAD_NORM_* */
    double eps;           /* added to the variance, > 0 */
} ress_head_norm_shape;

/* Between the projection and the attention, for every token and head of Q and of K
 *   y = turn(pos, (x - mean) rstd gamma + beta),  rstd = 1 / sqrt(var + eps),
 * with mean and variance over the head's D channels (RMS: mean 0, the variance the mean
 * square) and ress_rope's turn. Float32 (the mean is taken from the values before their squares and
 * products; values up to 2^56), angles as in ress_rope, rounded once to the type: what ress_layer_norm
 * and ress_rope would round in between is kept.
 *   pos                device int32 [N][n_axes]
 *   q_in, q_out        [H][N][D] by rope.q and rope.q_out; NULL where H is 0
 *   k_in, k_out        [H_kv][N][D] likewise; NULL where H_kv is 0
 *   gamma, beta        device float32 [D] for Q and for K, each may be NULL (1, 0)
 * An output may be its input where the strides are equal. Pointers are aligned to their
 * elements. */
int ress_qk_norm_rope(const ress_head_norm_shape *shape, const int32_t *pos, const void *q_in, const void *k_in,
                      const float *q_gamma, const float *q_beta, const float *k_gamma, const float *k_beta, void *q_out,
                      void *k_out, hipStream_t stream);

typedef struct {
    int n_pages;  /* >= 0; n_pages * page <= 2^31 - 1 */
    int page;     /* tokens of a page, 1..RESS_MAX_TOKENS */
    ress_page_strides k, v;
    ress_strides v_in;
} ress_page_cache;

/* ress_qk_norm_rope with K written into pages instead of k_out (rope.k_out is not used),
 * and V copied into pages as it is: token t into slot slots[t].
 *   slots             device int32 [N]; a token without a slot (outside [0, n_pages * page))
 *                     is not written, its q_out is. Two tokens must not have one slot.
 *   v_in              [H_kv][N][D] by cache->v_in, of the type of k_in
 *   k_pages, v_pages  [n_pages][H_kv][page][D] by cache->k and cache->v; no input */
int ress_qk_norm_rope_pages(const ress_head_norm_shape *shape, const ress_page_cache *cache, const int32_t *pos,
                            const int32_t *slots, const void *q_in, const void *k_in, const void *v_in,
                            const float *q_gamma, const float *q_beta, const float *k_gamma, const float *k_beta,
                            void *q_out, void *k_pages, void *v_pages, hipStream_t stream);

typedef struct {
    ress_strides dq_out, dk_out, dq, dk;
} ress_head_norm_grads;

/* Bytes of device workspace ress_qk_norm_rope_bwd needs (partial sums of the weights'
 * gradients, at most 4 MiB); depends on heads, tokens and channels only. */
int ress_qk_norm_rope_bwd_workspace_size(const ress_head_norm_shape *shape, size_t *bytes);

/* Gradients of ress_qk_norm_rope: with u the gradient of an output turned back, g = u gamma and
 * xh = (x - mean) rstd (formed again from x),
 *   dx = rstd (g - mean_c(g) - xh mean_c(g xh))   (RMS: without mean_c(g)),
 *   dgamma = sum over heads and tokens of u xh,  dbeta = sum over heads and tokens of u,
 * in float32, dx rounded once to the type.
 *   dq_out, dk_out    gradients of the outputs, by `grads`
 *   q_in, k_in        the forward pass's inputs, by rope.q and rope.k (rope.q_out and
 *                     rope.k_out are not used)
 *   dq, dk            out, by `grads`; each may be its dq_out, dk_out, or its input, where the
 *                     strides are equal
 *   *_dgamma, *_dbeta device float32 [D] out, each may be NULL; zeros where there are no
 *                     tokens or heads
 *   workspace         256-byte aligned; not needed where all four are NULL */
int ress_qk_norm_rope_bwd(const ress_head_norm_shape *shape, const ress_head_norm_grads *grads, const int32_t *pos,
                          const void *dq_out, const void *dk_out, const void *q_in, const void *k_in,
                          const float *q_gamma, const float *k_gamma, void *dq, void *dk, float *q_dgamma,
                          float *q_dbeta, float *k_dgamma, float *k_dbeta, void *workspace, size_t workspace_bytes,
                          hipStream_t stream);

/* ------------------------------------------------------- pages of a step */

typedef struct {
    int B;                /* sequences, 0..RESS_MAX_BATCH */
    int N;                /* entries of slots and pos, 0..RESS_MAX_TOKENS */
    int page;             /* tokens of a page, 1..RESS_MAX_TOKENS */
    int n_pages;          /* pages of the cache, and entries of free_pages; n_pages * page <= 2^31 - 1 */
    int max_pages;        /* entries of a sequence's table; max_pages * page <= RESS_MAX_TOKENS */
    int64_t table_stride; /* between tables, >= max_pages */
    int clear;            /* ress_pages_release: nonzero marks the entries that it gives back with -1 */
} ress_table_shape;

/* A step in which sequence b, of lens[b] cached tokens, gets new_lens[b] more: the pages that
 * they need beyond those that the sequence has, ceil(lens[b] / page) of them, go from the
 * top of the stack of free pages into its table, sequence by sequence, and every new token
 * gets its slot. The new tokens of all sequences lie one behind the other, as ress_paged_attn takes
 * them: those of b are cu_q[b] .. cu_q[b + 1] - 1.
 * A sequence whose table is too short for its tokens gets none of them. Of the others, the
 * first for which N or the free pages do not suffice, and all behind it, get none.
 *   lens, new_lens  device int32 [B]; lens is clamped to [0, max_pages * page], new_lens to >= 0
 *   free_pages      device int32 [n_pages], the stack's first *n_free entries are free pages
 *   n_free          device int32, clamped to [0, n_pages]
 *   tables          device int32 [B][max_pages] by table_stride, in and out
 *   lens_out        device int32 [B] out, the lengths behind the step; may be lens
 *   n_free_out      device int32 out; may be n_free (free_pages keeps its entries)
 *   cu_q            device int32 [B + 1] out
 *   slots, pos      device int32 [N] out, every entry: the tokens' slots and positions; -1 and 0
 *                   behind the last token. A token on a page outside [0, n_pages) has slot -1.
 *   n_refused       device int32 out, or NULL: sequences that got none of their new tokens */
int ress_page_tables(const ress_table_shape *shape, const int32_t *lens, const int32_t *new_lens,
                     const int32_t *free_pages, const int32_t *n_free, int32_t *tables, int32_t *lens_out,
                     int32_t *n_free_out, int32_t *cu_q, int32_t *slots, int32_t *pos, int32_t *n_refused,
                     hipStream_t stream);

/* Bytes of device workspace ress_pages_release needs; depends on B only. */
int ress_pages_release_workspace_size(const ress_table_shape *shape, size_t *bytes);

/* Gives back pages: entries [first[b], last[b]) of every table go on top of the stack of free pages, in order of
 * b and of the entries, those outside [0, n_pages) left out. (N is not used.)
 *   first, last  device int32 [B], clamped to [0, max_pages]
 *   free_pages   device int32 [n_pages], in and out: entries from *n_free on are written (none beyond
 *                n_pages)
 *   n_free, n_free_out  as above
 *   tables       entries given back become -1 with `clear`, which makes a second release of them
 *                harmless; without it they are left as they are
 *   workspace    256-byte aligned */
int ress_pages_release(const ress_table_shape *shape, const int32_t *first, const int32_t *last, int32_t *tables,
                       int32_t *free_pages, const int32_t *n_free, int32_t *n_free_out, void *workspace,
                       size_t workspace_bytes, hipStream_t stream);

/* --------------------------------------- attention of new tokens over pages */

typedef struct {
    int B;         /* sequences, 0..RESS_MAX_BATCH */
    int N;         /* rows of q and o: new tokens of all sequences and any padding, 0..RESS_MAX_TOKENS */
    int H, H_kv;   /* as in ress_window_shape */
    int D;         /* must be 64 */
    int page, n_pages, max_pages; /* as in ress_table_shape */
    int frame, window, n_sink;    /* as in ress_window_shape, causal */
    int64_t table_stride;
    ress_strides q, o;            /* multiples of 8; a token stride of at most 2^22, as those of pages */
    ress_page_strides k, v;       /* multiples of 8 */
} ress_paged_shape;

/* Bytes of device workspace ress_paged_attn needs: partial results of keys that are split over
 * workgroups (at most 100 MB), and a list of more than 512 sequences; strides do not matter. */
int ress_paged_attn_workspace_size(const ress_paged_shape *shape, size_t *bytes);

/* The new tokens of sequence b are rows cu_q[b] .. cu_q[b + 1] - 1 of q and the last ones of its lens[b] tokens,
 * whose keys and values are all in its pages. A token at position p sees the keys s < lens[b] that a
 * causal query of ress_window_attn at p sees, but for those on a page outside [0, n_pages):
 *   o = softmax over them of (scale q . k) v
 * in the precision of ress_window_attn at least: weights are rounded to bf16 for their product with v where N H / H_kv is
 * more than 32 min(B, N), kept to 16 bits where it is not; those of a row sum to one as they enter it, with lse and
 * without. A token that sees no key gets a zero output.
 *   q, o       bf16 [H][N][64]; rows of o outside every sequence are left as they are
 *   k, v       bf16 pages; what no token of a block of new tokens (up to 128 rows, neighbours in one
 *              sequence) sees is not read; a NaN or infinity that some of them see may reach the others of the block
 *   cu_q       device int32 [B + 1], ascending, clamped to [0, N] (of offsets that descend, results
 *              mean nothing)
 *   lens       device int32 [B], the new tokens counted, clamped to [0, max_pages * page]. New tokens
 *              beyond lens[b] stand before position 0 and see nothing.
 *   tables     device int32 [B][max_pages] by table_stride
 *   lse        device float32 [H][N] out, or NULL: as in ress_window_attn, rows outside every
 *              sequence left as they are
 *   scale      as for ress_window_attn, logits too
 *   workspace  256-byte aligned; may be NULL where none is needed */
int ress_paged_attn(const ress_paged_shape *shape, const void *q, const void *k, const void *v, const int32_t *cu_q,
                    const int32_t *lens, const int32_t *tables, float scale, void *o, float *lse, void *workspace,
                    size_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* RESS_PAGES_H */
