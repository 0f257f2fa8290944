/*
 * ress_layer.h - further steps of a layer in libress: layer norm (forward and
 * backward), rotary positions with several axes, and attention over a sliding
 * window of frames with sink tokens (forward, backward, and one token over a
 * cache). Status codes and limits are those of ress.h.
 *
 * Conventions shared by every entry point
 *  - Device pointers are owned by the caller; the library never allocates,
 *    frees or copies device memory and never synchronises. All work is enqueued
 *    on `stream` (of the current device) in order, as kernels only, so every call
 *    may be captured into a graph. RESS_OK means the work was enqueued.
 *  - On any error status nothing is enqueued and no output is written.
 *  - Strides count elements; the channels of a row are contiguous. An output
 *    must not overlap itself, another output or, unless a declaration says so, an
 *    input.
 *  - Results are the same in every call: no atomics, fixed orders of summation.
 *  - Calls are stateless; calls on different streams may run at once as long as
 *    their outputs and workspaces do not overlap. A workspace holds nothing
 *    between calls and needs no initial value; two graphs that may be replayed at
 *    once need two.
 */
#ifndef RESS_LAYER_H
#define RESS_LAYER_H

#include "ress.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of the layer norm and the rotary positions. */
#define RESS_DTYPE_BF16 0
#define RESS_DTYPE_F32 1

#define RESS_MAX_NORM_WIDTH 16384
#define RESS_MAX_ROPE_AXES 4
#define RESS_MAX_ROPE_D 256
#define RESS_MAX_BATCH 65535

/* Element strides of [heads][tokens][channels]. */
typedef struct {
    int64_t head, token;
} ress_strides;

/* ---------------------------------------------------------------- layer norm */

typedef struct {
    int64_t rows;     /* 0..2^31 - 1 */
    int width;        /* channels of a row, 1..RESS_MAX_NORM_WIDTH */
    int x_dtype;      /* of x and dx */
    int y_dtype;      /* of y and dy */
    int64_t x_stride; /* between rows of x and dx, >= width */
    int64_t y_stride; /* between rows of y and dy, >= width */
    double eps;       /* added to the variance, > 0; not used by the backward pass */
} ress_norm_shape;

/* y = (x - mean) rstd gamma + beta over the channels of every row, with
 * mean = sum(x) / width and rstd = 1 / sqrt(sum((x - mean)^2) / width + eps), in
 * float32 (the variance from centred values), rounded once to y's type (values up to
 * 2^56: float32 holds no sum of squares of larger ones). For
 * instance the residual stream before ress_qkv_proj_pool, or the heads of Q and K
 * (width 64).
 *   gamma, beta  device float32 [width], or NULL (1, 0)
 *   mean, rstd   device float32 [rows] out, both or neither; for the backward pass
 * y may be x where their types and strides are equal. Pointers are aligned to
 * their elements. */
int ress_layer_norm(const ress_norm_shape *shape, const void *x, const float *gamma, const float *beta, void *y,
                    float *mean, float *rstd, hipStream_t stream);

/* Bytes of device workspace ress_layer_norm_bwd needs (partial sums of the
 * weights' gradients, at most 64 MiB); depends on rows and width only. */
int ress_layer_norm_bwd_workspace_size(const ress_norm_shape *shape, size_t *bytes);

/* Gradients of ress_layer_norm: with g = dy gamma and xh = (x - mean) rstd,
 *   dx = rstd (g - mean_c(g) - xh mean_c(g xh)),
 *   dgamma = sum over rows of dy xh,  dbeta = sum over rows of dy,
 * in float32, dx rounded once to x's type.
 *   dy             of y's type and stride
 *   mean, rstd     device float32 [rows], as ress_layer_norm wrote them
 *   dx             of x's type and stride, out; may be x, or dy where the types
 *                  and strides are equal
 *   dgamma, dbeta  device float32 [width] out, each may be NULL; zeros where rows
 *                  is 0
 *   workspace      256-byte aligned; not needed where dgamma and dbeta are NULL */
int ress_layer_norm_bwd(const ress_norm_shape *shape, const void *dy, const void *x, const float *gamma,
                        const float *mean, const float *rstd, void *dx, float *dgamma, float *dbeta, void *workspace,
                        size_t workspace_bytes, hipStream_t stream);

/* --------------------------------------------------------- rotary positions */

/* Which channels turn together, and by which frequency. dims[a] channels belong to
 * axis a, their sum R <= D; the last D - R channels are copied.
 *   SPLIT        each axis has a run of dims[a] channels and a spectrum of its own:
 *                channels i and i + dims[a]/2 of the run, base^(-2i / dims[a])
 *   INTERLEAVED  the same with channels 2i and 2i + 1 of the run
 *   SECTIONS     channels i and i + R/2 of the head, base^(-2i / R); the axes take
 *                dims[a]/2 consecutive i each */
#define RESS_ROPE_SPLIT 0
#define RESS_ROPE_INTERLEAVED 1
#define RESS_ROPE_SECTIONS 2

typedef struct {
    int H, H_kv;   /* heads of q and of k, 0..RESS_MAX_HEADS */
    int N;         /* tokens, 0..RESS_MAX_TOKENS */
    int D;         /* channels of a head, even, 2..RESS_MAX_ROPE_D */
    int n_axes;    /* 1..RESS_MAX_ROPE_AXES */
    int dims[RESS_MAX_ROPE_AXES]; /* even, >= 0; unused entries are ignored */
    int layout;    /* RESS_ROPE_* */
    int inverse;   /* nonzero: turn back, which is the gradient's pass as well */
    int dtype;     /* of q, k and the outputs */
    double base;   /* >= 1, finite */
    ress_strides q, k, q_out, k_out;
} ress_rope_shape;

/* Rotary positions of Q and K between the projection and the attention: every pair
 * (a, b) of a token's channels becomes
 *   (a cos t - b sin t, a sin t + b cos t),  t = pos[token][axis] base^(...),
 * (the angle negated for `inverse`). The angle is formed in float64 and reduced
 * exactly, so that far positions keep their phase; products in float32, rounded
 * once to the type.
 *   pos           device int32 [N][n_axes]
 *   q_in, q_out   [H][N][D] by shape->q and shape->q_out; NULL where H is 0
 *   k_in, k_out   [H_kv][N][D] likewise; NULL where H_kv is 0
 * An output may be its input where the strides are equal (in place); strides may
 * place k_out in a cache. The pooled state that ress_qkv_proj_pool leaves is of Q and K as
 * they were projected: ress_select of turned ones takes pooled_in_workspace = 0. */
int ress_rope(const ress_rope_shape *shape, const int32_t *pos, const void *q_in, const void *k_in, void *q_out,
              void *k_out, hipStream_t stream);

/* -------------------------------------------- sliding window with sink tokens */

/* Query t stands at position p = q_offset + t among the keys. Positions are counted
 * in frames of `frame` tokens (1: plain tokens); with f(p) = floor(p / frame), query
 * p sees key s < n_k where
 *   causal:      f(s) <= f(p) and (f(s) > f(p) - window or s < n_sink)
 *   otherwise:   |f(s) - f(p)| < window or s < n_sink
 * so a frame is seen whole, and the first n_sink tokens stay visible. */
typedef struct {
    int H, H_kv;  /* heads of q, and of k and v: H_kv divides H, head h reads h / (H / H_kv); 0..RESS_MAX_HEADS */
    int n_q, n_k; /* 0..RESS_MAX_TOKENS */
    int D;        /* must be 64 */
    int q_offset; /* 0..RESS_MAX_TOKENS */
    int frame;    /* tokens of a frame, >= 1 */
    int window;   /* frames a query sees, its own among them, >= 1 */
    int n_sink;   /* >= 0 */
    int causal;
    ress_strides q, k, v, o; /* multiples of 8; a token stride of at most 2^22 */
} ress_window_shape;

/* Blocks: a block of 128 queries (keys, in the backward pass) is computed together. Keys
 * that none of its queries sees (queries that see none of its keys) are not read
 * and may hold anything; a NaN or infinity in one that some of them see may also
 * reach the others of the block. */

/* Bytes of device workspace ress_window_attn needs (0 but for long windows over too few
 * queries to fill the chip, whose keys are split over workgroups: at most 69 MB; strides
 * do not matter). */
int ress_window_attn_workspace_size(const ress_window_shape *shape, size_t *bytes);

/* o = softmax over the visible keys of (scale q . k) v, bf16 [H][n_q][64] by the
 * shape's strides, bf16 products, float32 softmax and accumulation (probabilities
 * rounded to bf16 for the product with v, o once). A query that sees no key gets a
 * zero output.
 *   lse  device float32 [H][n_q] out, or NULL: the natural logarithm of the sum of
 *        exp(scale q . k) over the visible keys, -inf where there are none
 *   workspace  256-byte aligned; may be NULL where none is needed
 * Pointers 16-byte aligned; 0 < scale <= 2^120. Logits (scale q . k) may be as large as float32
 * holds (2^126): a row's weights are those of its largest ones. */
int ress_window_attn(const ress_window_shape *shape, const void *q, const void *k, const void *v, float scale, void *o,
                     float *lse, void *workspace, size_t workspace_bytes, hipStream_t stream);

typedef struct {
    ress_strides d_o, dq, dk, dv;
} ress_window_grads;

/* Bytes of device workspace ress_window_attn_bwd needs (strides and pointers do
 * not matter). */
int ress_window_attn_bwd_workspace_size(const ress_window_shape *shape, size_t *bytes);

/* Gradients of ress_window_attn: with p the probabilities, formed again from lse,
 * and delta the sum over keys of p (d_o . v),
 *   dv = p^T d_o,  ds = p (d_o v^T - delta),  dq = scale ds k,  dk = scale ds^T q,
 * dk and dv summed over the query heads that share them. bf16 products, float32
 * accumulation; p and ds rounded to bf16 for their products, outputs once. (delta is
 * first taken from d_o . o; what the rounding of o leaves in it is summed beside dq
 * in float32 and taken out of all three. p is off by some 2^-22 |lse| of itself, as lse is
 * float32: less than its rounding for logits up to 10^4; from some 10^7 on, where lse no longer
 * tells one key from another, gradients mean nothing and may be infinite or NaN.)
 *   o, lse      as ress_window_attn wrote them (o by shape->o)
 *   dq, dk, dv  bf16 out by the strides of `grads`; dk and dv of keys that no query
 *               sees are zero
 *   workspace   256-byte aligned */
int ress_window_attn_bwd(const ress_window_shape *shape, const ress_window_grads *grads, const void *d_o, const void *q,
                         const void *k, const void *v, const void *o, const float *lse, float scale, void *dq, void *dk,
                         void *dv, void *workspace, size_t workspace_bytes, hipStream_t stream);

/* One new token of each of B sequences over its cache: the token of sequence b is the
 * last of its lens[b] cached ones (its key and value are in the cache), and sees
 * them as a causal query at position lens[b] - 1. */
typedef struct {
    int B;        /* sequences, 0..RESS_MAX_BATCH */
    int H, H_kv;  /* as in ress_window_shape */
    int capacity; /* tokens of the cache, 0..RESS_MAX_TOKENS */
    int D;        /* must be 64 */
    int frame, window, n_sink;
    int64_t q_batch, q_head; /* strides of q [B][H][64]; multiples of 8 as all of these */
    int64_t k_batch, v_batch;
    ress_strides k, v;       /* [B][H_kv][capacity][64]; a token stride of at most 2^22 */
    int64_t o_batch, o_head;
} ress_decode_shape;

/* Bytes of device workspace ress_window_attn_decode needs (strides do not matter). */
int ress_window_attn_decode_workspace_size(const ress_decode_shape *shape, size_t *bytes);

/*   lens       device int32 [B], read by the kernels (a captured call follows its
 *              changes); clamped to [0, capacity]. A sequence of length 0 gets a
 *              zero output.
 *   q, o       bf16 [B][H][64]
 *   k, v       bf16 caches; nothing at or behind lens[b] has a part in the result
 *   scale      as for ress_window_attn, logits too
 *   workspace  256-byte aligned */
int ress_window_attn_decode(const ress_decode_shape *shape, const void *q, const void *k, const void *v,
                            const int32_t *lens, float scale, void *o, void *workspace, size_t workspace_bytes,
                            hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* RESS_LAYER_H */
