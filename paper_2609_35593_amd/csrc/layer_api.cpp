// C ABI of ress_layer.h: argument validation, workspace layout and kernel launches.
// Every check runs on the host before anything is enqueued, so an error status
// means no device work and no output writes.
#include <math.h>
#include <string.h>

#include "checks.h"

namespace {

using namespace ress;

constexpr int64_t kMaxRows = 0x7fffffff;
constexpr int kHead = 64;

// Chunks of `per` channels, aligned to their size in every head and token.
bool rope_aligned(const ress_rope_shape &s, int per, const void *const (&src)[2], void *const (&dst)[2])
{
    const size_t bytes = per * dtype_size(s.dtype);
    const ress_strides *st[4] = {&s.q, &s.q_out, &s.k, &s.k_out};
    for (int i = 0; i < 2; ++i)
        if ((i ? s.H_kv : s.H) > 0 && (!aligned(src[i], bytes) || !aligned(dst[i], bytes) || !strides_ok(*st[2 * i], per) ||
                                       !strides_ok(*st[2 * i + 1], per)))
            return false;
    return true;
}

// ---------------------------------------------------------------- layer norm

int check_norm(const ress_norm_shape *s, bool forward)
{
    if (!s) return RESS_E_INVALID_ARG;
    if (s->rows < 0 || s->width < 1 || !dtype_ok(s->x_dtype) || !dtype_ok(s->y_dtype)) return RESS_E_INVALID_ARG;
    if (s->rows > kMaxRows || s->width > RESS_MAX_NORM_WIDTH) return RESS_E_UNSUPPORTED;
    if (s->x_stride < s->width || s->y_stride < s->width || s->x_stride > kMaxRows || s->y_stride > kMaxRows)
        return RESS_E_INVALID_ARG;
    if (forward && (!((float)s->eps > 0.f) || !isfinite((float)s->eps))) return RESS_E_INVALID_ARG;
    return RESS_OK;
}

size_t norm_workspace(const ress_norm_shape *s)
{
    return align256((size_t)ress::norm_bwd_parts(s->rows) * 2 * s->width * sizeof(float));
}

// An output that is an input must lie as it does.
bool norm_alias_ok(const void *out, int out_dtype, int64_t out_stride, const void *in, int in_dtype, int64_t in_stride)
{
    return out != in || (out_dtype == in_dtype && out_stride == in_stride);
}

// ------------------------------------------------------------------- windows

int check_window(const ress_window_shape *s, bool strides)
{
    if (!s) return RESS_E_INVALID_ARG;
    int st = check_heads(s->H, s->H_kv);
    if (st != RESS_OK) return st;
    if (s->n_q < 0 || s->n_k < 0 || s->q_offset < 0 || s->frame < 1 || s->window < 1 || s->n_sink < 0)
        return RESS_E_INVALID_ARG;
    if (s->D != kHead || s->n_q > RESS_MAX_TOKENS || s->n_k > RESS_MAX_TOKENS || s->q_offset > RESS_MAX_TOKENS)
        return RESS_E_UNSUPPORTED;
    if (strides && (!strides_ok(s->q, 8) || !strides_ok(s->k, 8) || !strides_ok(s->v, 8) || !strides_ok(s->o, 8)))
        return RESS_E_INVALID_ARG;
    return RESS_OK;
}

ress::WindowParams window_params(const ress_window_shape *s, float scale)
{
    ress::WindowParams p;
    memset(&p, 0, sizeof p);
    p.H = s->H;
    p.H_kv = s->H_kv;
    p.group = s->H / s->H_kv;
    p.n_q = s->n_q;
    p.n_k = s->n_k;
    p.q_offset = s->q_offset;
    ress::sights(s->frame, s->window, p.frame, p.window);
    p.frames = ress::divider(p.frame);
    p.groups = ress::divider(p.group);
    p.n_sink = s->n_sink;
    p.causal = s->causal != 0;
    p.n_qb = (s->n_q + 127) / 128;
    p.n_kb = (s->n_k + 127) / 128;
    p.scale = scale;
    p.scale_log2 = scale * 1.4426950408889634f;
    p.refs = ress::references(p.scale_log2);
    p.qs = s->q;
    p.ks = s->k;
    p.vs = s->v;
    p.os = s->o;
    return p;
}

size_t window_workspace(const ress_window_shape *s)
{
    if (s->H == 0) return 0;
    const int splits = ress::window_plan(s).splits;
    return splits == 1 ? 0 : align256((size_t)splits * s->H * s->n_q * 66 * sizeof(float));
}

// Per-query values (two of them), then the slices' sums.
size_t rows_bytes(const ress_window_shape *s) { return align256((size_t)s->H * s->n_q * sizeof(float)); }

size_t window_bwd_workspace(const ress_window_shape *s)
{
    const ress::WindowBwdPlan plan = ress::window_bwd_plan(s);
    const size_t cut = plan.slices > 1 || plan.sink_slices > 1 ? (size_t)s->H_kv * plan.items : 0;
    return 2 * rows_bytes(s) + cut * 2 * 128 * 64 * sizeof(float);
}

int check_decode(const ress_decode_shape *s)
{
    if (!s) return RESS_E_INVALID_ARG;
    int st = check_heads(s->H, s->H_kv);
    if (st != RESS_OK) return st;
    if (s->B < 0 || s->capacity < 0 || s->frame < 1 || s->window < 1 || s->n_sink < 0) return RESS_E_INVALID_ARG;
    if (s->D != kHead || s->B > RESS_MAX_BATCH || s->capacity > RESS_MAX_TOKENS) return RESS_E_UNSUPPORTED;
    return RESS_OK;
}

size_t decode_workspace(const ress_decode_shape *s)
{
    const int splits = ress::decode_splits(s);
    return splits == 1 ? 0 : align256((size_t)s->B * s->H * splits * 66 * sizeof(float));
}

bool batch_ok(int64_t stride) { return stride >= 0 && stride <= kMaxStride && stride % 8 == 0; }

}  // namespace

extern "C" {

int ress_layer_norm(const ress_norm_shape *shape, const void *x, const float *gamma, const float *beta, void *y,
                    float *mean, float *rstd, hipStream_t stream)
{
    int st = check_norm(shape, true);
    if (st != RESS_OK) return st;
    if ((mean == nullptr) != (rstd == nullptr)) return RESS_E_INVALID_ARG;
    if (shape->rows == 0) return RESS_OK;
    if (!x || !y || !aligned(x, dtype_size(shape->x_dtype)) || !aligned(y, dtype_size(shape->y_dtype)) ||
        !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean, 4) || !aligned(rstd, 4))
        return RESS_E_INVALID_ARG;
    if (!norm_alias_ok(y, shape->y_dtype, shape->y_stride, x, shape->x_dtype, shape->x_stride)) return RESS_E_INVALID_ARG;
    if (y == gamma || y == beta || (mean && (mean == rstd || mean == x || rstd == x || mean == y || rstd == y)))
        return RESS_E_INVALID_ARG;
    ress::NormParams p;
    p.rows = shape->rows;
    p.x_stride = shape->x_stride;
    p.y_stride = shape->y_stride;
    p.width = shape->width;
    p.eps = (float)shape->eps;
    p.x_f32 = shape->x_dtype == RESS_DTYPE_F32;
    p.y_f32 = shape->y_dtype == RESS_DTYPE_F32;
    p.x = x;
    p.gamma = gamma;
    p.beta = beta;
    p.y = y;
    p.mean = mean;
    p.rstd = rstd;
    return ress::launch_norm(p, stream) == hipSuccess ? RESS_OK : RESS_E_HIP;
}

int ress_layer_norm_bwd_workspace_size(const ress_norm_shape *shape, size_t *bytes)
{
    int st = check_norm(shape, false);
    if (st != RESS_OK) return st;
    if (!bytes) return RESS_E_INVALID_ARG;
    *bytes = norm_workspace(shape);
    return RESS_OK;
}

int ress_layer_norm_bwd(const ress_norm_shape *shape, const void *dy, const void *x, const float *gamma,
                        const float *mean, const float *rstd, void *dx, float *dgamma, float *dbeta, void *workspace,
                        size_t ws_bytes, hipStream_t stream)
{
    int st = check_norm(shape, false);
    if (st != RESS_OK) return st;
    const bool sums = dgamma || dbeta;
    if (shape->rows == 0 && !sums) return RESS_OK;
    if (shape->rows > 0) {
        const size_t xs = dtype_size(shape->x_dtype), ys = dtype_size(shape->y_dtype);
        if (!dy || !x || !mean || !rstd || !dx || !aligned(dy, ys) || !aligned(x, xs) || !aligned(dx, xs))
            return RESS_E_INVALID_ARG;
        if (!norm_alias_ok(dx, shape->x_dtype, shape->x_stride, dy, shape->y_dtype, shape->y_stride) || dx == gamma ||
            dx == mean || dx == rstd || dx == dgamma || dx == dbeta)
            return RESS_E_INVALID_ARG;
    }
    if (!aligned(gamma, 4) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(dgamma, 4) || !aligned(dbeta, 4))
        return RESS_E_INVALID_ARG;
    const void *ins[5] = {dy, x, gamma, mean, rstd};
    for (const void *in : ins)
        if (in && (in == dgamma || in == dbeta)) return RESS_E_INVALID_ARG;
    if (dgamma && dgamma == dbeta) return RESS_E_INVALID_ARG;
    if (sums && (!workspace || ws_bytes < norm_workspace(shape) || !aligned(workspace, 256))) return RESS_E_WORKSPACE;
    ress::NormBwdParams p;
    p.rows = shape->rows;
    p.x_stride = shape->x_stride;
    p.y_stride = shape->y_stride;
    p.width = shape->width;
    p.parts = ress::norm_bwd_parts(shape->rows);
    p.x_f32 = shape->x_dtype == RESS_DTYPE_F32;
    p.y_f32 = shape->y_dtype == RESS_DTYPE_F32;
    p.dy = dy;
    p.x = x;
    p.gamma = gamma;
    p.mean = mean;
    p.rstd = rstd;
    p.dx = dx;
    p.part = sums ? static_cast<float *>(workspace) : nullptr;
    p.dgamma = dgamma;
    p.dbeta = dbeta;
    return ress::launch_norm_bwd(p, stream) == hipSuccess ? RESS_OK : RESS_E_HIP;
}

int ress_rope(const ress_rope_shape *shape, const int32_t *pos, const void *q_in, const void *k_in, void *q_out,
              void *k_out, hipStream_t stream)
{
    if (!shape) return RESS_E_INVALID_ARG;
    const ress_rope_shape &s = *shape;
    int turned = 0, st = check_rope(s, turned);
    if (st != RESS_OK) return st;
    const ress_strides *in[2] = {&s.q, &s.k}, *out[2] = {&s.q_out, &s.k_out};
    const void *src[2] = {q_in, k_in};
    void *dst[2] = {q_out, k_out};
    const int heads[2] = {s.H, s.H_kv};
    const size_t size = dtype_size(s.dtype);
    for (int i = 0; i < 2; ++i) {
        if (heads[i] == 0 || s.N == 0) continue;
        if (!src[i] || !dst[i] || !pos || !aligned(src[i], size) || !aligned(dst[i], size) || !aligned(pos, 4))
            return RESS_E_INVALID_ARG;
        if (!strides_ok(*in[i], 1) || !strides_ok(*out[i], 1)) return RESS_E_INVALID_ARG;
        if (!disjoint(heads[i], out[i]->head, s.N, out[i]->token, s.D)) return RESS_E_INVALID_ARG;
        if (src[i] == dst[i] && !same(*in[i], *out[i])) return RESS_E_INVALID_ARG;
        if (dst[i] == pos || (heads[1 - i] && (dst[i] == src[1 - i] || dst[i] == dst[1 - i]))) return RESS_E_INVALID_ARG;
    }
    if (s.H + s.H_kv == 0 || s.N == 0) return RESS_OK;

    ress::RopeParams p;
    memset(&p, 0, sizeof p);
    for (int per = (int)(16 / size); per >= (int)(8 / size) && !p.chunk; per /= 2)
        if (rope_chunks(s, per, turned) && rope_aligned(s, per, src, dst)) p.chunk = per;
    rope_tables(s, turned, p);
    p.pos = pos;
    p.q_in = q_in;
    p.k_in = k_in;
    p.q_out = q_out;
    p.k_out = k_out;
    p.qi = s.q;
    p.ki = s.k;
    p.qo = s.q_out;
    p.ko = s.k_out;
    return ress::launch_rope(p, stream) == hipSuccess ? RESS_OK : RESS_E_HIP;
}

int ress_window_attn_workspace_size(const ress_window_shape *shape, size_t *bytes)
{
    int st = check_window(shape, false);
    if (st != RESS_OK) return st;
    if (!bytes) return RESS_E_INVALID_ARG;
    *bytes = window_workspace(shape);
    return RESS_OK;
}

int ress_window_attn(const ress_window_shape *shape, const void *q, const void *k, const void *v, float scale, void *o,
                     float *lse, void *workspace, size_t ws_bytes, hipStream_t stream)
{
    int st = check_window(shape, true);
    if (st != RESS_OK) return st;
    if (!scale_ok(scale)) return RESS_E_INVALID_ARG;
    if (shape->H == 0 || shape->n_q == 0) return RESS_OK;
    if (!q || !o || (shape->n_k > 0 && (!k || !v))) return RESS_E_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(o, 16) || !aligned(lse, 4))
        return RESS_E_INVALID_ARG;
    if (o == q || o == k || o == v || (lse && ((void *)lse == o || lse == q || lse == k || lse == v)))
        return RESS_E_INVALID_ARG;
    if (!disjoint(shape->H, shape->o.head, shape->n_q, shape->o.token, kHead)) return RESS_E_INVALID_ARG;
    const size_t need = window_workspace(shape);
    if (need && (!workspace || ws_bytes < need || !aligned(workspace, 256))) return RESS_E_WORKSPACE;
    const ress::WindowPlan plan = ress::window_plan(shape);
    ress::WindowParams p = window_params(shape, scale);
    p.q = static_cast<const uint16_t *>(q);
    p.k = static_cast<const uint16_t *>(k);
    p.v = static_cast<const uint16_t *>(v);
    p.o = static_cast<uint16_t *>(o);
    p.lse = lse;
    p.splits = plan.splits;
    p.n_qb = (p.n_q * plan.groups + 127) / 128;
    p.q_blocks = ress::divider(p.n_qb);
    if (plan.splits > 1) {
        p.part = static_cast<float *>(workspace);
        p.part_row = reinterpret_cast<float2 *>(p.part + (size_t)plan.splits * p.H * p.n_q * 64);
    }
    return ress::launch_window(p, plan.groups, stream) == hipSuccess ? RESS_OK : RESS_E_HIP;
}

int ress_window_attn_bwd_workspace_size(const ress_window_shape *shape, size_t *bytes)
{
    int st = check_window(shape, false);
    if (st != RESS_OK) return st;
    if (!bytes) return RESS_E_INVALID_ARG;
    *bytes = window_bwd_workspace(shape);
    return RESS_OK;
}

int ress_window_attn_bwd(const ress_window_shape *shape, const ress_window_grads *grads, const void *d_o, const void *q,
                         const void *k, const void *v, const void *o, const float *lse, float scale, void *dq, void *dk,
                         void *dv, void *workspace, size_t ws_bytes, hipStream_t stream)
{
    int st = check_window(shape, true);
    if (st != RESS_OK) return st;
    if (!grads || !scale_ok(scale)) return RESS_E_INVALID_ARG;
    if (!strides_ok(grads->d_o, 8) || !strides_ok(grads->dq, 8) || !strides_ok(grads->dk, 8) || !strides_ok(grads->dv, 8))
        return RESS_E_INVALID_ARG;
    if (shape->H == 0 || (shape->n_q == 0 && shape->n_k == 0)) return RESS_OK;
    if (shape->n_q > 0 && (!d_o || !q || !o || !lse || !dq)) return RESS_E_INVALID_ARG;
    if (shape->n_k > 0 && (!k || !v || !dk || !dv)) return RESS_E_INVALID_ARG;
    const void *ins[6] = {d_o, q, k, v, o, lse};
    void *outs[3] = {dq, dk, dv};
    for (const void *in : ins)
        if (!aligned(in, in == lse ? 4 : 16)) return RESS_E_INVALID_ARG;
    for (int i = 0; i < 3; ++i) {
        if (!aligned(outs[i], 16)) return RESS_E_INVALID_ARG;
        for (const void *in : ins)
            if (outs[i] && outs[i] == in) return RESS_E_INVALID_ARG;
        for (int e = 0; e < i; ++e)
            if (outs[i] && outs[i] == outs[e]) return RESS_E_INVALID_ARG;
    }
    if (!disjoint(shape->H, grads->dq.head, shape->n_q, grads->dq.token, kHead) ||
        !disjoint(shape->H_kv, grads->dk.head, shape->n_k, grads->dk.token, kHead) ||
        !disjoint(shape->H_kv, grads->dv.head, shape->n_k, grads->dv.token, kHead))
        return RESS_E_INVALID_ARG;
    const size_t rows = rows_bytes(shape), need = window_bwd_workspace(shape);
    if (need && (!workspace || ws_bytes < need || !aligned(workspace, 256))) return RESS_E_WORKSPACE;
    ress::WindowBwdParams b;
    b.w = window_params(shape, scale);
    // A query that sees one key has a probability of 1 whatever the logit, and dq and dk are 0 by the
    // formula. In these two calls, of no other query, they are written so; elsewhere such a query leaves in
    // them what float32 leaves of d_o v^T - delta.
    if (shape->n_k == 1 || (shape->frame == 1 && shape->window == 1 && shape->n_sink == 0)) b.w.scale = 0.f;
    b.w.q = static_cast<const uint16_t *>(q);
    b.w.k = static_cast<const uint16_t *>(k);
    b.w.v = static_cast<const uint16_t *>(v);
    b.w.o = static_cast<uint16_t *>(const_cast<void *>(o));
    b.w.lse = const_cast<float *>(lse);
    b.dos = grads->d_o;
    b.dqs = grads->dq;
    b.dks = grads->dk;
    b.dvs = grads->dv;
    b.d_o = static_cast<const uint16_t *>(d_o);
    b.dq = static_cast<uint16_t *>(dq);
    b.dk = static_cast<uint16_t *>(dk);
    b.dv = static_cast<uint16_t *>(dv);
    b.ndelta = static_cast<float *>(workspace);
    b.lse2 = reinterpret_cast<float *>(static_cast<char *>(workspace) + rows);
    const ress::WindowBwdPlan plan = ress::window_bwd_plan(shape);
    b.sink_blocks = plan.sink_blocks;
    b.sink_slices = plan.sink_slices;
    b.slices = plan.slices;
    b.items = plan.items;
    b.part = reinterpret_cast<float *>(static_cast<char *>(workspace) + 2 * rows);
    b.w.n_qb = (shape->n_q * plan.groups + 127) / 128;
    if (b.w.n_qb > 0) b.w.q_blocks = ress::divider(b.w.n_qb);
    return ress::launch_window_bwd(b, plan.groups, stream) == hipSuccess ? RESS_OK : RESS_E_HIP;
}

int ress_window_attn_decode_workspace_size(const ress_decode_shape *shape, size_t *bytes)
{
    int st = check_decode(shape);
    if (st != RESS_OK) return st;
    if (!bytes) return RESS_E_INVALID_ARG;
    *bytes = decode_workspace(shape);
    return RESS_OK;
}

int ress_window_attn_decode(const ress_decode_shape *shape, const void *q, const void *k, const void *v,
                            const int32_t *lens, float scale, void *o, void *workspace, size_t ws_bytes,
                            hipStream_t stream)
{
    int st = check_decode(shape);
    if (st != RESS_OK) return st;
    const ress_decode_shape &s = *shape;
    if (!scale_ok(scale)) return RESS_E_INVALID_ARG;
    if (!batch_ok(s.q_batch) || !batch_ok(s.q_head) || !batch_ok(s.k_batch) || !batch_ok(s.v_batch) ||
        !batch_ok(s.o_batch) || !batch_ok(s.o_head) || !strides_ok(s.k, 8) || !strides_ok(s.v, 8))
        return RESS_E_INVALID_ARG;
    if (s.B == 0 || s.H == 0) return RESS_OK;
    if (!q || !lens || !o || (s.capacity > 0 && (!k || !v))) return RESS_E_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(o, 16) || !aligned(lens, 4))
        return RESS_E_INVALID_ARG;
    if (o == q || o == k || o == v || o == lens) return RESS_E_INVALID_ARG;
    if (!disjoint(s.B, s.o_batch, s.H, s.o_head, kHead)) return RESS_E_INVALID_ARG;
    const size_t need = decode_workspace(shape);
    if (need && (!workspace || ws_bytes < need || !aligned(workspace, 256))) return RESS_E_WORKSPACE;
    ress::DecodeParams p;
    p.B = s.B;
    p.H = s.H;
    p.H_kv = s.H_kv;
    p.group = s.H / s.H_kv;
    p.capacity = s.capacity;
    ress::sights(s.frame, s.window, p.frame, p.window);
    p.frames = ress::divider(p.frame);
    p.n_sink = s.n_sink;
    p.splits = ress::decode_splits(shape);
    p.scale_log2 = scale * 1.4426950408889634f;
    p.q_batch = s.q_batch;
    p.q_head = s.q_head;
    p.k_batch = s.k_batch;
    p.v_batch = s.v_batch;
    p.o_batch = s.o_batch;
    p.o_head = s.o_head;
    p.ks = s.k;
    p.vs = s.v;
    p.q = static_cast<const uint16_t *>(q);
    p.k = static_cast<const uint16_t *>(k);
    p.v = static_cast<const uint16_t *>(v);
    p.lens = lens;
    p.o = static_cast<uint16_t *>(o);
    p.part = static_cast<float *>(workspace);
    return ress::launch_decode(p, stream) == hipSuccess ? RESS_OK : RESS_E_HIP;
}

}  // extern "C"
