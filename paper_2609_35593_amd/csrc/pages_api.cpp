// C ABI of ress_pages.h: argument validation, workspace layout and kernel launches.
// Every check runs on the host before anything is enqueued, so an error status
// means no device work and no output writes.
#include <math.h>
#include <string.h>

#include "checks.h"
#include "pages_internal.h"

namespace {

using namespace ress;

constexpr int64_t kMaxSlots = 0x7fffffff;

// Strides of [n_pages][heads][page][channels] whose furthest element's offset is below 2^62, multiples
// of `multiple`.
bool page_strides_ok(const ress_page_strides &s, int64_t n_pages, int64_t multiple)
{
    if (s.page < 0 || s.head < 0 || s.token < 0 || s.head > kMaxStride || s.token > kMaxTokenStride) return false;
    if (n_pages > 0 && s.page > ((int64_t)1 << 62) / n_pages) return false;
    return s.page % multiple == 0 && s.head % multiple == 0 && s.token % multiple == 0;
}

// Rows of `width` elements in three dimensions that do not overlap: taken from the smallest step up,
// each lies whole between two steps of the next.
bool disjoint3(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2, int64_t s2, int64_t width)
{
    int64_t n[3] = {n0, n1, n2}, s[3] = {s0, s1, s2};
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2 - i; ++j)
            if (s[j] > s[j + 1]) {
                const int64_t a = n[j], b = s[j];
                n[j] = n[j + 1], s[j] = s[j + 1];
                n[j + 1] = a, s[j + 1] = b;
            }
    __int128 extent = width;
    for (int i = 0; i < 3; ++i) {
        if (n[i] <= 1) continue;
        if (s[i] < extent) return false;
        extent += (__int128)(n[i] - 1) * s[i];
    }
    return true;
}

// ----------------------------------------------------------- norm of heads

int check_head_norm(const ress_head_norm_shape *s, int &turned)
{
    if (!s) return RESS_E_INVALID_ARG;
    const int st = check_rope(s->rope, turned);
    if (st != RESS_OK) return st;
    if (s->rope.inverse != 0 || (s->norm != RESS_HEAD_NORM_LAYER && s->norm != RESS_HEAD_NORM_RMS)) return RESS_E_INVALID_ARG;
    if (!((float)s->eps > 0.f) || !isfinite((float)s->eps)) return RESS_E_INVALID_ARG;
    return RESS_OK;
}

// One tensor of the norm's passes: [heads][N][D] by strides.
struct Tensor {
    const void *ptr;
    const ress_strides *strides;
    int heads;
    bool out;
};

// Pointers, strides, and that an output overlaps neither itself nor an equal pointer's other layout.
int check_tensors(const ress_rope_shape &s, const Tensor *t, int n)
{
    const size_t size = dtype_size(s.dtype);
    for (int i = 0; i < n; ++i) {
        if (t[i].heads == 0) continue;
        if (!t[i].ptr || !aligned(t[i].ptr, size) || !strides_ok(*t[i].strides, 1)) return RESS_E_INVALID_ARG;
        if (!t[i].out) continue;
        if (!disjoint(t[i].heads, t[i].strides->head, s.N, t[i].strides->token, s.D)) return RESS_E_INVALID_ARG;
    }
    return RESS_OK;
}

bool tensors_in_chunks(const ress_rope_shape &s, int per, const Tensor *t, int n)
{
    for (int i = 0; i < n; ++i)
        if (t[i].heads > 0 && (!aligned(t[i].ptr, per * dtype_size(s.dtype)) || !strides_ok(*t[i].strides, per))) return false;
    return true;
}

bool weights_ok(const float *const *w, int n, const void *const *outs, int n_outs)
{
    for (int i = 0; i < n; ++i) {
        if (!aligned(w[i], 4)) return false;
        for (int j = 0; j < n_outs; ++j)
            if (w[i] && w[i] == outs[j]) return false;
    }
    return true;
}

ChunkRuns chunk_runs(const ress_rope_shape &s, int turned, int per)
{
    ChunkRuns r;
    memset(&r, 0, sizeof r);
    if (per == 0) return r;
    if (s.layout != RESS_ROPE_SPLIT) {
        r.n = 1;
        r.half[0] = s.layout == RESS_ROPE_SECTIONS ? turned / 2 / per : 0;
        r.count[0] = turned / per;
        return r;
    }
    for (int a = 0, at = 0; a < s.n_axes; at += s.dims[a++]) {
        r.first[r.n] = at / per;
        r.half[r.n] = s.dims[a] / 2 / per;
        r.count[r.n] = s.dims[a] / per;
        r.pair[r.n++] = at / 2;
    }
    return r;
}

// The forward pass, into pages where `cache` is given.
int head_norm(const ress_head_norm_shape *shape, const ress_page_cache *cache, const int32_t *pos, const int32_t *slots,
              const void *q_in, const void *k_in, const void *v_in, const float *const (&weights)[4], void *q_out, void *k_out,
              void *v_out, hipStream_t stream)
{
    int turned = 0;
    const int st = check_head_norm(shape, turned);
    if (st != RESS_OK) return st;
    const ress_rope_shape &s = shape->rope;
    const size_t size = dtype_size(s.dtype);
    Tensor t[5] = {{q_in, &s.q, s.H, false}, {k_in, &s.k, s.H_kv, false}, {q_out, &s.q_out, s.H, true}};
    int n = 3;
    if (cache) {
        if (cache->n_pages < 0 || cache->page < 1) return RESS_E_INVALID_ARG;
        if (cache->page > RESS_MAX_TOKENS || (int64_t)cache->n_pages * cache->page > kMaxSlots) return RESS_E_UNSUPPORTED;
        t[n++] = {v_in, &cache->v_in, s.H_kv, false};
        if (s.H_kv > 0 && (!page_strides_ok(cache->k, cache->n_pages, 1) || !page_strides_ok(cache->v, cache->n_pages, 1) ||
                           !disjoint3(cache->n_pages, cache->k.page, s.H_kv, cache->k.head, cache->page, cache->k.token, s.D) ||
                           !disjoint3(cache->n_pages, cache->v.page, s.H_kv, cache->v.head, cache->page, cache->v.token, s.D)))
            return RESS_E_INVALID_ARG;
    } else {
        t[n++] = {k_out, &s.k_out, s.H_kv, true};
    }
    if (s.H + s.H_kv == 0 || s.N == 0) return RESS_OK;
    const int ct = check_tensors(s, t, n);
    if (ct != RESS_OK) return ct;
    if (!pos || !aligned(pos, 4) || (cache && (!slots || !aligned(slots, 4)))) return RESS_E_INVALID_ARG;
    const void *outs[3] = {s.H ? q_out : nullptr, s.H_kv ? k_out : nullptr, s.H_kv ? v_out : nullptr};
    if (cache && s.H_kv > 0 && cache->n_pages > 0) {
        if (!k_out || !v_out || !aligned(k_out, size) || !aligned(v_out, size) || k_out == v_out) return RESS_E_INVALID_ARG;
        for (int i = 1; i < 3; ++i)
            if (outs[i] == k_in || outs[i] == v_in) return RESS_E_INVALID_ARG;
    }
    for (int i = 0; i < 3; ++i)
        if (outs[i] && (outs[i] == pos || outs[i] == slots)) return RESS_E_INVALID_ARG;
    if (s.H && ((q_out == q_in && !same(s.q, s.q_out)) || (s.H_kv && (q_out == k_in || q_out == k_out || (cache && q_out == v_in)))))
        return RESS_E_INVALID_ARG;
    if (cache && s.H && s.H_kv && (v_out == q_in || q_out == v_out)) return RESS_E_INVALID_ARG;
    if (s.H && s.H_kv && k_out == q_in) return RESS_E_INVALID_ARG;
    if (!cache && s.H_kv && k_out == k_in && !same(s.k, s.k_out)) return RESS_E_INVALID_ARG;
    if (!weights_ok(weights, 4, outs, 3)) return RESS_E_INVALID_ARG;

    HeadNormParams p;
    memset(&p, 0, sizeof p);
    for (int per = (int)(16 / size); per >= (int)(8 / size) && !p.r.chunk; per /= 2) {
        if (!rope_chunks(s, per, turned) || !tensors_in_chunks(s, per, t, n)) continue;
        if (cache && s.H_kv > 0 &&
            (!aligned(k_out, per * size) || !aligned(v_out, per * size) || !page_strides_ok(cache->k, cache->n_pages, per) ||
             !page_strides_ok(cache->v, cache->n_pages, per)))
            continue;
        p.r.chunk = per;
    }
    rope_tables(s, turned, p.r);
    p.runs = chunk_runs(s, turned, p.r.chunk);
    p.r.pos = pos;
    p.r.q_in = q_in;
    p.r.k_in = k_in;
    p.r.q_out = q_out;
    p.r.k_out = k_out;
    p.r.qi = s.q;
    p.r.ki = s.k;
    p.r.qo = s.q_out;
    p.r.ko = s.k_out;
    p.layer = shape->norm == RESS_HEAD_NORM_LAYER;
    p.eps = (float)shape->eps;
    for (int i = 0; i < 2; ++i) {
        p.gamma[i] = weights[2 * i];
        p.beta[i] = weights[2 * i + 1];
    }
    if (cache) {
        p.slots = slots;
        p.n_slots = cache->n_pages * cache->page;
        p.pages = divider(cache->page);
        p.page = cache->page;
        p.v_in = v_in;
        p.v_out = v_out;
        p.vi = cache->v_in;
        p.kp = cache->k;
        p.vp = cache->v;
    }
    return launch_head_norm(p, stream) == hipSuccess ? RESS_OK : RESS_E_HIP;
}

size_t head_bwd_workspace(const ress_rope_shape &s)
{
    return align256((size_t)head_bwd_parts(s.H + s.H_kv, s.N) * 4 * s.D * sizeof(float));
}

// ------------------------------------------------------------------- pages

int check_pages(int B, int page, int n_pages, int max_pages, int64_t table_stride)
{
    if (B < 0 || page < 1 || n_pages < 0 || max_pages < 0 || table_stride < max_pages) return RESS_E_INVALID_ARG;
    if (B > RESS_MAX_BATCH || page > RESS_MAX_TOKENS || (int64_t)n_pages * page > kMaxSlots ||
        (int64_t)max_pages * page > RESS_MAX_TOKENS)
        return RESS_E_UNSUPPORTED;
    return table_stride > kMaxStride ? RESS_E_INVALID_ARG : RESS_OK;
}

int check_table(const ress_table_shape *s)
{
    if (!s || s->N < 0) return RESS_E_INVALID_ARG;
    const int st = check_pages(s->B, s->page, s->n_pages, s->max_pages, s->table_stride);
    if (st != RESS_OK) return st;
    return s->N > RESS_MAX_TOKENS ? RESS_E_UNSUPPORTED : RESS_OK;
}

// Pointers to int32; those of empty arrays may be null.
bool ints_ok(const void *const *ptr, const int64_t *entries, int n)
{
    for (int i = 0; i < n; ++i)
        if (!aligned(ptr[i], 4) || (entries[i] > 0 && !ptr[i])) return false;
    return true;
}

size_t release_workspace(const ress_table_shape *s) { return align256(((size_t)s->B + 1) * sizeof(int32_t)); }

// --------------------------------------------------------------- attention

int check_paged(const ress_paged_shape *s, bool strides)
{
    if (!s) return RESS_E_INVALID_ARG;
    int st = check_heads(s->H, s->H_kv);
    if (st != RESS_OK) return st;
    if (s->N < 0 || s->frame < 1 || s->window < 1 || s->n_sink < 0) return RESS_E_INVALID_ARG;
    st = check_pages(s->B, s->page, s->n_pages, s->max_pages, strides ? s->table_stride : s->max_pages);
    if (st != RESS_OK) return st;
    if (s->D != 64 || s->N > RESS_MAX_TOKENS) return RESS_E_UNSUPPORTED;
    if (strides && (!strides_ok(s->q, 8) || !strides_ok(s->o, 8) || !page_strides_ok(s->k, s->n_pages, 8) ||
                    !page_strides_ok(s->v, s->n_pages, 8)))
        return RESS_E_INVALID_ARG;
    return RESS_OK;
}

// Where a workspace's parts begin: outputs, references and sums, who shares a row, where sequences' blocks begin; its size.
struct PagedSpace {
    size_t rows, cuts, starts, bytes;
};
PagedSpace paged_space(const ress_paged_shape *s, const PagedPlan &plan)
{
    PagedSpace w = {0, 0, 0, 0};
    if (plan.splits > 1) {
        const size_t rows = plan.rows == 32 ? (size_t)plan.splits * s->H * s->N : (size_t)s->H_kv * plan.parts * 128;
        w.rows = rows * 64 * sizeof(float);
        w.cuts = w.rows + rows * sizeof(float2);
        w.starts = w.cuts + (plan.rows == 32 ? (size_t)s->H * s->N * sizeof(int32_t) : plan.blocks * sizeof(int4));
    }
    w.bytes = align256(w.starts + (plan.blocks > 0 && s->B > kMostScanned ? ((size_t)s->B + 1) * sizeof(int32_t) : 0));
    return w;
}

}  // namespace

extern "C" {

int ress_qk_norm_rope(const ress_head_norm_shape *shape, const int32_t *pos, const void *q_in, const void *k_in,
                      const float *q_gamma, const float *q_beta, const float *k_gamma, const float *k_beta, void *q_out,
                      void *k_out, hipStream_t stream)
{
    return head_norm(shape, nullptr, pos, nullptr, q_in, k_in, nullptr, {q_gamma, q_beta, k_gamma, k_beta}, q_out, k_out,
                     nullptr, stream);
}

int ress_qk_norm_rope_pages(const ress_head_norm_shape *shape, const ress_page_cache *cache, const int32_t *pos,
                            const int32_t *slots, const void *q_in, const void *k_in, const void *v_in,
                            const float *q_gamma, const float *q_beta, const float *k_gamma, const float *k_beta,
                            void *q_out, void *k_pages, void *v_pages, hipStream_t stream)
{
    if (!cache) return RESS_E_INVALID_ARG;
    return head_norm(shape, cache, pos, slots, q_in, k_in, v_in, {q_gamma, q_beta, k_gamma, k_beta}, q_out, k_pages, v_pages,
                     stream);
}

int ress_qk_norm_rope_bwd_workspace_size(const ress_head_norm_shape *shape, size_t *bytes)
{
    int turned = 0;
    const int st = check_head_norm(shape, turned);
    if (st != RESS_OK) return st;
    if (!bytes) return RESS_E_INVALID_ARG;
    *bytes = head_bwd_workspace(shape->rope);
    return RESS_OK;
}

int ress_qk_norm_rope_bwd(const ress_head_norm_shape *shape, const ress_head_norm_grads *grads, const int32_t *pos,
                          const void *dq_out, const void *dk_out, const void *q_in, const void *k_in,
                          const float *q_gamma, const float *k_gamma, void *dq, void *dk, float *q_dgamma,
                          float *q_dbeta, float *k_dgamma, float *k_dbeta, void *workspace, size_t ws_bytes,
                          hipStream_t stream)
{
    int turned = 0;
    const int st = check_head_norm(shape, turned);
    if (st != RESS_OK) return st;
    if (!grads) return RESS_E_INVALID_ARG;
    const ress_rope_shape &s = shape->rope;
    float *const sums[4] = {q_dgamma, q_dbeta, k_dgamma, k_dbeta};
    const bool wanted = q_dgamma || q_dbeta || k_dgamma || k_dbeta, work = s.H + s.H_kv > 0 && s.N > 0;
    const Tensor t[6] = {{dq_out, &grads->dq_out, s.H, false}, {q_in, &s.q, s.H, false}, {dq, &grads->dq, s.H, true},
                         {dk_out, &grads->dk_out, s.H_kv, false}, {k_in, &s.k, s.H_kv, false}, {dk, &grads->dk, s.H_kv, true}};
    if (!work && !wanted) return RESS_OK;
    if (work) {
        const int ct = check_tensors(s, t, 6);
        if (ct != RESS_OK) return ct;
        if (!pos || !aligned(pos, 4)) return RESS_E_INVALID_ARG;
        for (int i = 2; i < 6; i += 3) {
            if (t[i].heads == 0) continue;
            if (t[i].ptr == pos) return RESS_E_INVALID_ARG;
            for (int j = 0; j < 6; ++j) {
                if (j == i || t[j].heads == 0 || t[i].ptr != t[j].ptr) continue;
                // In place of its own gradient or input, laid out alike; nothing else.
                if (i / 3 != j / 3 || !same(*t[i].strides, *t[j].strides)) return RESS_E_INVALID_ARG;
            }
        }
    }
    const float *gamma[2] = {q_gamma, k_gamma};
    const void *outs[6] = {q_dgamma, q_dbeta, k_dgamma, k_dbeta, s.H ? dq : nullptr, s.H_kv ? dk : nullptr};
    if (!weights_ok(gamma, 2, outs, 6)) return RESS_E_INVALID_ARG;
    for (int i = 0; i < 4; ++i) {
        if (!sums[i]) continue;
        if (!aligned(sums[i], 4) || sums[i] == (const void *)pos) return RESS_E_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (sums[i] == sums[j]) return RESS_E_INVALID_ARG;
        for (int j = 0; j < 6; ++j)
            if (work && t[j].heads > 0 && t[j].ptr == sums[i]) return RESS_E_INVALID_ARG;
    }
    if (wanted && (!workspace || ws_bytes < head_bwd_workspace(s) || !aligned(workspace, 256))) return RESS_E_WORKSPACE;

    HeadNormBwdParams p;
    memset(&p, 0, sizeof p);
    const size_t size = dtype_size(s.dtype);
    for (int per = (int)(16 / size); per >= (int)(8 / size) && !p.r.chunk; per /= 2)
        if (rope_chunks(s, per, turned) && tensors_in_chunks(s, per, t, 6)) p.r.chunk = per;
    rope_tables(s, turned, p.r);
    p.runs = chunk_runs(s, turned, p.r.chunk);
    p.r.pos = pos;
    p.r.q_in = dq_out;
    p.r.k_in = dk_out;
    p.r.q_out = dq;
    p.r.k_out = dk;
    p.r.qi = grads->dq_out;
    p.r.ki = grads->dk_out;
    p.r.qo = grads->dq;
    p.r.ko = grads->dk;
    p.layer = shape->norm == RESS_HEAD_NORM_LAYER;
    p.eps = (float)shape->eps;
    p.gamma[0] = q_gamma;
    p.gamma[1] = k_gamma;
    p.x[0] = q_in;
    p.x[1] = k_in;
    p.xs[0] = s.q;
    p.xs[1] = s.k;
    p.part = wanted ? static_cast<float *>(workspace) : nullptr;
    for (int i = 0; i < 4; ++i) p.sums[i] = sums[i];
    return launch_head_norm_bwd(p, stream) == hipSuccess ? RESS_OK : RESS_E_HIP;
}

int ress_page_tables(const ress_table_shape *shape, const int32_t *lens, const int32_t *new_lens,
                     const int32_t *free_pages, const int32_t *n_free, int32_t *tables, int32_t *lens_out,
                     int32_t *n_free_out, int32_t *cu_q, int32_t *slots, int32_t *pos, int32_t *n_refused,
                     hipStream_t stream)
{
    const int st = check_table(shape);
    if (st != RESS_OK) return st;
    const ress_table_shape &s = *shape;
    const void *ptr[11] = {lens, new_lens, free_pages, n_free, tables, lens_out, n_free_out, cu_q, slots, pos, n_refused};
    const int64_t entries[11] = {s.B, s.B, s.n_pages, 1, (int64_t)s.B * s.max_pages, s.B, 1, 1, s.N, s.N, 0};
    if (!ints_ok(ptr, entries, 11)) return RESS_E_INVALID_ARG;
    for (int i = 4; i < 11; ++i)
        for (int j = 0; j < i; ++j) {
            const bool in_place = (i == 5 && j == 0) || (i == 6 && j == 3);
            if (ptr[i] && ptr[i] == ptr[j] && !in_place) return RESS_E_INVALID_ARG;
        }
    TableParams p;
    p.B = s.B;
    p.N = s.N;
    p.page = s.page;
    p.n_pages = s.n_pages;
    p.max_pages = s.max_pages;
    p.pages = divider(s.page);
    p.stride = s.table_stride;
    p.lens = lens;
    p.new_lens = new_lens;
    p.free_pages = free_pages;
    p.n_free = n_free;
    p.tables = tables;
    p.lens_out = lens_out;
    p.n_free_out = n_free_out;
    p.cu_q = cu_q;
    p.slots = slots;
    p.pos = pos;
    p.n_refused = n_refused;
    return launch_tables(p, stream) == hipSuccess ? RESS_OK : RESS_E_HIP;
}

int ress_pages_release_workspace_size(const ress_table_shape *shape, size_t *bytes)
{
    const int st = check_table(shape);
    if (st != RESS_OK) return st;
    if (!bytes) return RESS_E_INVALID_ARG;
    *bytes = release_workspace(shape);
    return RESS_OK;
}

int ress_pages_release(const ress_table_shape *shape, const int32_t *first, const int32_t *last, int32_t *tables,
                       int32_t *free_pages, const int32_t *n_free, int32_t *n_free_out, void *workspace, size_t ws_bytes,
                       hipStream_t stream)
{
    const int st = check_table(shape);
    if (st != RESS_OK) return st;
    const ress_table_shape &s = *shape;
    const void *ptr[6] = {first, last, n_free, tables, free_pages, n_free_out};
    const int64_t entries[6] = {s.B, s.B, 1, (int64_t)s.B * s.max_pages, s.n_pages, 1};
    if (!ints_ok(ptr, entries, 6)) return RESS_E_INVALID_ARG;
    for (int i = 3; i < 6; ++i)
        for (int j = 0; j < i; ++j)
            if (ptr[i] && ptr[i] == ptr[j] && !(i == 5 && j == 2)) return RESS_E_INVALID_ARG;
    if (!workspace || ws_bytes < release_workspace(shape) || !aligned(workspace, 256)) return RESS_E_WORKSPACE;
    ReleaseParams p;
    p.B = s.B;
    p.n_pages = s.n_pages;
    p.max_pages = s.max_pages;
    p.stride = s.table_stride;
    p.clear = s.clear != 0;
    p.first = first;
    p.last = last;
    p.n_free = n_free;
    p.tables = tables;
    p.free_pages = free_pages;
    p.n_free_out = n_free_out;
    p.counts = static_cast<int32_t *>(workspace);
    return launch_release(p, stream) == hipSuccess ? RESS_OK : RESS_E_HIP;
}

int ress_paged_attn_workspace_size(const ress_paged_shape *shape, size_t *bytes)
{
    const int st = check_paged(shape, false);
    if (st != RESS_OK) return st;
    if (!bytes) return RESS_E_INVALID_ARG;
    *bytes = paged_space(shape, paged_plan(shape)).bytes;
    return RESS_OK;
}

int ress_paged_attn(const ress_paged_shape *shape, const void *q, const void *k, const void *v, const int32_t *cu_q,
                    const int32_t *lens, const int32_t *tables, float scale, void *o, float *lse, void *workspace,
                    size_t ws_bytes, hipStream_t stream)
{
    const int st = check_paged(shape, true);
    if (st != RESS_OK) return st;
    const ress_paged_shape &s = *shape;
    if (!scale_ok(scale)) return RESS_E_INVALID_ARG;
    if (s.B == 0 || s.H == 0 || s.N == 0) return RESS_OK;
    const bool cached = s.n_pages > 0 && s.max_pages > 0;
    if (!q || !o || !cu_q || !lens || (cached && (!k || !v)) || (s.max_pages > 0 && !tables)) return RESS_E_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(o, 16) || !aligned(cu_q, 4) || !aligned(lens, 4) ||
        !aligned(tables, 4) || !aligned(lse, 4))
        return RESS_E_INVALID_ARG;
    const void *ins[6] = {q, k, v, cu_q, lens, tables};
    for (const void *in : ins)
        if (in && (in == o || in == lse)) return RESS_E_INVALID_ARG;
    if (o == lse) return RESS_E_INVALID_ARG;
    if (!disjoint(s.H, s.o.head, s.N, s.o.token, 64)) return RESS_E_INVALID_ARG;
    const PagedPlan plan = paged_plan(shape);
    const PagedSpace space = paged_space(shape, plan);
    if (space.bytes && (!workspace || ws_bytes < space.bytes || !aligned(workspace, 256))) return RESS_E_WORKSPACE;
    PagedParams p;
    memset(&p, 0, sizeof p);
    p.B = s.B;
    p.N = s.N;
    p.H = s.H;
    p.H_kv = s.H_kv;
    p.group = s.H / s.H_kv;
    p.page = s.page;
    p.n_pages = s.n_pages;
    p.max_pages = s.max_pages;
    p.capacity = s.max_pages * s.page;
    sights(s.frame, s.window, p.frame, p.window);
    p.n_sink = s.n_sink;
    p.frames = divider(p.frame);
    p.pages = divider(s.page);
    p.groups = divider(p.group);
    p.table_stride = s.table_stride;
    p.blocks = plan.blocks;
    p.splits = plan.splits;
    p.parts = plan.parts;
    if (plan.splits > 1) p.share = (float)s.H_kv / (float)plan.target;
    const int64_t reach = window_tokens(s.frame, s.window) + s.n_sink;
    p.most_keys = (int)(reach < p.capacity ? reach : p.capacity);
    p.scale = scale;
    p.scale_log2 = scale * 1.4426950408889634f;
    p.refs = references(p.scale_log2);
    p.qs = s.q;
    p.os = s.o;
    p.ks = s.k;
    p.vs = s.v;
    auto narrow = [&](const ress_page_strides &t) { return t.page / 8 <= 0xffffffff && t.token / 8 * s.page <= 0xffffffff; };
    p.eights = s.page % 8 == 0 && narrow(s.k) && narrow(s.v);
    p.alike = s.k.page == s.v.page && s.k.token == s.v.token;
    p.k_page16 = (uint32_t)(s.k.page / 8);
    p.k_token16 = (uint32_t)(s.k.token / 8);
    p.v_page16 = (uint32_t)(s.v.page / 8);
    p.v_token16 = (uint32_t)(s.v.token / 8);
    p.q = static_cast<const uint16_t *>(q);
    p.k = static_cast<const uint16_t *>(k);
    p.v = static_cast<const uint16_t *>(v);
    p.cu_q = cu_q;
    p.lens = lens;
    p.tables = tables;
    p.o = static_cast<uint16_t *>(o);
    p.lse = lse;
    char *const w = static_cast<char *>(workspace);
    if (s.B > kMostScanned) p.starts = reinterpret_cast<int32_t *>(w + space.starts);
    if (plan.splits > 1) {
        p.part = reinterpret_cast<float *>(w);
        p.part_row = reinterpret_cast<float2 *>(w + space.rows);
        if (plan.rows == 32)
            p.cuts = reinterpret_cast<int32_t *>(w + space.cuts);
        else
            p.cut = reinterpret_cast<int4 *>(w + space.cuts);
    }
    return launch_paged(p, plan.rows, stream) == hipSuccess ? RESS_OK : RESS_E_HIP;
}

}  // extern "C"
