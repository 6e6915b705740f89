// Entry points of the operators beside the mixer: linear attention with a decay for each head, layer norm,
// the router's balance loss.  Argument checks, workspace layout, sequencing.
#include <algorithm>
#include <cstring>

#include "handle.h"
#include "la.h"

namespace {

LaunchCtx open_ctx(swimba_handle *h, void *cuda_stream)
{
    h->prof.n = 0;
    return LaunchCtx{(cudaStream_t)cuda_stream, h->d_status, 0, &h->prof, (h->cfg.flags & SWIMBA_FLAG_CHECK_INDICES) != 0, &h->tmaps};
}
int close_ctx(swimba_handle *h, const LaunchCtx &ctx, int rc, const char *what)
{
    h->last_stream = ctx.stream;
    h->last_launches = ctx.launches;
    return rc == SWIMBA_OK ? rc : fail(h, rc, what);
}

// Rows of `width` elements, ld apart: 16-byte aligned rows that do not overlap.
int check_rows(swimba_handle *h, const void *p, int64_t ld, int64_t width)
{
    if (ld < width) return fail(h, SWIMBA_ERR_UNSUPPORTED_SHAPE, "a row stride is smaller than the row");
    if (ld > (int64_t)1 << 31) return fail(h, SWIMBA_ERR_UNSUPPORTED_SHAPE, "a row stride beyond 2^31 elements");
    if (!aligned16(p) || (ld * (int64_t)elt_size(h->cfg.dtype)) % 16 != 0)
        return fail(h, SWIMBA_ERR_MISALIGNED, "rows must start at multiples of 16 bytes");
    return SWIMBA_OK;
}
// Sequences of a call.  The kernels hold places in a sequence in 32 bits, one tile or segment beyond its end at most.
constexpr int kMaxSequences = 65535, kMaxTokens = 1 << 30;
bool la_sizes(int32_t B, int32_t L)
{
    return B <= kMaxSequences && L <= kMaxTokens && (int64_t)B * L < (int64_t)1 << 31;
}
int check_sizes(swimba_handle *h, int32_t B, int32_t L)
{
    if (B < 0 || L < 0) return fail(h, SWIMBA_ERR_UNSUPPORTED_SHAPE, "negative B or L");
    if (!la_sizes(B, L))
        return fail(h, SWIMBA_ERR_UNSUPPORTED_SHAPE, "more than 65535 sequences, 2^30 tokens of one, or B * L beyond 2^31");
    if ((int64_t)B * h->cfg.n_heads >= (int64_t)1 << 24)
        return fail(h, SWIMBA_ERR_UNSUPPORTED_SHAPE, "B * n_heads must stay below 2^24");
    if (h->cfg.head_dim % 8 != 0) return fail(h, SWIMBA_ERR_UNSUPPORTED_SHAPE, "head_dim must be a multiple of 8");
    return SWIMBA_OK;
}

// A sequence of rows ld apart: within the 2^40 bytes that the strides of a tensor map reach.
int check_reach(swimba_handle *h, int64_t ld, int32_t L)
{
    if (ld * (int64_t)elt_size(h->cfg.dtype) * L >= (int64_t)1 << 40)
        return fail(h, SWIMBA_ERR_UNSUPPORTED_SHAPE, "the rows of a sequence must lie within 2^40 bytes");
    return SWIMBA_OK;
}

// Workspace of a call of njobs jobs: the segment states of each, a copy of the states that enter, then (gradients with
// shared heads) the per-head gradients of queries and keys in fp32.
struct LaLayout {
    int seg_len, nseg, per;
    size_t seg[LA_MAX_JOBS], entry, dq, dk, total;
};
LaLayout la_layout(const swimba_handle *h, int B, int L, int njobs)
{
    const swimba_config &c = h->cfg;
    LaLayout l;
    la_plan(c.dtype, B, L, c.n_heads, c.d_state, c.head_dim, njobs, h->sm_count, &l.seg_len, &l.nseg, &l.per);
    size_t off = 0;
    for (int i = 0; i < njobs; ++i) {
        l.seg[i] = off;
        off += align_up(la_segment_bytes(c.dtype, B, L, c.n_heads, c.d_state, c.head_dim, njobs, h->sm_count));
    }
    l.entry = off;
    off += align_up((size_t)B * c.n_heads * c.head_dim * c.d_state * sizeof(float));
    l.dq = l.dk = off;
    if (njobs > 1 && c.n_groups != c.n_heads) {
        const size_t n = align_up((size_t)B * L * c.n_heads * c.d_state * sizeof(float));
        l.dk = l.dq + n;
        off = l.dk + n;
    }
    l.total = std::max<size_t>(off, kAlign);
    return l;
}

// States that enter and states that leave may be one tensor.  Blocks of one walk or job that read it need not have started
// when those of another are done and write it, so they read a copy.
int la_keep_entry(const swimba_handle *h, LaunchCtx &ctx, LaArgs &a, float *room)
{
    const float *shared = nullptr;
    for (int i = 0; i < a.njobs; ++i)
        for (int o = 0; o < a.njobs; ++o)
            if (a.job[i].s_in && a.job[i].s_in == a.job[o].s_out) shared = a.job[i].s_in;
    // (one job's whole walks: every block reads what it will write itself; walks of more than 64 values may be shared)
    if (!shared || (a.njobs == 1 && a.nseg == 1 && (h->cfg.head_dim <= 64 || a.L <= 128))) return SWIMBA_OK;
    const size_t n = (size_t)a.B * a.H * h->cfg.head_dim * h->cfg.d_state * sizeof(float);
    if (cudaMemcpyAsync(room, shared, n, cudaMemcpyDeviceToDevice, ctx.stream) != cudaSuccess) return SWIMBA_ERR_CUDA;
    for (int i = 0; i < a.njobs; ++i)
        if (a.job[i].s_in == shared) a.job[i].s_in = room;
    return SWIMBA_OK;
}

}  // namespace

extern "C" {

size_t swimba_linear_attention_workspace_bytes(const swimba_handle *h, int32_t B, int32_t L)
{
    if (!h || B <= 0 || L <= 0 || !la_sizes(B, L)) return 0;
    return la_layout(h, B, L, 1).total;
}

int swimba_linear_attention(swimba_handle *h, const float *log_decay, const void *q, int64_t ldq, const void *k,
                            int64_t ldk, const void *v, int64_t ldv, const float *state_in, int32_t B, int32_t L,
                            float scale, void *o, float *state_out, void *workspace, size_t workspace_bytes,
                            void *cuda_stream)
{
    if (!h) return SWIMBA_ERR_NULL_ARG;
    h->err[0] = 0;
    int rc = check_sizes(h, B, L);
    if (rc != SWIMBA_OK) return rc;
    if (B == 0 || L == 0) { h->last_launches = 0; return SWIMBA_OK; }
    if (!log_decay || !q || !k || !v || !o || !workspace)
        return fail(h, SWIMBA_ERR_NULL_ARG, "log_decay, q, k, v, o or workspace is NULL");
    const swimba_config &c = h->cfg;
    const int64_t GN = (int64_t)c.n_groups * c.d_state, HP = (int64_t)c.n_heads * c.head_dim;
    if ((rc = check_rows(h, q, ldq, GN)) != SWIMBA_OK || (rc = check_rows(h, k, ldk, GN)) != SWIMBA_OK ||
        (rc = check_rows(h, v, ldv, HP)) != SWIMBA_OK)
        return rc;
    for (int64_t ld : {ldq, ldk, ldv, HP})
        if ((rc = check_reach(h, ld, L)) != SWIMBA_OK) return rc;
    if (!aligned16(log_decay) || !aligned16(state_in) || !aligned16(o) || !aligned16(state_out) || !aligned16(workspace))
        return fail(h, SWIMBA_ERR_MISALIGNED, "tensors must be 16-byte aligned");
    const LaLayout l = la_layout(h, B, L, 1);
    if (workspace_bytes < l.total) return fail(h, SWIMBA_ERR_WORKSPACE_TOO_SMALL, "workspace too small");
    if ((rc = set_device(h)) != SWIMBA_OK) return rc;
    LaunchCtx ctx = open_ctx(h, cuda_stream);
    LaArgs a = {};
    a.njobs = 1;
    a.log_decay = log_decay;
    a.B = B; a.L = L; a.H = c.n_heads;
    a.seg_len = l.seg_len; a.nseg = l.nseg; a.per = l.per;
    const int r = c.n_heads / c.n_groups;
    a.job[0] = LaJob{q, k, v, ldq, ldk, ldv, r, r, 1, c.d_state, c.head_dim, 0, 0, state_in, state_out, o, HP, 0,
                     scale, scale, 1.f, (float *)((char *)workspace + l.seg[0])};
    rc = la_keep_entry(h, ctx, a, (float *)((char *)workspace + l.entry));
    if (rc == SWIMBA_OK) rc = launch_la(ctx, c.dtype, a, h->sm_count);
    return close_ctx(h, ctx, rc, "linear attention launch failed");
}

size_t swimba_linear_attention_backward_workspace_bytes(const swimba_handle *h, int32_t B, int32_t L)
{
    if (!h || B <= 0 || L <= 0 || !la_sizes(B, L)) return 0;
    return la_layout(h, B, L, 3).total;
}

int swimba_linear_attention_backward(swimba_handle *h, const float *log_decay, const void *q, int64_t ldq,
                                     const void *k, int64_t ldk, const void *v, int64_t ldv, const float *state_in,
                                     const void *d_o, const float *d_state_out, int32_t B, int32_t L, float scale,
                                     void *dq, void *dk, void *dv, float *d_state_in, void *workspace,
                                     size_t workspace_bytes, void *cuda_stream)
{
    if (!h) return SWIMBA_ERR_NULL_ARG;
    h->err[0] = 0;
    int rc = check_sizes(h, B, L);
    if (rc != SWIMBA_OK) return rc;
    if (B == 0 || L == 0) { h->last_launches = 0; return SWIMBA_OK; }
    if (!log_decay || !q || !k || !v || !d_o || !dq || !dk || !dv || !workspace)
        return fail(h, SWIMBA_ERR_NULL_ARG, "log_decay, q, k, v, d_o, dq, dk, dv or workspace is NULL");
    const swimba_config &c = h->cfg;
    const int64_t GN = (int64_t)c.n_groups * c.d_state, HN = (int64_t)c.n_heads * c.d_state,
                  HP = (int64_t)c.n_heads * c.head_dim;
    if ((rc = check_rows(h, q, ldq, GN)) != SWIMBA_OK || (rc = check_rows(h, k, ldk, GN)) != SWIMBA_OK ||
        (rc = check_rows(h, v, ldv, HP)) != SWIMBA_OK || (rc = check_rows(h, d_o, HP, HP)) != SWIMBA_OK)
        return rc;
    for (int64_t ld : {ldq, ldk, ldv, HP, HN})
        if ((rc = check_reach(h, ld, L)) != SWIMBA_OK) return rc;
    if (!aligned16(log_decay) || !aligned16(state_in) || !aligned16(d_state_out) || !aligned16(dq) || !aligned16(dk) ||
        !aligned16(dv) || !aligned16(d_state_in) || !aligned16(workspace))
        return fail(h, SWIMBA_ERR_MISALIGNED, "tensors must be 16-byte aligned");
    const LaLayout l = la_layout(h, B, L, 3);
    if (workspace_bytes < l.total) return fail(h, SWIMBA_ERR_WORKSPACE_TOO_SMALL, "workspace too small");
    if ((rc = set_device(h)) != SWIMBA_OK) return rc;
    LaunchCtx ctx = open_ctx(h, cuda_stream);
    char *ws = (char *)workspace;
    LaArgs a = {};
    a.njobs = 3;
    a.log_decay = log_decay;
    a.B = B; a.L = L; a.H = c.n_heads;
    a.seg_len = l.seg_len; a.nseg = l.nseg; a.per = l.per;
    const int r = c.n_heads / c.n_groups, N = c.d_state, P = c.head_dim;
    const bool shared = r > 1;
    void *gq = shared ? (void *)(ws + l.dq) : dq, *gk = shared ? (void *)(ws + l.dk) : dk;
    float *seg[3];
    for (int i = 0; i < 3; ++i) seg[i] = (float *)(ws + l.seg[i]);
    a.job[0] = LaJob{d_o, v, k, HP, ldv, ldk, 1, 1, r, P, N, 0, 1, state_in, nullptr, gq, HN, shared, scale, scale, 1.f, seg[0]};
    a.job[1] = LaJob{v, d_o, q, ldv, HP, ldq, 1, 1, r, P, N, 1, 1, d_state_out, nullptr, gk, HN, shared, scale, 1.f, scale, seg[1]};
    a.job[2] = LaJob{k, q, d_o, ldk, ldq, HP, r, r, 1, N, P, 1, 0, d_state_out, d_state_in, dv, HP, 0, scale, 1.f, scale, seg[2]};
    rc = la_keep_entry(h, ctx, a, (float *)(ws + l.entry));
    if (rc == SWIMBA_OK) rc = launch_la(ctx, c.dtype, a, h->sm_count);
    if (rc == SWIMBA_OK && shared) {
        rc = launch_la_head_sum(ctx, c.dtype, (const float *)gq, (int64_t)B * L, c.n_groups, r, N, dq);
        if (rc == SWIMBA_OK)
            rc = launch_la_head_sum(ctx, c.dtype, (const float *)gk, (int64_t)B * L, c.n_groups, r, N, dk);
    }
    return close_ctx(h, ctx, rc, "linear attention gradient launch failed");
}

int swimba_linear_attention_step(swimba_handle *h, const float *log_decay, const void *q, int64_t ldq, const void *k,
                                 int64_t ldk, const void *v, int64_t ldv, const float *state_in, int32_t B, float scale,
                                 void *o, float *state_out, void *cuda_stream)
{
    if (!h) return SWIMBA_ERR_NULL_ARG;
    h->err[0] = 0;
    int rc = check_sizes(h, B, 1);
    if (rc != SWIMBA_OK) return rc;
    if (B == 0) { h->last_launches = 0; return SWIMBA_OK; }
    if (!log_decay || !q || !k || !v || !state_in || !o || !state_out)
        return fail(h, SWIMBA_ERR_NULL_ARG, "log_decay, q, k, v, state_in, o or state_out is NULL");
    const swimba_config &c = h->cfg;
    const int64_t GN = (int64_t)c.n_groups * c.d_state, HP = (int64_t)c.n_heads * c.head_dim;
    if ((rc = check_rows(h, q, ldq, GN)) != SWIMBA_OK || (rc = check_rows(h, k, ldk, GN)) != SWIMBA_OK ||
        (rc = check_rows(h, v, ldv, HP)) != SWIMBA_OK)
        return rc;
    if (!aligned16(log_decay) || !aligned16(state_in) || !aligned16(o) || !aligned16(state_out))
        return fail(h, SWIMBA_ERR_MISALIGNED, "tensors must be 16-byte aligned");
    if ((rc = set_device(h)) != SWIMBA_OK) return rc;
    LaunchCtx ctx = open_ctx(h, cuda_stream);
    rc = launch_la_step(ctx, c.dtype, log_decay, q, ldq, k, ldk, v, ldv, state_in, B, c.n_heads, c.n_groups, c.head_dim,
                        c.d_state, scale, h->sm_count, o, state_out);
    return close_ctx(h, ctx, rc, "linear attention step launch failed");
}

// ------------------------------------------------------------------------------------------ layer norm

namespace {
constexpr int kMaxNormWidth = 16384;
int check_norm(swimba_handle *h, const void *x, int64_t ldx, int64_t rows, int32_t groups, int32_t width)
{
    if (rows < 0 || groups <= 0 || width <= 0 || width % 8 != 0 || width > kMaxNormWidth || groups > 65535)
        return fail(h, SWIMBA_ERR_UNSUPPORTED_SHAPE, "rows, groups or width out of range (width % 8 == 0, up to 16384)");
    if (rows >= (int64_t)1 << 40) return fail(h, SWIMBA_ERR_UNSUPPORTED_SHAPE, "too many rows");
    return rows > 0 && x ? check_rows(h, x, ldx, (int64_t)groups * width) : SWIMBA_OK;
}
}  // namespace

int swimba_layer_norm(swimba_handle *h, const void *x, int64_t ldx, const float *weight, const float *bias, int64_t rows,
                      int32_t groups, int32_t width, float eps, void *y, float *mean, float *rstd, void *cuda_stream)
{
    if (!h) return SWIMBA_ERR_NULL_ARG;
    h->err[0] = 0;
    int rc = check_norm(h, x, ldx, rows, groups, width);
    if (rc != SWIMBA_OK) return rc;
    if (rows == 0) { h->last_launches = 0; return SWIMBA_OK; }
    if (!x || !y) return fail(h, SWIMBA_ERR_NULL_ARG, "x or y is NULL");
    if (!aligned16(weight) || !aligned16(bias) || !aligned16(y) || !aligned16(mean) || !aligned16(rstd))
        return fail(h, SWIMBA_ERR_MISALIGNED, "tensors must be 16-byte aligned");
    if ((rc = set_device(h)) != SWIMBA_OK) return rc;
    LaunchCtx ctx = open_ctx(h, cuda_stream);
    rc = launch_layer_norm(ctx, h->cfg.dtype, x, ldx, weight, bias, rows, groups, width, eps, h->sm_count, y, mean, rstd);
    return close_ctx(h, ctx, rc, "layer norm launch failed");
}

size_t swimba_layer_norm_workspace_bytes(const swimba_handle *h, int64_t rows, int32_t groups, int32_t width)
{
    if (!h || rows <= 0 || groups <= 0 || width <= 0 || width % 8 != 0 || width > kMaxNormWidth || groups > 65535) return 0;
    return align_up(layer_norm_partial_bytes(rows, groups, width, h->sm_count));
}

int swimba_layer_norm_backward(swimba_handle *h, const void *dy, const void *x, int64_t ldx, const float *weight,
                               const float *mean, const float *rstd, int64_t rows, int32_t groups, int32_t width,
                               void *dx, float *dweight, float *dbias, void *workspace, size_t workspace_bytes,
                               void *cuda_stream)
{
    if (!h) return SWIMBA_ERR_NULL_ARG;
    h->err[0] = 0;
    int rc = check_norm(h, x, ldx, rows, groups, width);
    if (rc != SWIMBA_OK) return rc;
    const bool grads = dweight || dbias;
    if (!aligned16(dweight) || !aligned16(dbias)) return fail(h, SWIMBA_ERR_MISALIGNED, "tensors must be 16-byte aligned");
    if (rows > 0) {
        if (!dy || !x || !mean || !rstd || !dx) return fail(h, SWIMBA_ERR_NULL_ARG, "dy, x, mean, rstd or dx is NULL");
        if (!aligned16(dy) || !aligned16(weight) || !aligned16(mean) || !aligned16(rstd) || !aligned16(dx) || !aligned16(workspace))
            return fail(h, SWIMBA_ERR_MISALIGNED, "tensors must be 16-byte aligned");
        if (grads && !workspace) return fail(h, SWIMBA_ERR_NULL_ARG, "workspace is NULL");
        if (grads && workspace_bytes < swimba_layer_norm_workspace_bytes(h, rows, groups, width))
            return fail(h, SWIMBA_ERR_WORKSPACE_TOO_SMALL, "workspace too small");
    }
    if ((rc = set_device(h)) != SWIMBA_OK) return rc;
    if (rows == 0) {          // sums over no rows
        const size_t n = (size_t)groups * width * sizeof(float);
        h->last_launches = 0;
        h->last_stream = (cudaStream_t)cuda_stream;
        if ((dweight && cudaMemsetAsync(dweight, 0, n, h->last_stream) != cudaSuccess) ||
            (dbias && cudaMemsetAsync(dbias, 0, n, h->last_stream) != cudaSuccess))
            return fail(h, SWIMBA_ERR_CUDA, "clearing the gradients failed");
        return SWIMBA_OK;
    }
    LaunchCtx ctx = open_ctx(h, cuda_stream);
    rc = launch_layer_norm_backward(ctx, h->cfg.dtype, dy, x, ldx, weight, mean, rstd, rows, groups, width, h->sm_count, dx,
                                    dweight, dbias, grads ? (float *)workspace : nullptr);
    return close_ctx(h, ctx, rc, "layer norm gradient launch failed");
}

// ------------------------------------------------------------------------------------------ balance loss

size_t swimba_balance_loss_workspace_bytes(const swimba_handle *h, int64_t T)
{
    if (!h || T <= 0 || T * h->cfg.top_k >= (int64_t)1 << 31) return 0;
    return balance_workspace_bytes(h->cfg.dtype, T, h->cfg.d_model, h->cfg.n_experts, h->sm_count);
}

int swimba_balance_loss(swimba_handle *h, const swimba_weights *w, const void *u, const int32_t *topk_idx,
                        const uint8_t *valid, int64_t T, float coef, float *loss, int32_t *counts, float *mean_prob,
                        float *dW_router, int32_t accumulate, void *du, void *workspace, size_t workspace_bytes,
                        void *cuda_stream)
{
    if (!h) return SWIMBA_ERR_NULL_ARG;
    h->err[0] = 0;
    const swimba_config &c = h->cfg;
    if (T < 0 || T * c.top_k >= (int64_t)1 << 31)
        return fail(h, SWIMBA_ERR_UNSUPPORTED_SHAPE, "T out of range (T * top_k must stay below 2^31)");
    if (T == 0) { h->last_launches = 0; return SWIMBA_OK; }
    if (!w || !w->W_router) return fail(h, SWIMBA_ERR_NULL_ARG, "W_router is NULL");
    if (!u || !topk_idx || !loss || !workspace) return fail(h, SWIMBA_ERR_NULL_ARG, "u, topk_idx, loss or workspace is NULL");
    if (!aligned16(w->W_router) || !aligned16(u) || !aligned16(topk_idx) || !aligned16(loss) || !aligned16(counts) ||
        !aligned16(mean_prob) || !aligned16(dW_router) || !aligned16(du) || !aligned16(workspace))
        return fail(h, SWIMBA_ERR_MISALIGNED, "tensors must be 16-byte aligned");
    if (workspace_bytes < swimba_balance_loss_workspace_bytes(h, T))
        return fail(h, SWIMBA_ERR_WORKSPACE_TOO_SMALL, "workspace too small");
    int rc = set_device(h);
    if (rc != SWIMBA_OK) return rc;
    LaunchCtx ctx = open_ctx(h, cuda_stream);
    rc = launch_balance(ctx, c.dtype, u, w->W_router, topk_idx, valid, T, c.d_model, c.n_experts, c.top_k, coef,
                        h->sm_count, loss, counts, mean_prob, dW_router, accumulate != 0, du, workspace);
    return close_ctx(h, ctx, rc, "balance loss launch failed");
}

}  // extern "C"
