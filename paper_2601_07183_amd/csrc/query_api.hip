// C entries of the query side: argument checks only.
#include "query_ops.h"

#define FAIL(code, ...)              \
    do {                             \
        rairs_set_error(__VA_ARGS__); \
        return (code);               \
    } while (0)

static int check_projection(const rairs_projection_t *p, int64_t n)
{
    if (!p) FAIL(RAIRS_EINVAL, "projection is NULL");
    if (p->dtype != RAIRS_F32 && p->dtype != RAIRS_BF16) FAIL(RAIRS_EINVAL, "projection type %d: need RAIRS_F32 or RAIRS_BF16", p->dtype);
    if (p->d_in < 1 || p->d_out < 1) FAIL(RAIRS_EINVAL, "projection shape %d x %d: need both >= 1", p->d_out, p->d_in);
    if (p->d_in > RAIRS_MAX_WIDTH || p->d_out > RAIRS_MAX_WIDTH)
        FAIL(RAIRS_EUNSUPPORTED, "projection shape %d x %d above the built limit %d", p->d_out, p->d_in, RAIRS_MAX_WIDTH);
    if (p->n_adapters < 0) FAIL(RAIRS_EINVAL, "n_adapters is negative");
    if (p->n_adapters > RAIRS_MAX_ADAPTERS) FAIL(RAIRS_EUNSUPPORTED, "n_adapters=%d above the built limit %d", p->n_adapters, RAIRS_MAX_ADAPTERS);
    if (p->n_adapters > 0 && p->rank < 1) FAIL(RAIRS_EINVAL, "rank=%d: need rank >= 1", p->rank);
    if (p->n_adapters > 0 && p->rank > RAIRS_MAX_RANK) FAIL(RAIRS_EUNSUPPORTED, "rank=%d above the built limit %d", p->rank, RAIRS_MAX_RANK);
    if (n < 0) FAIL(RAIRS_EINVAL, "n is negative");
    if (n > RAIRS_MAX_ROWS) FAIL(RAIRS_EUNSUPPORTED, "n=%lld above the built limit %d", (long long)n, RAIRS_MAX_ROWS);
    return RAIRS_OK;
}

static int check_rows(const char *what, const void *p, int64_t ld, int64_t cols, int width)
{
    if (!p) FAIL(RAIRS_EINVAL, "%s is NULL", what);
    if ((uintptr_t)p % width) FAIL(RAIRS_EINVAL, "%s is not aligned to its type", what);
    if (ld < cols) FAIL(RAIRS_EINVAL, "row stride %lld of %s is less than its %lld columns", (long long)ld, what, (long long)cols);
    if (ld > (1ll << 31)) FAIL(RAIRS_EUNSUPPORTED, "row stride %lld of %s above the built limit", (long long)ld, what);
    return RAIRS_OK;
}

static int check_ws(const void *ws, size_t have, size_t need)
{
    if (need == 0) return RAIRS_OK;
    if (!ws) FAIL(RAIRS_EWORKSPACE, "workspace is NULL, %zu bytes needed", need);
    if ((uintptr_t)ws % 256) FAIL(RAIRS_EINVAL, "workspace is not 256-byte aligned");
    if (have < need) FAIL(RAIRS_EWORKSPACE, "workspace of %zu bytes, %zu needed", have, need);
    return RAIRS_OK;
}

#define TRY(call)              \
    do {                       \
        const int rc_ = (call); \
        if (rc_) return rc_;   \
    } while (0)

// (an address that is not null where no workspace is needed: the runs take a null one as "count only")
static void *ws_or_any(void *ws) { return ws ? ws : (void *)256; }

extern "C" size_t rairs_project_workspace_bytes(const rairs_projection_t *p, int64_t n)
{
    if (check_projection(p, n) || n == 0) return 0;
    ProjectArgs g = {};
    g.p = *p;
    g.n = n;
    size_t bytes = 0;
    rairs_run_project(g, nullptr, &bytes, nullptr);
    return bytes;
}

static int check_weights(const rairs_projection_t *p)
{
    const int w = dtype_width(p->dtype);
    TRY(check_rows("W", p->W, p->d_in, p->d_in, w));
    if (p->n_adapters == 0) return RAIRS_OK;
    TRY(check_rows("A", p->A, p->d_in, p->d_in, w));
    TRY(check_rows("B", p->B, p->rank, p->rank, w));
    return RAIRS_OK;
}

extern "C" int rairs_project(const rairs_projection_t *p, const void *d_x, int64_t ld_x, int64_t n, const int32_t *d_adapter, void *d_y,
                             int64_t ld_y, int y_dtype, void *d_ws, size_t ws_bytes, void *hip_stream)
{
    TRY(check_projection(p, n));
    if (y_dtype != RAIRS_F32 && y_dtype != p->dtype) FAIL(RAIRS_EINVAL, "output type %d: need RAIRS_F32 or the projection's", y_dtype);
    if (n == 0) return RAIRS_OK;
    TRY(check_weights(p));
    TRY(check_rows("d_x", d_x, ld_x, p->d_in, dtype_width(p->dtype)));
    TRY(check_rows("d_y", d_y, ld_y, p->d_out, dtype_width(y_dtype)));
    TRY(check_ws(d_ws, ws_bytes, rairs_project_workspace_bytes(p, n)));
    ProjectArgs g = {};
    g.p = *p;
    g.x = d_x; g.ldx = ld_x; g.n = n; g.adapter = d_adapter;
    g.y = d_y; g.ldy = ld_y; g.ytype = y_dtype;
    return rairs_run_project(g, ws_or_any(d_ws), nullptr, (hipStream_t)hip_stream);
}

extern "C" size_t rairs_project_backward_workspace_bytes(const rairs_projection_t *p, int64_t n)
{
    if (check_projection(p, n) || n == 0) return 0;
    ProjectArgs g = {};
    g.p = *p;
    g.n = n;
    size_t bytes = 0;
    rairs_run_project_backward(g, nullptr, &bytes, nullptr);
    return bytes;
}

extern "C" int rairs_project_backward(const rairs_projection_t *p, const void *d_x, int64_t ld_x, int64_t n, const int32_t *d_adapter,
                                      const void *d_dy, int64_t ld_dy, void *d_dx, int64_t ld_dx, void *d_dA, void *d_dB, void *d_ws,
                                      size_t ws_bytes, void *hip_stream)
{
    TRY(check_projection(p, n));
    const int w = dtype_width(p->dtype);
    if (!d_dA != !d_dB) FAIL(RAIRS_EINVAL, "d_dA and d_dB: both or neither");
    if (p->n_adapters == 0 && d_dA) FAIL(RAIRS_EINVAL, "no adapters to have gradients");
    if (d_dA && ((uintptr_t)d_dA % w || (uintptr_t)d_dB % w)) FAIL(RAIRS_EINVAL, "d_dA or d_dB is not aligned to its type");
    if (n > 0) {
        TRY(check_weights(p));
        TRY(check_rows("d_dy", d_dy, ld_dy, p->d_out, w));
        if (d_dA) TRY(check_rows("d_x", d_x, ld_x, p->d_in, w));
        if (d_dx) TRY(check_rows("d_dx", d_dx, ld_dx, p->d_in, w));
        TRY(check_ws(d_ws, ws_bytes, rairs_project_backward_workspace_bytes(p, n)));
    }
    ProjectArgs g = {};
    g.p = *p;
    g.x = d_x; g.ldx = ld_x; g.n = n; g.adapter = d_adapter;
    g.dy = d_dy; g.lddy = ld_dy; g.dx = d_dx; g.lddx = ld_dx; g.da = d_dA; g.db = d_dB;
    return rairs_run_project_backward(g, ws_or_any(d_ws), nullptr, (hipStream_t)hip_stream);
}

extern "C" int rairs_search_projected(rairs_index_t *h, const rairs_projection_t *p, const void *d_x, int64_t ld_x, int64_t n,
                                      const int32_t *d_adapter, float *d_queries, int k, int nprobe, int refine_k, int64_t *d_out_ids,
                                      float *d_out_dists, void *d_ws, size_t ws_bytes, void *hip_stream)
{
    if (!h) FAIL(RAIRS_EINVAL, "null handle");
    TRY(check_projection(p, n));
    if (p->d_out != h->v.d) FAIL(RAIRS_EINVAL, "the projection's d_out=%d is not the index's d=%d", p->d_out, h->v.d);
    // (what the search would refuse is refused before anything is enqueued)
    TRY(rairs_search_ready(h, n, k, nprobe, refine_k));
    if (n > 0 && (!d_out_ids || !d_out_dists)) FAIL(RAIRS_EINVAL, "null device pointer");
    TRY(rairs_project(p, d_x, ld_x, n, d_adapter, d_queries, p->d_out, RAIRS_F32, d_ws, ws_bytes, hip_stream));
    return rairs_search(h, d_queries, n, k, nprobe, refine_k, d_out_ids, d_out_dists, hip_stream);
}

extern "C" int rairs_index_table(const rairs_index_t *h, rairs_table_t *out)
{
    if (!h || !out) FAIL(RAIRS_EINVAL, "null argument");
    *out = rairs_table_t{};
    out->vectors = h->v.raw;
    out->ld = out->d = h->v.d;
    out->V = h->v.ntotal;
    out->dtype = h->v.raw_u8 ? RAIRS_U8 : RAIRS_F32;
    out->scale = 1.0f;
    return RAIRS_OK;
}

static int check_table(const rairs_table_t *t, int64_t n, int q_dtype)
{
    if (!t) FAIL(RAIRS_EINVAL, "table is NULL");
    if (t->dtype != RAIRS_F32 && t->dtype != RAIRS_BF16 && t->dtype != RAIRS_U8) FAIL(RAIRS_EINVAL, "unknown table type %d", t->dtype);
    if (q_dtype != (t->dtype == RAIRS_U8 ? RAIRS_F32 : t->dtype)) FAIL(RAIRS_EINVAL, "queries of type %d for a table of type %d", q_dtype, t->dtype);
    if (t->d < 1) FAIL(RAIRS_EINVAL, "d=%d: need d >= 1", t->d);
    if (t->d > RAIRS_MAX_WIDTH) FAIL(RAIRS_EUNSUPPORTED, "d=%d above the built limit %d", t->d, RAIRS_MAX_WIDTH);
    if (t->V < 1) FAIL(RAIRS_EINVAL, "a table needs at least one row");
    if (t->V > RAIRS_MAX_TABLE_ROWS) FAIL(RAIRS_EUNSUPPORTED, "V=%lld above the built limit %lld", (long long)t->V, (long long)RAIRS_MAX_TABLE_ROWS);
    if (!(t->scale >= 1e-30f && t->scale <= 1e30f)) FAIL(RAIRS_EINVAL, "scale must be within [1e-30, 1e30]");
    if (t->ld_live < 0 || (t->ld_live > 0 && t->ld_live < (t->V + 31) / 32))
        FAIL(RAIRS_EINVAL, "ld_live=%lld: need 0 or at least %lld words", (long long)t->ld_live, (long long)((t->V + 31) / 32));
    if (t->ld_live > 0 && !t->d_live) FAIL(RAIRS_EINVAL, "ld_live without a mask");
    if (n < 0) FAIL(RAIRS_EINVAL, "n is negative");
    if (n > RAIRS_MAX_ROWS) FAIL(RAIRS_EUNSUPPORTED, "n=%lld above the built limit %d", (long long)n, RAIRS_MAX_ROWS);
    return RAIRS_OK;
}

static LogprobArgs logprob_args(const rairs_table_t *t, const void *q, int64_t ldq, int q_dtype, int64_t n)
{
    LogprobArgs a = {};
    a.q = q; a.table = t->vectors;
    a.qtype = q_dtype; a.ttype = t->dtype;
    a.ldq = ldq; a.ldt = t->ld; a.n = n; a.V = t->V; a.d = t->d;
    a.scale = t->scale;
    a.live = t->d_live; a.ld_live = t->ld_live;
    return a;
}

static int check_top(int top)
{
    if (top < 0) FAIL(RAIRS_EINVAL, "top is negative");
    if (top > RAIRS_MAX_TOP) FAIL(RAIRS_EUNSUPPORTED, "top=%d above the built limit %d", top, RAIRS_MAX_TOP);
    return RAIRS_OK;
}

extern "C" size_t rairs_logprob_workspace_bytes(const rairs_table_t *t, int64_t n, int q_dtype, int top)
{
    if (check_table(t, n, q_dtype) || check_top(top) || n == 0) return 0;
    LogprobArgs a = logprob_args(t, nullptr, t->d, q_dtype, n);
    a.top = top;
    size_t bytes = 0;
    rairs_run_logprob(a, nullptr, &bytes, nullptr);
    return bytes;
}

extern "C" int rairs_logprob(const rairs_table_t *t, const void *d_q, int64_t ld_q, int q_dtype, int64_t n, const int64_t *d_targets,
                             float *d_logp, float *d_lse, float *d_entropy, int top, int64_t *d_top_ids, float *d_top_logp, void *d_ws,
                             size_t ws_bytes, void *hip_stream)
{
    TRY(check_table(t, n, q_dtype));
    TRY(check_top(top));
    if (n == 0) return RAIRS_OK;
    TRY(check_rows("vectors", t->vectors, t->ld, t->d, dtype_width(t->dtype)));
    TRY(check_rows("d_q", d_q, ld_q, t->d, dtype_width(q_dtype)));
    if (!d_targets || !d_logp || !d_lse) FAIL(RAIRS_EINVAL, "null device pointer");
    if (top > 0 && (!d_top_ids || !d_top_logp)) FAIL(RAIRS_EINVAL, "top without room for the rows");
    TRY(check_ws(d_ws, ws_bytes, rairs_logprob_workspace_bytes(t, n, q_dtype, top)));
    LogprobArgs a = logprob_args(t, d_q, ld_q, q_dtype, n);
    a.targets = d_targets; a.logp = d_logp; a.lse = d_lse; a.entropy = d_entropy;
    a.top = top; a.top_ids = d_top_ids; a.top_logp = d_top_logp;
    return rairs_run_logprob(a, d_ws, nullptr, (hipStream_t)hip_stream);
}

// (rows of the gradient of the logits, three pieces a value, are within 32-bit offsets of a tile's first)
static int check_grad_rows(int64_t n)
{
    if (n > RAIRS_MAX_GRAD_ROWS) FAIL(RAIRS_EUNSUPPORTED, "n=%lld above the built limit %d of the gradient", (long long)n, RAIRS_MAX_GRAD_ROWS);
    return RAIRS_OK;
}

extern "C" size_t rairs_logprob_backward_workspace_bytes(const rairs_table_t *t, int64_t n, int q_dtype, int table_grad)
{
    if (check_table(t, n, q_dtype) || check_grad_rows(n) || n == 0) return 0;
    LogprobArgs a = logprob_args(t, nullptr, t->d, q_dtype, n);
    a.dq = a.dtable = (void *)256;                                    // (wanted or not: not looked at)
    if (!table_grad) a.dtable = nullptr;
    size_t bytes = 0;
    rairs_run_logprob_backward(a, nullptr, &bytes, nullptr);
    return bytes;
}

extern "C" int rairs_logprob_backward(const rairs_table_t *t, const void *d_q, int64_t ld_q, int q_dtype, int64_t n,
                                      const int64_t *d_targets, const float *d_lse, const float *d_entropy, const float *d_dlogp,
                                      const float *d_dentropy, void *d_dq, int64_t ld_dq, void *d_dtable, int64_t ld_dtable, void *d_ws,
                                      size_t ws_bytes, void *hip_stream)
{
    TRY(check_table(t, n, q_dtype));
    TRY(check_grad_rows(n));
    if (d_dtable && t->dtype == RAIRS_U8) FAIL(RAIRS_EINVAL, "a table of bytes has no gradient");
    const int tw = dtype_width(t->dtype);
    if (d_dtable) TRY(check_rows("d_dtable", d_dtable, ld_dtable, t->d, tw));
    if (n == 0) {
        if (!d_dtable) return RAIRS_OK;
        return rairs_launch_clear_rows(d_dtable, t->V, t->d, ld_dtable, t->dtype, (hipStream_t)hip_stream);
    }
    TRY(check_rows("vectors", t->vectors, t->ld, t->d, tw));
    TRY(check_rows("d_q", d_q, ld_q, t->d, dtype_width(q_dtype)));
    if (d_dq) TRY(check_rows("d_dq", d_dq, ld_dq, t->d, dtype_width(q_dtype)));
    if (!d_targets || !d_lse || !d_dlogp) FAIL(RAIRS_EINVAL, "null device pointer");
    if (d_dentropy && !d_entropy) FAIL(RAIRS_EINVAL, "d_dentropy without d_entropy");
    TRY(check_ws(d_ws, ws_bytes, rairs_logprob_backward_workspace_bytes(t, n, q_dtype, d_dtable != nullptr)));
    if (!d_dq && !d_dtable) return RAIRS_OK;
    LogprobArgs a = logprob_args(t, d_q, ld_q, q_dtype, n);
    a.targets = d_targets; a.lse_in = d_lse; a.entropy_in = d_entropy; a.dlogp = d_dlogp; a.dentropy = d_dentropy;
    a.dq = d_dq; a.lddq = ld_dq; a.dtable = d_dtable; a.lddt = ld_dtable;
    return rairs_run_logprob_backward(a, d_ws, nullptr, (hipStream_t)hip_stream);
}
