// C ABI of the operators around the layers of a language model: argument checks and dispatch (include/netmax.h documents each call).
#include "block_norm.h"
#include "clip.h"
#include "embed.h"
#include "lm_checks.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

using namespace netmax;

// ---- embedding -------------------------------------------------------------------------------------------------------

static int check_embed(const netmax_embed_shape *s)
{
    if (!s) return netmax_fail(NETMAX_EINVAL, "shape is NULL");
    if (s->batch < 0 || s->batch > 65535 || s->tokens < 0 || s->tokens > 0x7FFFFFFF || s->vocab < 1 || s->vocab >= 1 << 22 || s->width < 1 || s->width >= 1 << 22)
        return netmax_fail(NETMAX_EINVAL, "need 0 <= batch <= 65535, 0 <= tokens < 2^31, 1 <= vocab < 2^22 and 1 <= width < 2^22");
    if (!product_fits(s->batch, s->tokens, s->width) || !product_fits(s->batch, s->vocab, s->width)) return netmax_fail(NETMAX_EINVAL, "the embedding is too large");
    if (!dtype_known(s->dtype)) return netmax_fail(NETMAX_EINVAL, "dtype must be NETMAX_F32 or NETMAX_BF16");
    return NETMAX_OK;
}

static EmbedArgs embed_args(const netmax_embed_shape *s, const int32_t *ids, void *table, void *y)
{
    return EmbedArgs{s->batch, s->tokens, s->vocab, s->width, s->dtype == NETMAX_BF16, s->accumulate != 0, s->scale, ids, table, y, s->s_ids, s->ldt, s->st, s->ldy, s->sy};
}

struct EmbedPlaces { Named ids, table, rows; };
static int check_embed_operands(const netmax_embed_shape *s, const int32_t *ids, const void *table, const char *table_name, bool table_written, const void *rows, const char *rows_name, EmbedPlaces &at)
{
    const bool any = s->tokens > 0;
    TRY(check_matrix("ids", ids, any, NETMAX_F32, s->batch, 1, s->tokens, s->tokens, s->s_ids));
    TRY(check_matrix(table_name, table, true, s->dtype, s->batch, s->vocab, s->width, s->ldt, s->st, table_written));
    TRY(check_matrix(rows_name, rows, any, s->dtype, s->batch, s->tokens, s->width, s->ldy, s->sy, !table_written));
    const int64_t es = size_of(s->dtype);
    at = EmbedPlaces{{"ids", Place(ids, 4, s->batch, 1, s->tokens, 0, s->s_ids)}, {table_name, Place(table, es, s->batch, s->vocab, s->width, s->ldt, s->st)},
                     {rows_name, Place(rows, es, s->batch, s->tokens, s->width, s->ldy, s->sy)}};
    return NETMAX_OK;
}

extern "C" int netmax_embed(const netmax_embed_shape *s, const int32_t *ids, const void *table, void *y, void *stream)
{
    TRY(check_embed(s));
    if (s->batch == 0 || s->tokens == 0) return NETMAX_OK;
    EmbedPlaces at;
    TRY(check_embed_operands(s, ids, table, "table", false, y, "y", at));
    TRY(check_apart(at.rows, {at.ids, at.table}));
    launch_embed((hipStream_t)stream, embed_args(s, ids, const_cast<void *>(table), y));
    return launched("embedding");
}

extern "C" int64_t netmax_embed_grad_workspace(const netmax_embed_shape *s)
{
    if (check_embed(s) != NETMAX_OK) return -1;
    return embed_grad_workspace(embed_args(s, nullptr, nullptr, nullptr));
}

extern "C" int netmax_embed_grad(const netmax_embed_shape *s, const int32_t *ids, const void *dy, void *dtable, void *work, int64_t work_bytes, void *stream)
{
    TRY(check_embed(s));
    if (s->batch == 0) return NETMAX_OK;
    EmbedPlaces at;
    TRY(check_embed_operands(s, ids, dtable, "dtable", true, dy, "dy", at));
    const EmbedArgs a = embed_args(s, ids, dtable, const_cast<void *>(dy));
    const int64_t need = embed_grad_workspace(a);
    TRY(check_work(work, work_bytes, need));
    TRY(check_apart(at.table, {at.ids, at.rows}));
    TRY(check_apart(workspace_at(work, need), {at.ids, at.table, at.rows}));
    launch_embed_grad((hipStream_t)stream, a, work);
    return launched("embedding gradient");
}

// ---- norms of a block ------------------------------------------------------------------------------------------------

static int check_block_norm(const netmax_block_norm_shape *s)
{
    if (!s) return netmax_fail(NETMAX_EINVAL, "shape is NULL");
    if (s->batch < 0 || s->batch > 65535 || s->rows < 0 || s->rows > 0x7FFFFFFF || s->width < 1 || s->width >= 1 << 22)
        return netmax_fail(NETMAX_EINVAL, "need 0 <= batch <= 65535, 0 <= rows < 2^31 and 1 <= width < 2^22");
    if (!product_fits(s->batch, s->rows, s->width) || !product_fits(s->batch, 1, s->width)) return netmax_fail(NETMAX_EINVAL, "the rows are too large");
    if (!dtype_known(s->dtype)) return netmax_fail(NETMAX_EINVAL, "dtype must be NETMAX_F32 or NETMAX_BF16");
    if (s->norm != NETMAX_NORM_RMS && s->norm != NETMAX_NORM_LAYER) return netmax_fail(NETMAX_EINVAL, "norm must be NETMAX_NORM_RMS or NETMAX_NORM_LAYER");
    if (s->gate_act < NETMAX_GATE_NONE || s->gate_act > NETMAX_GATE_TANH) return netmax_fail(NETMAX_EINVAL, "unknown gate_act");
    if (!(s->eps > 0.0f)) return netmax_fail(NETMAX_EINVAL, "eps must be positive");
    return NETMAX_OK;
}

static Span span(const netmax_span &s) { return Span{s.p, s.ld, s.s}; }

static NormArgs norm_args(const netmax_block_norm_shape *s, const netmax_block_norm_data *d, const netmax_block_norm_grads *g)
{
    NormArgs a{};
    a.batch = s->batch; a.rows = s->rows; a.width = s->width; a.bf16 = s->dtype == NETMAX_BF16; a.layer = s->norm == NETMAX_NORM_LAYER; a.act = s->gate_act;
    a.gate_rows = s->gate_rows != 0; a.post = s->post != 0; a.pre = s->pre != 0; a.x_scale = s->x_scale; a.f_scale = s->f_scale; a.eps = s->eps;
    a.share = 1.0 / (double)s->width;
    if (d) {
        a.x = span(d->x); a.f = span(d->f); a.gate = span(d->gate); a.post_gain = span(d->post_gain); a.post_bias = span(d->post_bias); a.pre_gain = span(d->pre_gain);
        a.pre_bias = span(d->pre_bias); a.h = span(d->h); a.y = span(d->y);
    }
    if (g) {
        a.dy = span(g->dy); a.dh = span(g->dh); a.dx = span(g->dx); a.df = span(g->df); a.dgate = span(g->dgate); a.dpost_gain = span(g->dpost_gain);
        a.dpost_bias = span(g->dpost_bias); a.dpre_gain = span(g->dpre_gain); a.dpre_bias = span(g->dpre_bias);
    }
    return a;
}

struct NormOperand { const char *name; const netmax_span *span; bool vector, needed, written; };

// Strides of all operands; nothing that is written shares memory with anything else, but for rows written in the place of rows that are read.
template <int N> static int check_spans(const netmax_block_norm_shape *s, const NormOperand (&all)[N], int64_t es, const Named &space)
{
    Named at[N];
    for (int k = 0; k < N; ++k) {
        const NormOperand &o = all[k];
        const int64_t rows = o.vector ? 1 : s->rows, ld = o.vector ? s->width : o.span->ld;
        TRY(check_matrix(o.name, o.span->p, o.needed, s->dtype, s->batch, rows, s->width, ld, o.span->s, o.written));
        at[k] = Named{o.name, Place(o.span->p, es, s->batch, rows, s->width, ld, o.span->s)};
    }
    for (int k = 0; k < N; ++k) {
        if (!all[k].written) continue;
        for (int i = 0; i < N; ++i) {
            if (i == k || (all[i].written && i < k)) continue;
            if (!all[k].vector && !all[i].vector && !all[i].written && at[k].at == at[i].at) continue;
            TRY(check_apart(at[k], at[i]));
        }
    }
    for (const Named &n : at) TRY(check_apart(space, n));
    return NETMAX_OK;
}

static int check_forms(const netmax_block_norm_shape *s, const netmax_block_norm_data *d)
{
    if (!d) return netmax_fail(NETMAX_EINVAL, "data is NULL");
    const bool any = s->batch > 0 && s->rows > 0;                   // no rows: f may be NULL for that
    if (any && !d->f.p && (d->gate.p || d->post_gain.p || d->post_bias.p)) return netmax_fail(NETMAX_EINVAL, "gate, post_gain or post_bias without f");
    if (!s->post && (d->post_gain.p || d->post_bias.p)) return netmax_fail(NETMAX_EINVAL, "post_gain or post_bias without a norm of f");
    if (!s->pre && (d->pre_gain.p || d->pre_bias.p)) return netmax_fail(NETMAX_EINVAL, "pre_gain or pre_bias without a norm of h");
    return NETMAX_OK;
}

extern "C" int netmax_block_norm(const netmax_block_norm_shape *s, const netmax_block_norm_data *d, void *stream)
{
    TRY(check_block_norm(s));
    TRY(check_forms(s, d));
    if (!s->pre && d->y.p) return netmax_fail(NETMAX_EINVAL, "y without a norm of h");
    if (s->batch == 0 || s->rows == 0) return NETMAX_OK;
    if (!d->h.p && !d->y.p) return netmax_fail(NETMAX_EINVAL, "h and y are NULL");
    const NormOperand all[] = {{"x", &d->x, false, true, false}, {"f", &d->f, false, false, false}, {"gate", &d->gate, !s->gate_rows, false, false}, {"post_gain", &d->post_gain, true, false, false},
                            {"post_bias", &d->post_bias, true, false, false}, {"pre_gain", &d->pre_gain, true, false, false}, {"pre_bias", &d->pre_bias, true, false, false},
                            {"h", &d->h, false, false, true}, {"y", &d->y, false, false, true}};
    TRY(check_spans(s, all, size_of(s->dtype), workspace_at(nullptr, 0)));
    launch_block_norm((hipStream_t)stream, norm_args(s, d, nullptr));
    return launched("block norm");
}

extern "C" int64_t netmax_block_norm_grad_workspace(const netmax_block_norm_shape *s, const netmax_block_norm_data *d, const netmax_block_norm_grads *g)
{
    if (check_block_norm(s) != NETMAX_OK) return -1;
    if (!d || !g) {
        netmax_fail(NETMAX_EINVAL, "data or grads is NULL");
        return -1;
    }
    return block_norm_grad_workspace(norm_args(s, d, g));
}

extern "C" int netmax_block_norm_grad(const netmax_block_norm_shape *s, const netmax_block_norm_data *d, const netmax_block_norm_grads *g, void *work, int64_t work_bytes, void *stream)
{
    TRY(check_block_norm(s));
    TRY(check_forms(s, d));
    if (!g) return netmax_fail(NETMAX_EINVAL, "grads is NULL");
    if (s->rows > 0 && !d->f.p && (g->df.p || g->dgate.p || g->dpost_gain.p || g->dpost_bias.p)) return netmax_fail(NETMAX_EINVAL, "df, dgate, dpost_gain or dpost_bias without f");
    if (!d->gate.p && g->dgate.p) return netmax_fail(NETMAX_EINVAL, "dgate without a gate");
    if (!s->post && (g->dpost_gain.p || g->dpost_bias.p)) return netmax_fail(NETMAX_EINVAL, "dpost_gain or dpost_bias without a norm of f");
    if (!s->pre && (g->dy.p || g->dpre_gain.p || g->dpre_bias.p)) return netmax_fail(NETMAX_EINVAL, "dy, dpre_gain or dpre_bias without a norm of h");
    if (s->batch == 0) return NETMAX_OK;
    const bool any = s->rows > 0;
    const NormOperand all[] = {{"dy", &g->dy, false, any && s->pre, false}, {"dh", &g->dh, false, any && !s->pre, false}, {"x", &d->x, false, any, false}, {"f", &d->f, false, false, false},
                            {"gate", &d->gate, !s->gate_rows, false, false}, {"post_gain", &d->post_gain, true, false, false}, {"post_bias", &d->post_bias, true, false, false},
                            {"pre_gain", &d->pre_gain, true, false, false}, {"pre_bias", &d->pre_bias, true, false, false}, {"dx", &g->dx, false, false, true}, {"df", &g->df, false, false, true},
                            {"dgate", &g->dgate, !s->gate_rows, false, true}, {"dpost_gain", &g->dpost_gain, true, false, true}, {"dpost_bias", &g->dpost_bias, true, false, true},
                            {"dpre_gain", &g->dpre_gain, true, false, true}, {"dpre_bias", &g->dpre_bias, true, false, true}};
    const NormArgs a = norm_args(s, d, g);
    const int64_t need = block_norm_grad_workspace(a);
    TRY(check_work(work, work_bytes, need));
    TRY(check_spans(s, all, size_of(s->dtype), workspace_at(work, need)));
    launch_block_norm_grad((hipStream_t)stream, a, work);
    return launched("block norm gradient");
}

// ---- clipping --------------------------------------------------------------------------------------------------------

static int check_gradients(int64_t batch, int64_t n, const netmax_gradient *g)
{
    if (batch < 0 || batch > 65535 || n < 0 || n > 65535) return netmax_fail(NETMAX_EINVAL, "need 0 <= batch <= 65535 and 0 <= n <= 65535");
    if (n > 0 && !g) return netmax_fail(NETMAX_EINVAL, "gradients is NULL");
    for (int64_t k = 0; k < n; ++k) {
        if (!dtype_known(g[k].dtype)) return netmax_fail(NETMAX_EINVAL, "dtype must be NETMAX_F32 or NETMAX_BF16");
        // pieces of 16 bytes, too: a launch counts its units of them in 32 bits
        if (!product_fits(batch, g[k].rows, g[k].cols) || (double)g[k].rows * (double)((g[k].cols + 3) / 4) > 68719476736.0)
            return netmax_fail(NETMAX_EINVAL, "a gradient is too large, or its size is negative");
    }
    return NETMAX_OK;
}

struct GradientPlace { Place at; int64_t tensor; bool written; };

static int shared(const GradientPlace &a, const GradientPlace &b)
{
    char buf[160];
    const char *const names[] = {"g", "out"};
    snprintf(buf, sizeof buf, "%s %lld and %s %lld share memory", names[a.written], (long long)a.tensor, names[b.written], (long long)b.tensor);
    return netmax_fail(NETMAX_EINVAL, buf);
}

// Whether operands of batches that lie equally far apart, each no longer than that, are apart on the circle of one such distance: then they are apart.
static bool apart_on_circle(const GradientPlace *first, const GradientPlace *end, std::vector<std::pair<int64_t, int64_t>> &arcs)
{
    const int64_t step = first->at.step;
    arcs.clear();
    for (const GradientPlace *p = first; p != end; ++p) {
        if (p->at.step != step || step == 0 || p->at.span() > step) return false;
        arcs.emplace_back(p->at.lo % step, p->at.span());
    }
    std::sort(arcs.begin(), arcs.end());
    for (size_t k = 1; k < arcs.size(); ++k)
        if (arcs[k - 1].first + arcs[k - 1].second > arcs[k].first) return false;
    return arcs.back().first + arcs.back().second <= arcs.front().first + step;
}

// Results apart from one another and from everything that is read, but for their own gradients.  Sorted by where they begin, operands are compared with those whose hulls they meet.
static int check_gradients_apart(int64_t batch, int64_t n, const netmax_gradient *g, const Named &norm, const Named &space)
{
    std::vector<GradientPlace> all;
    all.reserve(2 * n);
    for (int64_t k = 0; k < n; ++k) {
        const netmax_gradient &t = g[k];
        const int64_t es = size_of(t.dtype);
        const Place from(t.g, es, batch, t.rows, t.cols, t.ldg, t.sg), to(t.out, es, batch, t.rows, t.cols, t.ldo, t.so);
        if (to.lo == to.hi) continue;
        all.push_back(GradientPlace{to, k, true});
        if (!(from == to)) all.push_back(GradientPlace{from, k, false});
    }
    std::sort(all.begin(), all.end(), [](const GradientPlace &a, const GradientPlace &b) { return a.at.lo < b.at.lo; });
    std::vector<std::pair<int64_t, int64_t>> arcs;
    for (size_t first = 0; first < all.size();) {
        int64_t hi = all[first].at.hi;
        size_t end = first + 1;
        while (end < all.size() && all[end].at.lo < hi) hi = std::max(hi, all[end++].at.hi);
        if (end - first > 2 && apart_on_circle(&all[first], &all[first] + (end - first), arcs)) { first = end; continue; }
        for (size_t i = first; i < end; ++i)
            for (size_t k = i + 1; k < end && all[k].at.lo < all[i].at.hi; ++k)
                if ((all[i].written || all[k].written) && share_memory(all[i].at, all[k].at)) return shared(all[i], all[k]);
        first = end;
    }
    for (const GradientPlace &p : all) {
        const Named here{p.written ? "out" : "g", p.at};
        TRY(check_apart(norm, here));
        TRY(check_apart(space, here));
    }
    return check_apart(space, norm);
}

extern "C" int64_t netmax_grad_norm_workspace(int64_t batch, int64_t n, const netmax_gradient *g)
{
    if (check_gradients(batch, n, g) != NETMAX_OK) return -1;
    return batch == 0 ? 0 : clip_workspace(batch, n, g);
}

static int check_places(int64_t batch, int64_t n, const netmax_gradient *g, bool scale)
{
    for (int64_t k = 0; k < n; ++k) {
        const netmax_gradient &t = g[k];
        const bool any = t.rows > 0 && t.cols > 0;
        TRY(check_matrix("g", t.g, any, t.dtype, batch, t.rows, t.cols, t.ldg, t.sg));
        if (scale) TRY(check_matrix("out", t.out, any, t.dtype, batch, t.rows, t.cols, t.ldo, t.so, any));
    }
    return NETMAX_OK;
}

extern "C" int netmax_grad_norm(int64_t batch, int64_t n, const netmax_gradient *g, float *norm, void *work, int64_t work_bytes, void *stream)
{
    TRY(check_gradients(batch, n, g));
    if (batch == 0) return NETMAX_OK;
    TRY(check_places(batch, n, g, false));
    TRY(check_matrix("norm", norm, true, NETMAX_F32, 1, 1, batch, batch, 0));
    const int64_t need = clip_workspace(batch, n, g);
    TRY(check_work(work, work_bytes, need));
    const Named out{"norm", Place(norm, 4, 1, 1, batch, 0, 0)}, space = workspace_at(work, need);
    for (int64_t k = 0; k < n; ++k) {
        const Named in{"g", Place(g[k].g, size_of(g[k].dtype), batch, g[k].rows, g[k].cols, g[k].ldg, g[k].sg)};
        TRY(check_apart(out, in));
        TRY(check_apart(space, in));
    }
    TRY(check_apart(space, out));
    launch_clip((hipStream_t)stream, ClipArgs{batch, n, g, false, INFINITY, norm}, work);
    return launched("gradient norm");
}

extern "C" int netmax_clip_grads(int64_t batch, int64_t n, const netmax_gradient *g, float max_norm, float *norm, void *work, int64_t work_bytes, void *stream)
{
    TRY(check_gradients(batch, n, g));
    if (!(max_norm > 0.0f)) return netmax_fail(NETMAX_EINVAL, "max_norm must be positive");
    if (batch == 0) return NETMAX_OK;
    TRY(check_places(batch, n, g, true));
    TRY(check_matrix("norm", norm, false, NETMAX_F32, 1, 1, batch, batch, 0));
    const int64_t need = clip_workspace(batch, n, g);
    TRY(check_work(work, work_bytes, need));
    try {
        TRY(check_gradients_apart(batch, n, g, Named{"norm", Place(norm, 4, 1, 1, batch, 0, 0)}, workspace_at(work, need)));
    } catch (const std::bad_alloc &) {
        return netmax_fail(NETMAX_ENOMEM, "no host memory to compare where the gradients lie");
    }
    launch_clip((hipStream_t)stream, ClipArgs{batch, n, g, true, max_norm, norm}, work);
    return launched("clipping");
}
