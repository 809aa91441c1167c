// C ABI of the operators for language models: argument checks and dispatch (include/netmax.h documents each call).
#include "errors.h"
#include "linear.h"
#include "orth.h"
#include "places.h"
#include "token_loss.h"

#include <cstdio>

using namespace netmax;

static int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return NETMAX_OK;
    char buf[200];
    snprintf(buf, sizeof buf, "%s: %s", what, hipGetErrorString(e));
    return netmax_fail(NETMAX_EDEVICE, buf);
}

static bool dtype_known(int32_t d) { return d == NETMAX_F32 || d == NETMAX_BF16; }
static int64_t size_of(int32_t dtype) { return dtype == NETMAX_BF16 ? 2 : 4; }
static bool aligned(const void *p, int32_t dtype) { return (uintptr_t)p % size_of(dtype) == 0; }

// Sizes that keep every product of them, in bytes, far inside 64 bits.
constexpr int64_t MOST = (int64_t)1 << 40;
static bool product_fits(int64_t a, int64_t b, int64_t c)
{
    return a >= 0 && b >= 0 && c >= 0 && (double)a * (double)b * (double)c <= (double)MOST && a <= MOST && b <= MOST && c <= MOST;
}
// Blocks of 64 x 64 results of a whole batch: one launch's workgroups of 256 threads, and a launch has fewer than 2^32 of them.
static bool blocks_fit(int64_t batch, int64_t m, int64_t n) { return (double)batch * (double)((m + 63) / 64) * (double)((n + 63) / 64) < 16777216.0; }

static bool strides_ok(int64_t batch, int64_t rows, int64_t cols, int64_t ld, int64_t step)
{
    return (rows <= 1 || ld >= cols) && ld >= 0 && ld <= MOST && step >= 0 && step <= MOST && (rows == 0 || product_fits(rows, ld, 1)) && product_fits(batch, step, 1);
}

static int check_linear(const netmax_linear_shape *s)
{
    if (!s) return netmax_fail(NETMAX_EINVAL, "shape is NULL");
    if (s->batch < 0 || s->batch > 65535 || s->rows < 0 || s->d_in < 1 || s->d_out < 1 || s->d_in >= 1 << 22 || s->d_out >= 1 << 22)
        return netmax_fail(NETMAX_EINVAL, "need 0 <= batch <= 65535, rows >= 0, 1 <= d_in < 2^22 and 1 <= d_out < 2^22");
    if (!product_fits(s->batch, s->rows, s->d_in) || !product_fits(s->batch, s->rows, s->d_out) || !product_fits(s->batch, s->d_in, s->d_out) ||
        !blocks_fit(s->batch, s->rows, s->d_in) || !blocks_fit(s->batch, s->rows, s->d_out) || !blocks_fit(s->batch, s->d_in, s->d_out) || s->rows > (int64_t)65535 * 64)
        return netmax_fail(NETMAX_EINVAL, "the layer is too large");
    if (!dtype_known(s->dtype)) return netmax_fail(NETMAX_EINVAL, "dtype must be NETMAX_F32 or NETMAX_BF16");
    if (s->act < NETMAX_ACT_NONE || s->act > NETMAX_ACT_SILU) return netmax_fail(NETMAX_EINVAL, "unknown activation");
    return NETMAX_OK;
}

// `written`: results of a batch need memory of their own each.
static int check_matrix(const char *name, const void *p, bool needed, int32_t dtype, int64_t batch, int64_t rows, int64_t cols, int64_t ld, int64_t step, bool written = false)
{
    char buf[160];
    if (!p) {
        if (!needed) return NETMAX_OK;
        snprintf(buf, sizeof buf, "%s is NULL", name);
        return netmax_fail(NETMAX_EINVAL, buf);
    }
    if (aligned(p, dtype) && strides_ok(batch, rows, cols, ld, step) &&
        !(written && batch > 1 && (step == 0 || batch_overlaps(Place(p, size_of(dtype), batch, rows, cols, ld, step))))) return NETMAX_OK;
    snprintf(buf, sizeof buf, "%s: misaligned, or rows closer together than they are long, or a negative stride, or results in the same place", name);
    return netmax_fail(NETMAX_EINVAL, buf);
}

#define TRY(call) do { const int rc_ = (call); if (rc_ != NETMAX_OK) return rc_; } while (0)

static LinearArgs linear_args(const netmax_linear_shape *s)
{
    LinearArgs a{};
    a.batch = s->batch; a.rows = s->rows; a.din = s->d_in; a.dout = s->d_out; a.bf16 = s->dtype == NETMAX_BF16; a.act = s->act;
    a.ldx = s->ldx; a.ldw = s->ldw; a.ldr = s->ldr; a.ldy = s->ldy; a.ldz = s->ldz;
    a.sx = s->sx; a.sw = s->sw; a.sb = s->sb; a.sr = s->sr; a.sy = s->sy; a.sz = s->sz;
    return a;
}

static int check_work(const void *work, int64_t have, int64_t need)
{
    if (need == 0 || (work && have >= need && (uintptr_t)work % 256 == 0)) return NETMAX_OK;
    char buf[160];
    snprintf(buf, sizeof buf, "the workspace must be 256-byte aligned and hold %lld bytes (%lld given)", (long long)need, (long long)have);
    return netmax_fail(NETMAX_EINVAL, buf);
}

// ---- memory that a call writes: nothing that it still reads, and nothing twice ---------------------------------------

struct Named { const char *name; Place at; };

static int check_apart(const Named &a, const Named &b)
{
    if (!share_memory(a.at, b.at)) return NETMAX_OK;
    char buf[160];
    snprintf(buf, sizeof buf, "%s and %s share memory", a.name, b.name);
    return netmax_fail(NETMAX_EINVAL, buf);
}
template <int N> static int check_apart(const Named &a, const Named (&others)[N])
{
    for (const Named &o : others) TRY(check_apart(a, o));
    return NETMAX_OK;
}
// The workspace, if the call needs one, lies apart from everything else.
static Named workspace_at(const void *work, int64_t bytes) { return Named{"the workspace", Place(bytes ? work : nullptr, 1, 1, 1, bytes, 0, 0)}; }

extern "C" int64_t netmax_linear_workspace(const netmax_linear_shape *s, const void *x, const void *w)
{
    if (check_linear(s) != NETMAX_OK) return -1;
    LinearArgs a = linear_args(s);
    a.x = x; a.w = w;
    return linear_workspace(a);
}

extern "C" int netmax_linear(const netmax_linear_shape *s, const void *x, const void *w, const void *bias, const void *residual, void *y, void *z,
                             void *work, int64_t work_bytes, void *stream)
{
    TRY(check_linear(s));
    if (s->batch == 0 || s->rows == 0) return NETMAX_OK;
    const int32_t d = s->dtype;
    TRY(check_matrix("x", x, true, d, s->batch, s->rows, s->d_in, s->ldx, s->sx));
    TRY(check_matrix("w", w, true, d, s->batch, s->d_in, s->d_out, s->ldw, s->sw));
    TRY(check_matrix("bias", bias, false, d, s->batch, 1, s->d_out, s->d_out, s->sb));
    TRY(check_matrix("residual", residual, false, d, s->batch, s->rows, s->d_out, s->ldr, s->sr));
    TRY(check_matrix("y", y, true, d, s->batch, s->rows, s->d_out, s->ldy, s->sy, true));
    TRY(check_matrix("z", z, false, d, s->batch, s->rows, s->d_out, s->ldz, s->sz, true));
    LinearArgs a = linear_args(s);
    a.x = x; a.w = w; a.bias = bias; a.residual = residual; a.y = y; a.z = z;
    const int64_t need = linear_workspace(a), es = size_of(d);
    TRY(check_work(work, work_bytes, need));
    const Named in_x{"x", Place(x, es, s->batch, s->rows, s->d_in, s->ldx, s->sx)}, in_w{"w", Place(w, es, s->batch, s->d_in, s->d_out, s->ldw, s->sw)},
        in_b{"bias", Place(bias, es, s->batch, 1, s->d_out, 0, s->sb)}, in_r{"residual", Place(residual, es, s->batch, s->rows, s->d_out, s->ldr, s->sr)},
        out_y{"y", Place(y, es, s->batch, s->rows, s->d_out, s->ldy, s->sy)}, out_z{"z", Place(z, es, s->batch, s->rows, s->d_out, s->ldz, s->sz)};
    TRY(check_apart(out_y, {in_x, in_w, in_b, out_z}));
    if (!(out_y.at == in_r.at)) TRY(check_apart(out_y, in_r));       // value by value in place
    TRY(check_apart(out_z, {in_x, in_w, in_b, in_r}));
    TRY(check_apart(workspace_at(work, need), {in_x, in_w, in_b, in_r, out_y, out_z}));
    launch_linear((hipStream_t)stream, a, work);
    return launched("linear");
}

static LinearGradArgs linear_grad_args(const netmax_linear_shape *s)
{
    LinearGradArgs a{};
    a.batch = s->batch; a.rows = s->rows; a.din = s->d_in; a.dout = s->d_out; a.bf16 = s->dtype == NETMAX_BF16; a.act = s->act;
    a.lddy = s->ldy; a.ldx = s->ldx; a.ldw = s->ldw; a.ldz = s->ldz; a.lddx = s->lddx; a.lddw = s->lddw;
    a.sdy = s->sy; a.sx = s->sx; a.sw = s->sw; a.sz = s->sz; a.sdx = s->sdx; a.sdw = s->sdw; a.sdb = s->sdb;
    return a;
}

extern "C" int64_t netmax_linear_grad_workspace(const netmax_linear_shape *s, const void *dy, const void *x, const void *w)
{
    if (check_linear(s) != NETMAX_OK) return -1;
    LinearGradArgs a = linear_grad_args(s);
    a.dy = dy; a.x = x; a.w = w;
    return linear_grad_workspace(a);
}

extern "C" int netmax_linear_grad(const netmax_linear_shape *s, const void *dy, const void *x, const void *w, const void *z, void *dx, void *dw, void *db,
                                  void *work, int64_t work_bytes, void *stream)
{
    TRY(check_linear(s));
    if (s->batch == 0) return NETMAX_OK;
    const int32_t d = s->dtype;
    const bool any = s->rows > 0;
    TRY(check_matrix("dy", dy, any, d, s->batch, s->rows, s->d_out, s->ldy, s->sy));
    TRY(check_matrix("x", x, any && dw, d, s->batch, s->rows, s->d_in, s->ldx, s->sx));
    TRY(check_matrix("w", w, any && dx, d, s->batch, s->d_in, s->d_out, s->ldw, s->sw));
    TRY(check_matrix("z", z, any && s->act != NETMAX_ACT_NONE, d, s->batch, s->rows, s->d_out, s->ldz, s->sz));
    TRY(check_matrix("dx", dx, false, d, s->batch, s->rows, s->d_in, s->lddx, s->sdx, true));
    TRY(check_matrix("dw", dw, false, d, s->batch, s->d_in, s->d_out, s->lddw, s->sdw, true));
    TRY(check_matrix("db", db, false, d, s->batch, 1, s->d_out, s->d_out, s->sdb, true));
    LinearGradArgs a = linear_grad_args(s);
    a.dy = dy; a.x = x; a.w = w; a.z = z; a.dx = dx; a.dw = dw; a.db = db;
    const int64_t need = linear_grad_workspace(a), es = size_of(d);
    TRY(check_work(work, work_bytes, need));
    const auto place = [&](const char *name, const void *p, int64_t rows, int64_t cols, int64_t ld, int64_t step) { return Named{name, Place(p, es, s->batch, rows, cols, ld, step)}; };
    // what the products read while results are written; with an activation dy and z are read before anything is
    const bool late = s->act == NETMAX_ACT_NONE && (dx || dw);
    const Named in_dy = place("dy", dy, s->rows, s->d_out, s->ldy, s->sy), in_z = place("z", s->act == NETMAX_ACT_NONE ? nullptr : z, s->rows, s->d_out, s->ldz, s->sz),
        in_x = place("x", dw ? x : nullptr, s->rows, s->d_in, s->ldx, s->sx), in_w = place("w", dx ? w : nullptr, s->d_in, s->d_out, s->ldw, s->sw),
        out_x = place("dx", dx, s->rows, s->d_in, s->lddx, s->sdx), out_w = place("dw", dw, s->d_in, s->d_out, s->lddw, s->sdw), out_b = place("db", db, 1, s->d_out, 0, s->sdb);
    for (const Named *o : {&out_x, &out_w, &out_b}) {
        if (late) TRY(check_apart(*o, in_dy));
        TRY(check_apart(*o, {in_x, in_w}));
    }
    TRY(check_apart(out_x, {out_w, out_b}));
    TRY(check_apart(out_w, out_b));
    TRY(check_apart(workspace_at(work, need), {in_dy, in_z, in_x, in_w, out_x, out_w, out_b}));
    launch_linear_grad((hipStream_t)stream, a, work);
    return launched("linear gradient");
}

// ---- orthogonalised updates ------------------------------------------------------------------------------------------

static int check_orth(const netmax_orth_shape *s)
{
    if (!s) return netmax_fail(NETMAX_EINVAL, "shape is NULL");
    if (s->batch < 0 || s->batch > 65535 || s->rows < 1 || s->cols < 1 || s->rows >= 1 << 22 || s->cols >= 1 << 22)
        return netmax_fail(NETMAX_EINVAL, "need 0 <= batch <= 65535, 1 <= rows < 2^22 and 1 <= cols < 2^22");
    if (!product_fits(s->batch, s->rows, s->cols) || !blocks_fit(s->batch, s->rows, s->cols)) return netmax_fail(NETMAX_EINVAL, "the matrices are too large");
    if (!dtype_known(s->dtype)) return netmax_fail(NETMAX_EINVAL, "dtype must be NETMAX_F32 or NETMAX_BF16");
    if (s->steps < 1 || s->steps > 64) return netmax_fail(NETMAX_EINVAL, "steps must be in 1..64");
    if (!(s->eps > 0.0f)) return netmax_fail(NETMAX_EINVAL, "eps must be positive");
    return NETMAX_OK;
}

static OrthArgs orth_args(const netmax_orth_shape *s)
{
    OrthArgs a{};
    a.batch = s->batch; a.rows = s->rows; a.cols = s->cols; a.bf16 = s->dtype == NETMAX_BF16; a.steps = s->steps; a.nesterov = s->nesterov;
    a.mu = s->mu; a.a = s->a; a.b = s->b; a.c = s->c; a.eps = s->eps; a.scale = s->scale;
    a.ldg = s->ldg; a.sg = s->sg; a.ldm = s->ldm; a.sm = s->sm; a.ldo = s->ldo; a.so = s->so;
    return a;
}

extern "C" int64_t netmax_orthogonalize_workspace(const netmax_orth_shape *s)
{
    if (check_orth(s) != NETMAX_OK) return -1;
    return orth_workspace(orth_args(s));
}

extern "C" int netmax_orthogonalize(const netmax_orth_shape *s, const void *g, const float *m, float *m_out, void *out, void *work, int64_t work_bytes, void *stream)
{
    TRY(check_orth(s));
    if (s->batch == 0) return NETMAX_OK;
    TRY(check_matrix("g", g, true, s->dtype, s->batch, s->rows, s->cols, s->ldg, s->sg));
    TRY(check_matrix("m", m, m_out != nullptr, NETMAX_F32, s->batch, s->rows, s->cols, s->ldm, s->sm));
    TRY(check_matrix("m_out", m_out, m != nullptr, NETMAX_F32, s->batch, s->rows, s->cols, s->ldm, s->sm, true));
    TRY(check_matrix("out", out, true, s->dtype, s->batch, s->rows, s->cols, s->ldo, s->so, true));
    OrthArgs a = orth_args(s);
    a.g = g; a.m = m; a.m_out = m_out; a.out = out;
    const int64_t need = orth_workspace(a), es = size_of(s->dtype);
    TRY(check_work(work, work_bytes, need));
    // out is written when g and m have been read, m_out while they are
    const Named in_g{"g", Place(g, es, s->batch, s->rows, s->cols, s->ldg, s->sg)}, in_m{"m", Place(m, 4, s->batch, s->rows, s->cols, s->ldm, s->sm)},
        out_m{"m_out", Place(m_out, 4, s->batch, s->rows, s->cols, s->ldm, s->sm)}, out_u{"out", Place(out, es, s->batch, s->rows, s->cols, s->ldo, s->so)};
    TRY(check_apart(out_m, {in_g, out_u}));
    if (!(out_m.at == in_m.at)) TRY(check_apart(out_m, in_m));       // value by value in place
    TRY(check_apart(workspace_at(work, need), {in_g, in_m, out_m, out_u}));
    launch_orth((hipStream_t)stream, a, work);
    return launched("orthogonalize");
}

// ---- losses on sampled tokens ----------------------------------------------------------------------------------------

static int check_rows(int64_t tokens, int64_t vocab, int32_t dtype, const void *logits, int64_t ld, const int32_t *labels, const void *grad, int64_t ldg)
{
    if (tokens < 0 || tokens > 0x7FFFFFFF || vocab < 1 || vocab > 0x7FFFFFFF) return netmax_fail(NETMAX_EINVAL, "need 0 <= tokens < 2^31 and 1 <= vocab < 2^31");
    if (!dtype_known(dtype)) return netmax_fail(NETMAX_EINVAL, "dtype must be NETMAX_F32 or NETMAX_BF16");
    TRY(check_matrix("logits", logits, tokens > 0, dtype, 1, tokens, vocab, ld, 0));
    TRY(check_matrix("grad", grad, false, dtype, 1, tokens, vocab, ldg, 0));
    if (grad == logits && grad && ldg != ld) return netmax_fail(NETMAX_EINVAL, "a gradient in the logits' place needs the logits' distance of rows");
    if (tokens > 0 && !labels) return netmax_fail(NETMAX_EINVAL, "labels is NULL");
    return NETMAX_OK;
}

extern "C" int netmax_policy_loss(int64_t tokens, int64_t vocab, int32_t dtype, const void *logits, int64_t ld, const int32_t *labels, const float *old_logp,
                                  const float *ref_logp, const float *advantage, const float *weight, float clip_low, float clip_high, float kl, float *loss,
                                  float *logp, void *grad, int64_t ldg, void *stream)
{
    TRY(check_rows(tokens, vocab, dtype, logits, ld, labels, grad, ldg));
    if (!(clip_low >= 0.0f && clip_low <= 1.0f) || !(clip_high >= 0.0f)) return netmax_fail(NETMAX_EINVAL, "need 0 <= clip_low <= 1 and clip_high >= 0");
    if (tokens == 0) return NETMAX_OK;
    if (!old_logp || !advantage || !loss) return netmax_fail(NETMAX_EINVAL, "old_logp, advantage or loss is NULL");
    if (kl != 0.0f && !ref_logp) return netmax_fail(NETMAX_EINVAL, "a KL term needs ref_logp");
    const auto each = [&](const char *name, const void *p) { return Named{name, Place(p, 4, 1, 1, tokens, 0, 0)}; };
    const Named in_z{"logits", Place(logits, size_of(dtype), 1, tokens, vocab, ld, 0)}, out_g{"grad", Place(grad, size_of(dtype), 1, tokens, vocab, ldg, 0)},
        out_l = each("loss", loss), out_p = each("logp", logp);
    const Named in[] = {each("labels", labels), each("old_logp", old_logp), each("ref_logp", ref_logp), each("advantage", advantage), each("weight", weight)};
    for (const Named *o : {&out_l, &out_p, &out_g}) TRY(check_apart(*o, in));
    TRY(check_apart(out_l, {in_z, out_p, out_g}));
    TRY(check_apart(out_p, {in_z, out_g}));
    if (!(out_g.at == in_z.at)) TRY(check_apart(out_g, in_z));       // row by row in place
    const TokenRows rows{tokens, vocab, ld, logits, labels, weight, dtype == NETMAX_BF16};
    launch_policy_loss((hipStream_t)stream, rows, PolicyArgs{old_logp, ref_logp, advantage, clip_low, clip_high, kl, loss, logp, grad, ldg});
    return launched("policy loss");
}

static int64_t up(int64_t n) { return (n + 255) / 256 * 256; }

extern "C" int64_t netmax_preference_workspace(int64_t tokens, int64_t pairs)
{
    if (tokens < 0 || tokens > 0x7FFFFFFF || pairs < 1 || pairs > 0x3FFFFFFF) return -1;
    return up(8 * tokens) * 2 + up(8 * pairs);
}

extern "C" int netmax_preference_loss(int64_t tokens, int64_t vocab, int32_t dtype, const void *logits, int64_t ld, const int32_t *labels, int64_t pairs,
                                      const int32_t *offsets, const float *ref_logp, const float *weight, float beta, float smoothing, float scale, float *loss,
                                      float *ratio, void *grad, int64_t ldg, void *work, int64_t work_bytes, void *stream)
{
    TRY(check_rows(tokens, vocab, dtype, logits, ld, labels, grad, ldg));
    if (pairs < 1 || pairs > 0x3FFFFFFF) return netmax_fail(NETMAX_EINVAL, "need 1 <= pairs < 2^30");
    if (!(smoothing >= 0.0f && smoothing <= 1.0f)) return netmax_fail(NETMAX_EINVAL, "need 0 <= smoothing <= 1");
    if (!offsets || !loss || !ratio || (tokens > 0 && !ref_logp)) return netmax_fail(NETMAX_EINVAL, "offsets, ref_logp, loss or ratio is NULL");
    const int64_t need = netmax_preference_workspace(tokens, pairs);
    TRY(check_work(work, work_bytes, need));
    const auto each = [&](const char *name, const void *p, int64_t n) { return Named{name, Place(p, 4, 1, 1, n, 0, 0)}; };
    const Named in_z{"logits", Place(logits, size_of(dtype), 1, tokens, vocab, ld, 0)}, out_g{"grad", Place(grad, size_of(dtype), 1, tokens, vocab, ldg, 0)},
        out_l = each("loss", loss, pairs), out_r = each("ratio", ratio, 2 * pairs);
    const Named in[] = {each("labels", labels, tokens), each("offsets", offsets, 2 * pairs + 1), each("weight", weight, tokens), each("ref_logp", ref_logp, tokens)};
    for (const Named *o : {&out_l, &out_r, &out_g}) TRY(check_apart(*o, in));
    TRY(check_apart(out_l, {in_z, out_r, out_g}));
    TRY(check_apart(out_r, {in_z, out_g}));
    if (!(out_g.at == in_z.at)) TRY(check_apart(out_g, in_z));       // row by row in place
    const Named space = workspace_at(work, need);
    TRY(check_apart(space, in));
    TRY(check_apart(space, {in_z, out_l, out_r, out_g}));
    char *w = (char *)work;
    const TokenRows rows{tokens, vocab, ld, logits, labels, weight, dtype == NETMAX_BF16};
    launch_preference_loss((hipStream_t)stream, rows,
                           PreferenceArgs{pairs, offsets, ref_logp, beta, smoothing, scale, loss, ratio, grad, ldg, (float2 *)w,
                                          (double *)(w + up(8 * tokens)), (float *)(w + 2 * up(8 * tokens))});
    return launched("preference loss");
}
