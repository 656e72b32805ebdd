// rows_api.hip -- host side of the C ABI declared in include/umap_rows.h: every
// argument is checked here, before any HIP call, so that a launch never reads or
// writes outside the arrays it was given.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include <initializer_list>

#include "internal.hpp"
#include "rows_internal.hpp"

namespace {

__attribute__((format(printf, 2, 3))) int fail(int code, const char *fmt, ...)
{
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    try {
        return ul::set_error(code, buf);
    } catch (...) {   // no memory for the message: the code alone
        return code;
    }
}

int launched(hipError_t e, const char *what)
{
    if (e == hipSuccess) return UMAP_OK;
    (void)hipGetLastError();   // reported here, and not by the next launch's check again
    return fail(UMAP_E_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

int elem_bytes(int32_t type)
{
    switch (type) {
    case UMAP_F32: return 4;
    case UMAP_F16:
    case UMAP_BF16: return 2;
    case UMAP_I8:
    case UMAP_F8: return 1;
    }
    return 0;
}
bool is_float(int32_t type) { return type == UMAP_F32 || type == UMAP_F16 || type == UMAP_BF16; }
bool is_8bit(int32_t type) { return type == UMAP_I8 || type == UMAP_F8; }

int64_t scale_count(const umap_rows &m) { return m.group ? (m.cols + m.group - 1) / m.group : 1; }

// The bytes of one array: rows of `width` bytes, `pitch` apart.
struct Span {
    uintptr_t at;
    int64_t rows, width, pitch;
    uintptr_t end() const { return rows > 0 ? at + (uintptr_t)((rows - 1) * pitch + width) : at; }
};
Span span(const umap_rows &m)
{
    const int64_t e = elem_bytes(m.type);
    return {(uintptr_t)m.data, m.rows, m.cols * e, m.stride * e};
}
Span scale_span(const umap_rows &m)
{
    return {(uintptr_t)m.scales, m.scales ? 1 : 0, m.rows * scale_count(m) * 4, 0};
}
Span flat(const void *p, int64_t bytes) { return {(uintptr_t)p, p && bytes > 0 ? 1 : 0, bytes, 0}; }

// Whether two arrays share a byte.  Columns of one wider buffer (the same pitch, or a
// single row among the other's) do not, though their address ranges interleave.
bool overlap(const Span &a, const Span &b)
{
    if (a.rows < 1 || b.rows < 1 || a.end() <= b.at || b.end() <= a.at) return false;
    const int64_t pitch = a.rows > 1 ? a.pitch : b.pitch;
    if ((a.rows > 1 || b.rows > 1) && (b.rows == 1 || b.pitch == pitch) && pitch > 0) {
        const Span &lo = a.at <= b.at ? a : b, &hi = a.at <= b.at ? b : a;
        const int64_t off = (int64_t)((hi.at - lo.at) % (uintptr_t)pitch);
        return !(off >= lo.width && off + hi.width <= pitch);
    }
    return true;
}
bool same_place(const umap_rows &a, const umap_rows &b)
{
    return a.data == b.data && (a.stride == b.stride || a.rows <= 1) && a.type == b.type;
}
int refuse_overlap(const char *name, const Span &out, std::initializer_list<Span> others)
{
    for (const Span &o : others)
        if (overlap(out, o)) return fail(UMAP_E_INVAL, "%s overlaps another array of the call", name);
    return UMAP_OK;
}

constexpr int32_t kMaxCols = 1 << 20;
constexpr int32_t kMaxNormCols = 32768;
constexpr int64_t kMaxElements = (int64_t)1 << 56;   // of a matrix, gaps included: byte offsets fit 64 bits

#define UL_TRY(expr)                    \
    do {                                \
        const int ul_c_ = (expr);       \
        if (ul_c_ != UMAP_OK) return ul_c_; \
    } while (0)

// One matrix: its scalars, and data non-NULL where it has rows.
int check(const umap_rows *m, const char *name, int32_t max_cols, bool written, bool eight)
{
    if (!m) return fail(UMAP_E_INVAL, "%s must not be NULL", name);
    const int e = elem_bytes(m->type);
    if (!e || (!eight && is_8bit(m->type)))
        return fail(UMAP_E_INVAL, "%s: element type %d is not one this call takes", name, m->type);
    if (m->reserved) return fail(UMAP_E_INVAL, "%s: reserved must be 0", name);
    if (m->cols < 1 || m->cols > max_cols)
        return fail(UMAP_E_INVAL, "%s: cols must be in [1, %d], got %d", name, max_cols, m->cols);
    if (m->rows < 0) return fail(UMAP_E_INVAL, "%s: rows must be >= 0, got %lld", name, (long long)m->rows);
    if (m->stride < m->cols && m->rows > 1 && (written || m->stride != 0))
        return fail(UMAP_E_INVAL, "%s: stride %lld is below its %d cols", name, (long long)m->stride, m->cols);
    if (m->stride < 0 || (m->stride > 0 && m->rows > kMaxElements / m->stride) || m->rows > kMaxElements / m->cols)
        return fail(UMAP_E_INVAL, "%s: too many elements", name);
    if (m->rows > 0 && !m->data) return fail(UMAP_E_INVAL, "%s: data must not be NULL", name);
    if ((uintptr_t)m->data % e) return fail(UMAP_E_INVAL, "%s: data is not aligned to its elements", name);
    if (is_8bit(m->type)) {
        if (m->group != 0 && m->group != 32 && m->group != 64 && m->group != 128)
            return fail(UMAP_E_INVAL, "%s: group must be 0, 32, 64 or 128, got %d", name, m->group);
        if (m->rows > 0 && !m->scales) return fail(UMAP_E_INVAL, "%s: 8-bit rows need scales", name);
        if ((uintptr_t)m->scales % 4) return fail(UMAP_E_INVAL, "%s: scales are not aligned", name);
    } else if (m->scales || m->group) {
        return fail(UMAP_E_INVAL, "%s: scales and group are for 8-bit types", name);
    }
    return UMAP_OK;
}

int check_ids(const void *ids, int32_t id_type, int64_t n, ul::RowIds *out)
{
    *out = {nullptr, 0};
    if (!ids) return UMAP_OK;
    if (id_type != UMAP_I32 && id_type != UMAP_I64)
        return fail(UMAP_E_INVAL, "id_type must be UMAP_I32 or UMAP_I64, got %d", id_type);
    *out = {ids, id_type == UMAP_I32 ? 4 : 8};
    if ((uintptr_t)ids % out->bytes) return fail(UMAP_E_INVAL, "ids are not aligned");
    return n > kMaxElements ? fail(UMAP_E_INVAL, "too many ids") : UMAP_OK;
}

int check_shape(const umap_rows &m, const char *name, int64_t rows, int32_t cols)
{
    if (m.cols != cols) return fail(UMAP_E_INVAL, "%s has %d cols, the call %d", name, m.cols, cols);
    if (rows >= 0 && m.rows != rows)
        return fail(UMAP_E_INVAL, "%s has %lld rows, the call %lld", name, (long long)m.rows, (long long)rows);
    return UMAP_OK;
}

int check_workspace(const void *workspace, int64_t have, int64_t need)
{
    if (!workspace || have < need)
        return fail(UMAP_E_INVAL, "workspace of %lld bytes, the call needs %lld", workspace ? (long long)have : 0LL,
                    (long long)need);
    if ((uintptr_t)workspace % 16) return fail(UMAP_E_INVAL, "workspace must be aligned to 16 bytes");
    return UMAP_OK;
}

int check_weight(const void *weight, int32_t type, ul::RowWeight *out, const char *name = "weight")
{
    *out = {weight, UMAP_F32};
    if (!weight) return UMAP_OK;
    if (!is_float(type)) return fail(UMAP_E_INVAL, "%s_type %d is not a float type", name, type);
    out->type = type;
    if ((uintptr_t)weight % elem_bytes(type)) return fail(UMAP_E_INVAL, "%s is not aligned", name);
    return UMAP_OK;
}

int check_eps(float eps)
{
    return isfinite(eps) && eps >= 0.0f ? UMAP_OK : fail(UMAP_E_INVAL, "eps must be finite and >= 0");
}

int check_grad_sizes(int64_t n, int64_t rows, int32_t cols)
{
    if (n < 0 || n >= ((int64_t)1 << 31)) return fail(UMAP_E_INVAL, "rows of dout must be in [0, 2^31), got %lld", (long long)n);
    if (rows < 0 || rows >= ((int64_t)1 << 31) - 1)
        return fail(UMAP_E_INVAL, "rows of grad must be in [0, 2^31 - 1), got %lld", (long long)rows);
    if (cols < 1 || cols > kMaxCols) return fail(UMAP_E_INVAL, "cols must be in [1, %d], got %d", kMaxCols, cols);
    return UMAP_OK;
}

int check_norm_sizes(int64_t n, int32_t cols)
{
    if (n < 0 || n >= ((int64_t)1 << 31)) return fail(UMAP_E_INVAL, "rows must be in [0, 2^31), got %lld", (long long)n);
    if (cols < 1 || cols > kMaxNormCols)
        return fail(UMAP_E_INVAL, "cols must be in [1, %d], got %d", kMaxNormCols, cols);
    return UMAP_OK;
}

constexpr int64_t kMaxHeadRows = (int64_t)1 << 24, kMaxTokens = (int64_t)1 << 26;
constexpr int32_t kMaxTaught = 256;

int check_head_sizes(int64_t n, int64_t rows, int32_t cols, int32_t k, int32_t type)
{
    if (n < 0 || n >= kMaxHeadRows) return fail(UMAP_E_INVAL, "rows of h must be in [0, 2^24), got %lld", (long long)n);
    if (rows < 1 || rows >= kMaxTokens)
        return fail(UMAP_E_INVAL, "rows of table must be in [1, 2^26), got %lld", (long long)rows);
    if (cols < 1 || cols > kMaxNormCols)
        return fail(UMAP_E_INVAL, "cols must be in [1, %d], got %d", kMaxNormCols, cols);
    if (k < 1 || k > kMaxTaught) return fail(UMAP_E_INVAL, "k must be in [1, %d], got %d", kMaxTaught, k);
    return is_float(type) ? UMAP_OK : fail(UMAP_E_INVAL, "element type %d is not one this call takes", type);
}

// What the head's calls have in common: h, table, the rows' tokens, the teacher (which may be
// null where `taught` is false) and the scales.
int check_head(const umap_rows *h, const umap_rows *table, const void *ids, int32_t id_type, bool taught,
               const umap_rows *teacher, float scale, float teacher_scale, ul::RowIds *at)
{
    UL_TRY(check(h, "h", kMaxNormCols, false, false));
    UL_TRY(check(table, "table", kMaxNormCols, false, false));
    UL_TRY(check_shape(*table, "table", -1, h->cols));
    if (table->type != h->type) return fail(UMAP_E_INVAL, "table must have h's type");
    if (taught) {
        UL_TRY(check(teacher, "teacher", kMaxTaught, false, false));
        UL_TRY(check_shape(*teacher, "teacher", h->rows, teacher->cols));
    }
    const int32_t k = taught ? teacher->cols : 1;
    UL_TRY(check_head_sizes(h->rows, table->rows, h->cols, k, h->type));
    UL_TRY(check_ids(ids, id_type, h->rows * k, at));
    if (!ids && h->rows > 0) return fail(UMAP_E_INVAL, "%s must not be NULL", taught ? "ids" : "targets");
    if (!isfinite(scale)) return fail(UMAP_E_INVAL, "scale must be finite");
    return isfinite(teacher_scale) ? UMAP_OK : fail(UMAP_E_INVAL, "teacher_scale must be finite");
}

int check_floats(const float *p, const char *name, int64_t n, bool needed)
{
    if (needed && n > 0 && !p) return fail(UMAP_E_INVAL, "%s must not be NULL", name);
    return (uintptr_t)p % 4 ? fail(UMAP_E_INVAL, "%s is not aligned", name) : UMAP_OK;
}

int head(const char *name, const umap_rows *h, const umap_rows *table, const void *ids, int32_t id_type, bool taught,
         const umap_rows *teacher, float scale, float teacher_scale, float *loss, float *lse, void *workspace,
         int64_t workspace_bytes, void *stream)
{
    ul::RowIds at;
    UL_TRY(check_head(h, table, ids, id_type, taught, teacher, scale, teacher_scale, &at));
    const int64_t n = h->rows, k = taught ? teacher->cols : 1;
    UL_TRY(check_floats(loss, "loss", n, true));
    UL_TRY(check_floats(lse, "lse", n, true));
    const int64_t need = ul::rows_head_bytes(n, table->rows, h->cols, h->type);
    UL_TRY(check_workspace(workspace, workspace_bytes, need));
    const Span hs = span(*h), ts = span(*table), is = flat(ids, n * k * at.bytes), as = taught ? span(*teacher) : flat(nullptr, 0),
               ls = flat(loss, n * 4), es = flat(lse, n * 4), work = flat(workspace, need);
    UL_TRY(refuse_overlap("loss", ls, {hs, ts, is, as, es, work}));
    UL_TRY(refuse_overlap("lse", es, {hs, ts, is, as, work}));
    UL_TRY(refuse_overlap("workspace", work, {hs, ts, is, as}));
    if (n == 0) return UMAP_OK;
    return launched(ul::launch_rows_head(*h, *table, at, taught ? teacher : nullptr, scale, teacher_scale, loss, lse,
                                         workspace, static_cast<hipStream_t>(stream)),
                    name);
}

int head_grad(const char *name, const umap_rows *h, const umap_rows *table, const void *ids, int32_t id_type, bool taught,
              const umap_rows *teacher, float scale, float teacher_scale, const float *lse, const float *dloss,
              float dscale, const umap_rows *dh, const umap_rows *dtable, int32_t accumulate, void *workspace,
              int64_t workspace_bytes, void *stream)
{
    ul::RowIds at;
    UL_TRY(check_head(h, table, ids, id_type, taught, teacher, scale, teacher_scale, &at));
    const int64_t n = h->rows, k = taught ? teacher->cols : 1;
    UL_TRY(check_floats(lse, "lse", n, true));
    UL_TRY(check_floats(dloss, "dloss", n, false));
    if (!isfinite(dscale)) return fail(UMAP_E_INVAL, "dscale must be finite");
    if (!dh && !dtable) return fail(UMAP_E_INVAL, "dh and dtable must not both be NULL");
    if (dh) {
        UL_TRY(check(dh, "dh", kMaxNormCols, true, false));
        UL_TRY(check_shape(*dh, "dh", n, h->cols));
        if (dh->type != h->type) return fail(UMAP_E_INVAL, "dh must have h's type");
    }
    if (dtable) {
        UL_TRY(check(dtable, "dtable", kMaxNormCols, true, false));
        UL_TRY(check_shape(*dtable, "dtable", table->rows, h->cols));
        if (dtable->type != h->type) return fail(UMAP_E_INVAL, "dtable must have table's type");
    }
    if (accumulate != 0 && accumulate != 1) return fail(UMAP_E_INVAL, "accumulate must be 0 or 1, got %d", accumulate);
    const int64_t need = ul::rows_head_grad_bytes(n, table->rows, h->cols, (int32_t)k, h->type);
    UL_TRY(check_workspace(workspace, workspace_bytes, need));
    const Span none = flat(nullptr, 0), hs = span(*h), ts = span(*table), is = flat(ids, n * k * at.bytes),
               as = taught ? span(*teacher) : none, es = flat(lse, n * 4), ws = flat(dloss, n * 4),
               dhs = dh ? span(*dh) : none, dts = dtable ? span(*dtable) : none, work = flat(workspace, need);
    UL_TRY(refuse_overlap("dh", dhs, {hs, ts, is, as, es, ws, dts, work}));
    UL_TRY(refuse_overlap("dtable", dts, {hs, ts, is, as, es, ws, work}));
    UL_TRY(refuse_overlap("workspace", work, {hs, ts, is, as, es, ws}));
    if (n == 0 && (!dtable || accumulate)) return UMAP_OK;
    return launched(ul::launch_rows_head_grad(*h, *table, at, taught ? teacher : nullptr, scale, teacher_scale, lse, dloss,
                                              dscale, dh, dtable, accumulate != 0, workspace,
                                              static_cast<hipStream_t>(stream)),
                    name);
}

}  // namespace

extern "C" {

int umap_rows_lookup(const umap_rows *table, const void *ids, int32_t id_type, float scale, const umap_rows *out,
                     void *stream)
{
    UL_TRY(check(table, "table", kMaxCols, false, true));
    UL_TRY(check(out, "out", kMaxCols, true, false));
    UL_TRY(check_shape(*out, "out", -1, table->cols));
    ul::RowIds at;
    UL_TRY(check_ids(ids, id_type, out->rows, &at));
    if (!ids && out->rows > table->rows)
        return fail(UMAP_E_INVAL, "out has %lld rows, the table %lld", (long long)out->rows, (long long)table->rows);
    if (!isfinite(scale)) return fail(UMAP_E_INVAL, "scale must be finite");
    UL_TRY(refuse_overlap("out", span(*out), {span(*table), scale_span(*table), flat(ids, out->rows * at.bytes)}));
    if (out->rows == 0) return UMAP_OK;
    return launched(ul::launch_rows_lookup(*table, at, scale, *out, static_cast<hipStream_t>(stream)),
                    "umap_rows_lookup");
}

int64_t umap_rows_lookup_grad_workspace(int64_t n, int64_t rows, int32_t cols)
{
    UL_TRY(check_grad_sizes(n, rows, cols));
    return ul::rows_lookup_grad_bytes(n, rows, cols);
}

int umap_rows_lookup_grad(const umap_rows *dout, const void *ids, int32_t id_type, float scale, const umap_rows *grad,
                          int32_t accumulate, void *workspace, int64_t workspace_bytes, void *stream)
{
    UL_TRY(check(dout, "dout", kMaxCols, false, false));
    UL_TRY(check(grad, "grad", kMaxCols, true, false));
    UL_TRY(check_shape(*grad, "grad", -1, dout->cols));
    UL_TRY(check_grad_sizes(dout->rows, grad->rows, grad->cols));
    ul::RowIds at;
    UL_TRY(check_ids(ids, id_type, dout->rows, &at));
    if (!ids && dout->rows > 0) return fail(UMAP_E_INVAL, "ids must not be NULL");
    if (!isfinite(scale)) return fail(UMAP_E_INVAL, "scale must be finite");
    if (accumulate != 0 && accumulate != 1) return fail(UMAP_E_INVAL, "accumulate must be 0 or 1, got %d", accumulate);
    const int64_t need = ul::rows_lookup_grad_bytes(dout->rows, grad->rows, grad->cols);
    UL_TRY(check_workspace(workspace, workspace_bytes, need));
    const Span id_span = flat(ids, dout->rows * at.bytes), work = flat(workspace, need);
    UL_TRY(refuse_overlap("grad", span(*grad), {span(*dout), id_span, work}));
    UL_TRY(refuse_overlap("workspace", work, {span(*dout), id_span}));
    if (grad->rows == 0 || (accumulate && dout->rows == 0)) return UMAP_OK;
    return launched(ul::launch_rows_lookup_grad(*dout, at, scale, *grad, accumulate != 0, workspace,
                                                static_cast<hipStream_t>(stream)),
                    "umap_rows_lookup_grad");
}

int umap_rows_norm(const umap_rows *x, const void *ids, int32_t id_type, float scale, const umap_rows *residual,
                   const umap_rows *h, const void *weight, int32_t weight_type, float eps, const umap_rows *y,
                   void *stream)
{
    UL_TRY(check(x, "x", kMaxNormCols, false, false));
    UL_TRY(check(y, "y", kMaxNormCols, true, true));
    const int64_t n = y->rows;
    UL_TRY(check_norm_sizes(n, x->cols));
    UL_TRY(check_shape(*y, "y", -1, x->cols));
    ul::RowIds at;
    UL_TRY(check_ids(ids, id_type, n, &at));
    if (!ids) UL_TRY(check_shape(*x, "x", n, x->cols));
    if (!isfinite(scale)) return fail(UMAP_E_INVAL, "scale must be finite");
    if (residual) {
        UL_TRY(check(residual, "residual", kMaxNormCols, false, false));
        UL_TRY(check_shape(*residual, "residual", n, x->cols));
        if (residual->type != x->type) return fail(UMAP_E_INVAL, "residual must have x's type");
    }
    if (h) {
        UL_TRY(check(h, "h", kMaxNormCols, true, false));
        UL_TRY(check_shape(*h, "h", n, x->cols));
        if (h->type != x->type) return fail(UMAP_E_INVAL, "h must have x's type");
    }
    ul::RowWeight w;
    UL_TRY(check_weight(weight, weight_type, &w));
    UL_TRY(check_eps(eps));
    const Span none = flat(nullptr, 0), xs = span(*x), rs = residual ? span(*residual) : none,
               hs = h ? span(*h) : none, ws = flat(weight, (int64_t)x->cols * elem_bytes(w.type)),
               is = flat(ids, n * at.bytes);
    const bool h_is_x = h && !ids && same_place(*h, *x), h_is_r = h && residual && same_place(*h, *residual);
    UL_TRY(refuse_overlap("y", span(*y), {xs, rs, hs, ws, is, scale_span(*y)}));
    UL_TRY(refuse_overlap("y's scales", scale_span(*y), {xs, rs, hs, ws, is}));
    UL_TRY(refuse_overlap("h", hs, {h_is_x ? none : xs, h_is_r ? none : rs, ws, is}));
    if (n == 0) return UMAP_OK;
    return launched(ul::launch_rows_norm(*x, at, scale, residual, h, w, eps, *y, static_cast<hipStream_t>(stream)),
                    "umap_rows_norm");
}

int64_t umap_rows_norm_grad_workspace(int64_t n, int32_t cols)
{
    UL_TRY(check_norm_sizes(n, cols));
    return ul::rows_norm_grad_bytes(n, cols);
}

int umap_rows_norm_grad(const umap_rows *dy, const umap_rows *h, const umap_rows *dh, const void *weight,
                        int32_t weight_type, float eps, const umap_rows *dx, float *dweight, void *workspace,
                        int64_t workspace_bytes, void *stream)
{
    UL_TRY(check(dy, "dy", kMaxNormCols, false, false));
    UL_TRY(check(h, "h", kMaxNormCols, false, false));
    UL_TRY(check(dx, "dx", kMaxNormCols, true, false));
    const int64_t n = dy->rows;
    const int32_t cols = dy->cols;
    UL_TRY(check_norm_sizes(n, cols));
    UL_TRY(check_shape(*h, "h", n, cols));
    UL_TRY(check_shape(*dx, "dx", n, cols));
    if (dh) {
        UL_TRY(check(dh, "dh", kMaxNormCols, false, false));
        UL_TRY(check_shape(*dh, "dh", n, cols));
    }
    if (h->type != dy->type || dx->type != dy->type || (dh && dh->type != dy->type))
        return fail(UMAP_E_INVAL, "dy, h, dh and dx must have one type");
    ul::RowWeight w;
    UL_TRY(check_weight(weight, weight_type, &w));
    UL_TRY(check_eps(eps));
    if ((uintptr_t)dweight % 4) return fail(UMAP_E_INVAL, "dweight is not aligned");
    const int64_t need = dweight ? ul::rows_norm_grad_bytes(n, cols) : 0;
    if (dweight) UL_TRY(check_workspace(workspace, workspace_bytes, need));
    const Span none = flat(nullptr, 0), ys = span(*dy), hs = span(*h), us = dh ? span(*dh) : none,
               ws = flat(weight, (int64_t)cols * elem_bytes(w.type)), os = span(*dx),
               gs = flat(dweight, (int64_t)cols * 4), work = flat(dweight ? workspace : nullptr, need);
    const bool is_dy = same_place(*dx, *dy), is_dh = dh && same_place(*dx, *dh);
    UL_TRY(refuse_overlap("dx", os, {is_dy ? none : ys, hs, is_dh ? none : us, ws, gs, work}));
    UL_TRY(refuse_overlap("dweight", gs, {ys, hs, us, ws, work}));
    UL_TRY(refuse_overlap("workspace", work, {ys, hs, us, ws}));
    if (n == 0 && !dweight) return UMAP_OK;
    return launched(ul::launch_rows_norm_grad(*dy, *h, dh, w, eps, *dx, dweight, workspace,
                                              static_cast<hipStream_t>(stream)),
                    "umap_rows_norm_grad");
}

int umap_rows_layer_norm(const umap_rows *x, const umap_rows *residual, const umap_rows *h, const void *weight,
                         int32_t weight_type, const void *bias, int32_t bias_type, float eps, const umap_rows *y,
                         void *stream)
{
    UL_TRY(check(x, "x", kMaxNormCols, false, false));
    UL_TRY(check(y, "y", kMaxNormCols, true, false));
    const int64_t n = x->rows;
    UL_TRY(check_norm_sizes(n, x->cols));
    UL_TRY(check_shape(*y, "y", n, x->cols));
    if (residual) {
        UL_TRY(check(residual, "residual", kMaxNormCols, false, false));
        UL_TRY(check_shape(*residual, "residual", n, x->cols));
        if (residual->type != x->type) return fail(UMAP_E_INVAL, "residual must have x's type");
    }
    if (h) {
        UL_TRY(check(h, "h", kMaxNormCols, true, false));
        UL_TRY(check_shape(*h, "h", n, x->cols));
        if (h->type != x->type) return fail(UMAP_E_INVAL, "h must have x's type");
    }
    ul::RowWeight w, b;
    UL_TRY(check_weight(weight, weight_type, &w));
    UL_TRY(check_weight(bias, bias_type, &b, "bias"));
    UL_TRY(check_eps(eps));
    const Span none = flat(nullptr, 0), xs = span(*x), rs = residual ? span(*residual) : none, hs = h ? span(*h) : none,
               ws = flat(weight, (int64_t)x->cols * elem_bytes(w.type)), bs = flat(bias, (int64_t)x->cols * elem_bytes(b.type));
    const bool h_is_x = h && same_place(*h, *x), h_is_r = h && residual && same_place(*h, *residual);
    UL_TRY(refuse_overlap("y", span(*y), {xs, rs, hs, ws, bs}));
    UL_TRY(refuse_overlap("h", hs, {h_is_x ? none : xs, h_is_r ? none : rs, ws, bs}));
    if (n == 0) return UMAP_OK;
    return launched(ul::launch_rows_layer_norm(*x, residual, h, w, b, eps, *y, static_cast<hipStream_t>(stream)),
                    "umap_rows_layer_norm");
}

int64_t umap_rows_layer_norm_grad_workspace(int64_t n, int32_t cols)
{
    UL_TRY(check_norm_sizes(n, cols));
    return ul::rows_layer_norm_grad_bytes(n, cols);
}

int umap_rows_layer_norm_grad(const umap_rows *dy, const umap_rows *h, const umap_rows *dh, const void *weight,
                              int32_t weight_type, float eps, const umap_rows *dx, float *dweight, float *dbias,
                              void *workspace, int64_t workspace_bytes, void *stream)
{
    UL_TRY(check(dy, "dy", kMaxNormCols, false, false));
    UL_TRY(check(h, "h", kMaxNormCols, false, false));
    UL_TRY(check(dx, "dx", kMaxNormCols, true, false));
    const int64_t n = dy->rows;
    const int32_t cols = dy->cols;
    UL_TRY(check_norm_sizes(n, cols));
    UL_TRY(check_shape(*h, "h", n, cols));
    UL_TRY(check_shape(*dx, "dx", n, cols));
    if (dh) {
        UL_TRY(check(dh, "dh", kMaxNormCols, false, false));
        UL_TRY(check_shape(*dh, "dh", n, cols));
    }
    if (h->type != dy->type || dx->type != dy->type || (dh && dh->type != dy->type))
        return fail(UMAP_E_INVAL, "dy, h, dh and dx must have one type");
    ul::RowWeight w;
    UL_TRY(check_weight(weight, weight_type, &w));
    UL_TRY(check_eps(eps));
    UL_TRY(check_floats(dweight, "dweight", cols, false));
    UL_TRY(check_floats(dbias, "dbias", cols, false));
    const bool sums = dweight || dbias;
    const int64_t need = sums ? ul::rows_layer_norm_grad_bytes(n, cols) : 0;
    if (sums) UL_TRY(check_workspace(workspace, workspace_bytes, need));
    const Span none = flat(nullptr, 0), ys = span(*dy), hs = span(*h), us = dh ? span(*dh) : none,
               ws = flat(weight, (int64_t)cols * elem_bytes(w.type)), os = span(*dx), gs = flat(dweight, (int64_t)cols * 4),
               bs = flat(dbias, (int64_t)cols * 4), work = flat(sums ? workspace : nullptr, need);
    const bool is_dy = same_place(*dx, *dy), is_dh = dh && same_place(*dx, *dh);
    UL_TRY(refuse_overlap("dx", os, {is_dy ? none : ys, hs, is_dh ? none : us, ws, gs, bs, work}));
    UL_TRY(refuse_overlap("dweight", gs, {ys, hs, us, ws, bs, work}));
    UL_TRY(refuse_overlap("dbias", bs, {ys, hs, us, ws, work}));
    UL_TRY(refuse_overlap("workspace", work, {ys, hs, us, ws}));
    if (n == 0 && !sums) return UMAP_OK;
    return launched(ul::launch_rows_layer_norm_grad(*dy, *h, dh, w, eps, *dx, dweight, dbias, workspace,
                                                    static_cast<hipStream_t>(stream)),
                    "umap_rows_layer_norm_grad");
}

int64_t umap_rows_cross_entropy_workspace(int64_t n, int64_t rows, int32_t cols, int32_t type)
{
    UL_TRY(check_head_sizes(n, rows, cols, 1, type));
    return ul::rows_head_bytes(n, rows, cols, type);
}

int umap_rows_cross_entropy(const umap_rows *h, const umap_rows *table, const void *targets, int32_t target_type,
                            float scale, float *loss, float *lse, void *workspace, int64_t workspace_bytes, void *stream)
{
    return head("umap_rows_cross_entropy", h, table, targets, target_type, false, nullptr, scale, 1.0f, loss, lse,
                workspace, workspace_bytes, stream);
}

int64_t umap_rows_cross_entropy_grad_workspace(int64_t n, int64_t rows, int32_t cols, int32_t type)
{
    UL_TRY(check_head_sizes(n, rows, cols, 1, type));
    return ul::rows_head_grad_bytes(n, rows, cols, 1, type);
}

int umap_rows_cross_entropy_grad(const umap_rows *h, const umap_rows *table, const void *targets, int32_t target_type,
                                 float scale, const float *lse, const float *dloss, float dscale, const umap_rows *dh,
                                 const umap_rows *dtable, int32_t accumulate, void *workspace, int64_t workspace_bytes,
                                 void *stream)
{
    return head_grad("umap_rows_cross_entropy_grad", h, table, targets, target_type, false, nullptr, scale, 1.0f, lse,
                     dloss, dscale, dh, dtable, accumulate, workspace, workspace_bytes, stream);
}

int64_t umap_rows_distill_workspace(int64_t n, int64_t rows, int32_t cols, int32_t k, int32_t type)
{
    UL_TRY(check_head_sizes(n, rows, cols, k, type));
    return ul::rows_head_bytes(n, rows, cols, type);
}

int umap_rows_distill(const umap_rows *h, const umap_rows *table, const void *ids, int32_t id_type,
                      const umap_rows *teacher, float scale, float teacher_scale, float *loss, float *lse,
                      void *workspace, int64_t workspace_bytes, void *stream)
{
    return head("umap_rows_distill", h, table, ids, id_type, true, teacher, scale, teacher_scale, loss, lse, workspace,
                workspace_bytes, stream);
}

int64_t umap_rows_distill_grad_workspace(int64_t n, int64_t rows, int32_t cols, int32_t k, int32_t type)
{
    UL_TRY(check_head_sizes(n, rows, cols, k, type));
    return ul::rows_head_grad_bytes(n, rows, cols, k, type);
}

int umap_rows_distill_grad(const umap_rows *h, const umap_rows *table, const void *ids, int32_t id_type,
                           const umap_rows *teacher, float scale, float teacher_scale, const float *lse,
                           const float *dloss, float dscale, const umap_rows *dh, const umap_rows *dtable,
                           int32_t accumulate, void *workspace, int64_t workspace_bytes, void *stream)
{
    return head_grad("umap_rows_distill_grad", h, table, ids, id_type, true, teacher, scale, teacher_scale, lse, dloss,
                     dscale, dh, dtable, accumulate, workspace, workspace_bytes, stream);
}

}  // extern "C"
