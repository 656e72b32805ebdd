/*
 * umap_rows.h -- C ABI of the token-row operators of libumap_layout.so: rows of
 * a learned table by id (with scaling) and the gradient of that by sorted ids,
 * and the root-mean-square norm of rows, with a residual's addition, into a
 * float type or into 8 bits with scales, and its gradient; the mean and variance
 * norm and its gradient; and the head over a table of tokens, as a loss (softmax
 * cross entropy, or the divergence from a teacher's largest logits) and its
 * gradient, without the logits ever being kept.
 *
 * They stand in front of the layout: a table of word or token vectors is
 * trained, its rows are read by id, normalised (Euclidean distances of
 * normalised rows order as cosines do), kept in 8 bits, and their neighbours
 * become the graph of umap_fuzzy_graph_device and umap_layout_create_device.
 *
 * Conventions: those of umap_layout.h (status codes, umap_layout_last_error,
 * no exception crosses the ABI, argument checks before any HIP call).  All
 * arrays are device memory of the current device.  The calls enqueue kernels
 * on `stream` (a hipStream_t, or NULL for the null stream) and return: they do
 * not block, allocate or copy, and can be captured into a HIP graph.  Arrays
 * that another stream writes or frees are for the caller to order.  Results
 * are the same bit for bit from call to call.
 */
#ifndef UMAP_ROWS_H
#define UMAP_ROWS_H

#include <stdint.h>

#include "umap_layout.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types.  8-bit values stand for q times their scale. */
#define UMAP_F32 0
#define UMAP_F16 1
#define UMAP_BF16 2
#define UMAP_I8 3     /* two's complement, -127 .. 127 when written          */
#define UMAP_F8 4     /* E4M3: 4 exponent and 3 mantissa bits, largest 448,
                         NaN, no infinity                                    */
/* Id types. */
#define UMAP_I32 8
#define UMAP_I64 9

/*
 * umap_rows -- a matrix of rows: element (i, c) is element i * stride + c of
 * data.  stride (elements) >= cols, any value, as is data's alignment beyond
 * the element's own; for a matrix that is only read it may also be 0 (every row
 * the same).  For UMAP_I8 and UMAP_F8 scales holds ceil(cols / group) fp32
 * per row, without gaps, one for each `group` columns (32, 64 or 128; 0: one
 * for the whole row, stored as one per row); else scales is NULL and group 0.
 */
typedef struct {
    void *data;
    float *scales;
    int64_t rows;
    int64_t stride;
    int32_t cols;
    int32_t type;
    int32_t group;
    int32_t reserved;   /* 0 */
} umap_rows;

/*
 * umap_rows_lookup -- out[t] = scale * table[ids[t]] for t < out->rows.
 *
 *   table    rows of any type, cols 1 .. 2^20.
 *   ids      out->rows ids of type id_type (UMAP_I32 or UMAP_I64); an id outside
 *            [0, table->rows) -- padding is -1, say -- gives a row of zeros.
 *            NULL: row t is table row t (a stored table read back; out->rows <=
 *            table->rows).
 *   scale    finite.
 *   out      UMAP_F32, UMAP_F16 or UMAP_BF16, the table's cols; the product is
 *            formed in fp32 and rounded once (to nearest even).
 *
 * out must not overlap the table or its scales.  Errors: UMAP_E_INVAL, UMAP_E_DEVICE.
 */
int umap_rows_lookup(const umap_rows *table, const void *ids, int32_t id_type, float scale, const umap_rows *out,
                     void *stream);

/*
 * umap_rows_lookup_grad -- the gradient of umap_rows_lookup for the table:
 * grad[v] = scale * sum over the t with ids[t] = v of dout[t], added in fp32 in a
 * fixed order (no atomics), rounded once to grad's type.
 *
 *   dout       UMAP_F32, UMAP_F16 or UMAP_BF16, one row per id, cols 1 .. 2^20,
 *              rows < 2^31.  Rows whose id is outside [0, grad->rows) take no
 *              part (nothing of them is read: they may hold NaN).
 *   grad       UMAP_F32, UMAP_F16 or UMAP_BF16, rows < 2^31 - 1.
 *   accumulate 0: every row of grad is written, zeros where no id points.
 *              1: the sums are added to grad (in fp32, rounded once); rows without
 *              an id are neither read nor written.  With scale = -step this is an
 *              SGD step on the rows in use.
 *   workspace  workspace_bytes >= umap_rows_lookup_grad_workspace(rows of dout,
 *              rows of grad, cols) bytes of device memory, 16-byte aligned,
 *              contents of no meaning before or after; it must stay untouched
 *              until the work on `stream` is done.
 *
 * No two of dout, ids, grad and workspace may overlap.  Errors: UMAP_E_INVAL, UMAP_E_DEVICE.
 */
int umap_rows_lookup_grad(const umap_rows *dout, const void *ids, int32_t id_type, float scale, const umap_rows *grad,
                          int32_t accumulate, void *workspace, int64_t workspace_bytes, void *stream);

/* Bytes of umap_rows_lookup_grad's workspace for n ids, a table of `rows` rows
 * and `cols` columns (> 0), or UMAP_E_INVAL.  Host only. */
int64_t umap_rows_lookup_grad_workspace(int64_t n, int64_t rows, int32_t cols);

/*
 * umap_rows_norm -- root-mean-square norm of rows:
 *   h[t] = x[t] + residual[t]                 (x[t]: scale * x[ids[t]] with ids)
 *   y[t] = h[t] / sqrt(mean_c h[t][c]^2 + eps) * weight
 * all in fp32 from the inputs on; h and y are rounded once each (y is computed
 * from the unrounded h).
 *
 *   x         UMAP_F32, UMAP_F16 or UMAP_BF16, cols 1 .. 32768.
 *   ids       NULL (x has y's rows; scale applies too), or y->rows ids of type
 *             id_type into x's rows: the lookup and the norm in one pass.  An id
 *             outside [0, x->rows) stands for a row of zeros.
 *   residual  NULL, or rows of x's type.
 *   h         NULL, or receives h in x's type.  It may be the residual itself or,
 *             without ids, x itself (the same data and stride).
 *   weight    cols values of type weight_type (UMAP_F32, UMAP_F16 or UMAP_BF16),
 *             or NULL for ones.
 *   eps       finite, >= 0 (a row of zeros with eps = 0 gives NaN).
 *   y         rows < 2^31 of UMAP_F32, UMAP_F16 or UMAP_BF16, or of UMAP_I8 / UMAP_F8
 *             with scales, which are written too: of each group of columns the scale
 *             is the largest |y| / 127 (UMAP_I8) or / 448 (UMAP_F8), and the values
 *             are y / scale, both quotients formed in fp32 to nearest even, the
 *             values then rounded likewise.  A group whose largest |y| is below
 *             2^-100 is stored as zeros with scale 0, one that holds a NaN or an
 *             infinity as zeros with scale NaN (it reads back as NaN).
 *
 * Sums of squares beyond fp32's range are formed again from scaled values, so
 * finite rows have finite norms.  Apart from h's aliases no output may overlap
 * an input or another output.  Errors: UMAP_E_INVAL, UMAP_E_DEVICE.
 */
int umap_rows_norm(const umap_rows *x, const void *ids, int32_t id_type, float scale, const umap_rows *residual,
                   const umap_rows *h, const void *weight, int32_t weight_type, float eps, const umap_rows *y,
                   void *stream);

/*
 * umap_rows_norm_grad -- the gradient of y = h / sqrt(mean h^2 + eps) * weight.  With
 * rho = 1 / sqrt(mean_c h^2 + eps) and g = dy * weight:
 *   dx[t]   = rho g - h rho^3 mean_c(g h) + dh[t]
 *   dweight = sum_t dy[t] * h[t] * rho
 * in fp32, rounded once.  dx is the gradient of h, which is also the residual's.
 * That of umap_rows_norm's x is scale * dx: dx itself where scale is 1, else what
 * umap_rows_lookup(dx, NULL, .., scale) gives or, where x was gathered,
 * umap_rows_lookup_grad with that scale.
 *
 *   dy, h    UMAP_F32, UMAP_F16 or UMAP_BF16, of one type, cols 1 .. 32768,
 *            rows < 2^31.
 *   dh       NULL, or the gradient that reaches h by other ways (the same type).
 *   weight   as for umap_rows_norm.
 *   dx       the same type; receives the gradient of h.  It may be dy or dh itself
 *            (the same data and stride).
 *   dweight  NULL, or cols fp32, overwritten; rows are added in a fixed order.
 *   workspace  NULL when dweight is NULL, else workspace_bytes >=
 *            umap_rows_norm_grad_workspace(rows, cols) bytes of device memory,
 *            16-byte aligned, as for umap_rows_lookup_grad.
 *
 * Apart from dx's aliases no output may overlap an input or another output.
 * Errors: UMAP_E_INVAL, UMAP_E_DEVICE.
 */
int umap_rows_norm_grad(const umap_rows *dy, const umap_rows *h, const umap_rows *dh, const void *weight,
                        int32_t weight_type, float eps, const umap_rows *dx, float *dweight, void *workspace,
                        int64_t workspace_bytes, void *stream);

/* Bytes of umap_rows_norm_grad's workspace (> 0), or UMAP_E_INVAL.  Host only. */
int64_t umap_rows_norm_grad_workspace(int64_t n, int32_t cols);

/*
 * umap_rows_layer_norm -- mean and variance norm of rows:
 *   h[t] = x[t] + residual[t]
 *   y[t] = (h[t] - mean_c h[t][c]) / sqrt(mean_c (h[t][c] - mean h[t])^2 + eps) * weight + bias
 * all in fp32 from the inputs on; h and y are rounded once each (y is computed
 * from the unrounded h).
 *
 *   x         UMAP_F32, UMAP_F16 or UMAP_BF16, cols 1 .. 32768, rows < 2^31.
 *   residual  NULL, or rows of x's type.
 *   h         NULL, or receives h in x's type.  It may be x or the residual itself
 *             (the same data and stride).
 *   weight, bias  cols values each of type weight_type and bias_type (UMAP_F32,
 *             UMAP_F16 or UMAP_BF16), or NULL for ones and for zeros.
 *   eps       finite, >= 0 (with eps = 0 a row of equal values gives NaN).
 *   y         UMAP_F32, UMAP_F16 or UMAP_BF16, x's rows and cols.
 *
 * Sums of squares beyond fp32's range are formed again from scaled values, so
 * finite rows have finite norms.  Apart from h's aliases no output may overlap
 * an input or another output.  Errors: UMAP_E_INVAL, UMAP_E_DEVICE.
 */
int umap_rows_layer_norm(const umap_rows *x, const umap_rows *residual, const umap_rows *h, const void *weight,
                         int32_t weight_type, const void *bias, int32_t bias_type, float eps, const umap_rows *y,
                         void *stream);

/*
 * umap_rows_layer_norm_grad -- its gradient.  With u = (h - mean h) rho,
 * rho = 1 / sqrt(mean (h - mean h)^2 + eps) and g = dy * weight:
 *   dx[t]   = rho (g - mean_c g - u mean_c(g u)) + dh[t]
 *   dweight = sum_t dy[t] * u[t],  dbias = sum_t dy[t]
 * in fp32, rounded once.  dx is the gradient of h, which is also x's and the
 * residual's.
 *
 *   dy, h    UMAP_F32, UMAP_F16 or UMAP_BF16, of one type, cols 1 .. 32768,
 *            rows < 2^31.
 *   dh       NULL, or the gradient that reaches h by other ways (the same type).
 *   weight   as for umap_rows_layer_norm.
 *   dx       the same type; receives the gradient of h.  It may be dy or dh itself
 *            (the same data and stride).
 *   dweight, dbias  NULL, or cols fp32 each, overwritten; rows are added in a fixed
 *            order.
 *   workspace  NULL when both are NULL, else workspace_bytes >=
 *            umap_rows_layer_norm_grad_workspace(rows, cols) bytes of device
 *            memory, 16-byte aligned, as for umap_rows_lookup_grad.
 *
 * Apart from dx's aliases no output may overlap an input or another output.
 * Errors: UMAP_E_INVAL, UMAP_E_DEVICE.
 */
int umap_rows_layer_norm_grad(const umap_rows *dy, const umap_rows *h, const umap_rows *dh, const void *weight,
                              int32_t weight_type, float eps, const umap_rows *dx, float *dweight, float *dbias,
                              void *workspace, int64_t workspace_bytes, void *stream);

/* Bytes of umap_rows_layer_norm_grad's workspace (> 0), or UMAP_E_INVAL.  Host only. */
int64_t umap_rows_layer_norm_grad_workspace(int64_t n, int32_t cols);

/*
 * umap_rows_cross_entropy -- softmax cross entropy of rows against a whole table:
 *   z[t][v] = scale * sum_c h[t][c] table[v][c]
 *   lse[t]  = log sum_v exp z[t][v]
 *   loss[t] = lse[t] - z[t][targets[t]]
 * in fp32 from the inputs on.  The logits z are formed tile by tile and not kept.
 * One row is a call like any other: a token's log-likelihood is minus its loss.
 *
 *   h        UMAP_F32, UMAP_F16 or UMAP_BF16, cols 1 .. 32768, rows < 2^24.
 *   table    h's type and cols, 1 <= rows < 2^26.
 *   targets  h->rows ids of type target_type (UMAP_I32 or UMAP_I64).  A row whose
 *            target lies outside [0, table->rows) -- padding is -1, say -- takes
 *            no part: its loss is 0 (its lse is computed all the same).
 *   scale    finite.
 *   loss, lse  h->rows fp32 each, overwritten.
 *   workspace  workspace_bytes >= umap_rows_cross_entropy_workspace(h->rows,
 *            table->rows, cols, type) bytes of device memory, 16-byte aligned,
 *            contents of no meaning before or after; it must stay untouched until
 *            the work on `stream` is done.
 *
 * A row of h or table that is not finite, or logits beyond fp32's range, make the
 * lse of the rows concerned infinite or NaN.  No output may overlap an input or
 * another output.  Errors: UMAP_E_INVAL, UMAP_E_DEVICE.
 */
int umap_rows_cross_entropy(const umap_rows *h, const umap_rows *table, const void *targets, int32_t target_type,
                            float scale, float *loss, float *lse, void *workspace, int64_t workspace_bytes,
                            void *stream);

/* Bytes of umap_rows_cross_entropy's workspace (> 0), or UMAP_E_INVAL.  Host only.
 * They do for any stride and alignment: room for a copy of h (its columns a
 * multiple of 64), for one of 128 MB of the table (or of 256 of its rows, if that is
 * more), used where they are not whole pieces of 16 bytes, and for the tiles' sums,
 * 128 MB at most, or 32 bytes for each of the table's rows if that is more. */
int64_t umap_rows_cross_entropy_workspace(int64_t n, int64_t rows, int32_t cols, int32_t type);

/*
 * umap_rows_cross_entropy_grad -- the gradient of dscale * sum_t dloss[t] loss[t].  With
 *   D[t][v] = dscale dloss[t] (exp(z[t][v] - lse[t]) - (1 if v = targets[t], else 0))
 *   dh[t]     = scale sum_v D[t][v] table[v]
 *   dtable[v] = scale sum_t D[t][v] h[t]
 * The logits are formed again, for a piece of the table at a time, and D of the piece
 * is kept in h's type (fp32: not rounded; 16 bits: in two parts up to 256 rows, else
 * each entry rounded, by up to half a unit in its last place, which the sums average out);
 * all sums are fp32 and rounded once; their order is fixed.
 *
 *   h, table, targets, scale  as for umap_rows_cross_entropy.
 *   lse        what that call gave: the rounding of its logits then cancels against
 *              that of the same logits here, which one formed otherwise brings along.
 *   dloss      NULL (ones), or a weight for each row, fp32.  Rows of weight 0 and
 *              rows whose target lies outside the table take no part: their dh is
 *              zeros, and nothing of them reaches dtable (they may hold NaN).
 *              Weights may lie far apart: in fp16 dtable takes rows within 2^6 of the
 *              largest weight together, then those within 2^12, and so on down to
 *              2^96, beyond which they do not reach it; in bf16 and fp32 a row counts
 *              as far as h times its weight over the largest is in its type's range.
 *   dscale     finite (one over the rows for a mean, times a loss scale for fp16).
 *   dh         NULL, or receives the gradient of h: its type and shape.
 *   dtable     NULL, or receives the gradient of table: its type and shape.  Not
 *              both NULL.
 *   accumulate 0: dtable is overwritten; 1: the gradient is added to it (in fp32,
 *              rounded once), as for a table whose rows are looked up as well.
 *   workspace  as above, umap_rows_cross_entropy_grad_workspace(..) bytes.
 *
 * No output may overlap an input, another output or the workspace.  Errors:
 * UMAP_E_INVAL, UMAP_E_DEVICE.
 */
int umap_rows_cross_entropy_grad(const umap_rows *h, const umap_rows *table, const void *targets, int32_t target_type,
                                 float scale, const float *lse, const float *dloss, float dscale, const umap_rows *dh,
                                 const umap_rows *dtable, int32_t accumulate, void *workspace,
                                 int64_t workspace_bytes, void *stream);

/* Bytes of umap_rows_cross_entropy_grad's workspace (> 0), or UMAP_E_INVAL.  Host only.
 * Room for two copies of h (of up to 256 rows of 16 bits, four), for 128 MB of the
 * table as above, for D, 256 MB at most, or 256 entries for each row of h if that is
 * more, for dh in fp32 (once; up to 72 MB of it if that is more), and 100 + 8 k bytes
 * for each row.  The more rows, the fewer tokens a piece has, and every piece reads
 * and writes all sums of dh: of a very large batch, calls of some 16,384 rows each that
 * add to dtable take less time than one (131,072 rows of bf16 against 32,000 x 2,048:
 * 43 ms and 92), at the price of dtable's rounding in each.
 */
int64_t umap_rows_cross_entropy_grad_workspace(int64_t n, int64_t rows, int32_t cols, int32_t type);

/*
 * umap_rows_distill -- the divergence of the softmax over a table from a teacher
 * of which each row's largest logits are known.  With z and lse as for
 * umap_rows_cross_entropy, k = teacher->cols, places e, f < k and tokens v:
 *   s[t][e] = exp(teacher_scale teacher[t][e]) / sum_f exp(teacher_scale teacher[t][f])
 *   q[t][v] = sum of s[t][e] over ids[t][e] = v
 *   loss[t] = sum_v q[t][v] (log q[t][v] - (z[t][v] - lse[t])),  0 log 0 = 0
 * scale and teacher_scale are one over the temperature, times what else scales the
 * logits; the factor temperature^2 that usually goes with it is dscale's.
 *
 *   h, table, scale, loss, lse, workspace  as for umap_rows_cross_entropy.
 *   ids       h->rows x k ids of type id_type, without gaps: the teacher's tokens.
 *             Places whose id lies outside [0, table->rows), and places with a
 *             logit of -infinity, are empty: they take no part in the sums.  A row
 *             with empty places only takes no part: its loss is 0.  A token may come
 *             in several places of a row.
 *   teacher   UMAP_F32, UMAP_F16 or UMAP_BF16, h->rows rows of 1 <= k <= 256 logits.
 *
 * Errors: UMAP_E_INVAL, UMAP_E_DEVICE.
 */
int umap_rows_distill(const umap_rows *h, const umap_rows *table, const void *ids, int32_t id_type,
                      const umap_rows *teacher, float scale, float teacher_scale, float *loss, float *lse,
                      void *workspace, int64_t workspace_bytes, void *stream);

/* Bytes of umap_rows_distill's workspace (> 0), or UMAP_E_INVAL.  Host only. */
int64_t umap_rows_distill_workspace(int64_t n, int64_t rows, int32_t cols, int32_t k, int32_t type);

/*
 * umap_rows_distill_grad -- its gradient for h and table (the teacher's logits are
 * constants): umap_rows_cross_entropy_grad with
 *   D[t][v] = dscale dloss[t] (exp(z[t][v] - lse[t]) - q[t][v])
 * and the arguments of both.
 */
int umap_rows_distill_grad(const umap_rows *h, const umap_rows *table, const void *ids, int32_t id_type,
                           const umap_rows *teacher, float scale, float teacher_scale, const float *lse,
                           const float *dloss, float dscale, const umap_rows *dh, const umap_rows *dtable,
                           int32_t accumulate, void *workspace, int64_t workspace_bytes, void *stream);

/* Bytes of umap_rows_distill_grad's workspace (> 0), or UMAP_E_INVAL.  Host only. */
int64_t umap_rows_distill_grad_workspace(int64_t n, int64_t rows, int32_t cols, int32_t k, int32_t type);

#ifdef __cplusplus
}
#endif

#endif /* UMAP_ROWS_H */
