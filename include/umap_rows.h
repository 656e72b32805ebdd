/*
 * umap_rows.h -- C ABI of the token-row operators of libumap_layout.so: rows of
 * a learned table by id (with scaling) and the gradient of that by sorted ids,
 * and the root-mean-square norm of rows, with a residual's addition, into a
 * float type or into 8 bits with scales, and its gradient.
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

#ifdef __cplusplus
}
#endif

#endif /* UMAP_ROWS_H */
