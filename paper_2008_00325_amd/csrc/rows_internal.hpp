// rows_internal.hpp -- launchers of the token-row operators (umap_rows.h), whose
// arguments rows_api.hip has checked.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "umap_rows.h"

namespace ul {

// Ids of a call: null, or int32 (bytes 4) or int64 (bytes 8) values.
struct RowIds {
    const void *data;
    int32_t bytes;
};

hipError_t launch_rows_lookup(const umap_rows &table, RowIds ids, float scale, const umap_rows &out, hipStream_t s);

// ---- gradient by sorted ids ----
int64_t rows_lookup_grad_bytes(int64_t n, int64_t rows, int32_t cols);
hipError_t launch_rows_lookup_grad(const umap_rows &dout, RowIds ids, float scale, const umap_rows &grad,
                                   bool accumulate, void *workspace, hipStream_t s);

// ---- norm ----
struct RowWeight {
    const void *data;   // or null: ones
    int32_t type;
};
// residual and h may be null.
hipError_t launch_rows_norm(const umap_rows &x, RowIds ids, float scale, const umap_rows *residual, const umap_rows *h,
                            RowWeight weight, float eps, const umap_rows &y, hipStream_t s);
int64_t rows_norm_grad_bytes(int64_t n, int32_t cols);
// dh and dweight may be null.
hipError_t launch_rows_norm_grad(const umap_rows &dy, const umap_rows &h, const umap_rows *dh, RowWeight weight,
                                 float eps, const umap_rows &dx, float *dweight, void *workspace, hipStream_t s);

// residual and h may be null.
hipError_t launch_rows_layer_norm(const umap_rows &x, const umap_rows *residual, const umap_rows *h, RowWeight weight,
                                  RowWeight bias, float eps, const umap_rows &y, hipStream_t s);
int64_t rows_layer_norm_grad_bytes(int64_t n, int32_t cols);
// dh, dweight and dbias may be null.
hipError_t launch_rows_layer_norm_grad(const umap_rows &dy, const umap_rows &h, const umap_rows *dh, RowWeight weight, float eps,
                                       const umap_rows &dx, float *dweight, float *dbias, void *workspace, hipStream_t s);

// ---- head: loss of rows against a table, with its gradient ----
// teacher may be null: one token a row, with share 1.
int64_t rows_head_bytes(int64_t n, int64_t vocab, int32_t cols, int32_t type);
hipError_t launch_rows_head(const umap_rows &h, const umap_rows &table, RowIds ids, const umap_rows *teacher, float scale,
                            float teacher_scale, float *loss, float *lse, void *workspace, hipStream_t s);
int64_t rows_head_grad_bytes(int64_t n, int64_t vocab, int32_t cols, int32_t k, int32_t type);
// dloss, dh and dtable may be null.
hipError_t launch_rows_head_grad(const umap_rows &h, const umap_rows &table, RowIds ids, const umap_rows *teacher, float scale,
                                 float teacher_scale, const float *lse, const float *dloss, float dscale, const umap_rows *dh,
                                 const umap_rows *dtable, bool accumulate, void *workspace, hipStream_t s);

}  // namespace ul
