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

}  // namespace ul
