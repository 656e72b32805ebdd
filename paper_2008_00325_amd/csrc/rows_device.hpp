// rows_device.hpp -- element types and row helpers of the token-row kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "umap_rows.h"

namespace ul {

// Element `i` of an array of type `type` as fp32 (8-bit values without their scale).
__device__ __forceinline__ float load_elem(const void *p, int32_t type, int64_t i)
{
    switch (type) {
    case UMAP_F32: return static_cast<const float *>(p)[i];
    case UMAP_F16: return (float)static_cast<const _Float16 *>(p)[i];
    case UMAP_BF16: return __uint_as_float((uint32_t)static_cast<const uint16_t *>(p)[i] << 16);
    case UMAP_I8: return (float)static_cast<const int8_t *>(p)[i];
    default: return __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t *>(p)[i], 0);
    }
}

// Rounds to nearest even; 8-bit values come in range.
__device__ __forceinline__ void store_elem(void *p, int32_t type, int64_t i, float v)
{
    switch (type) {
    case UMAP_F32: static_cast<float *>(p)[i] = v; break;
    case UMAP_F16: static_cast<_Float16 *>(p)[i] = (_Float16)v; break;
    case UMAP_BF16: static_cast<__bf16 *>(p)[i] = (__bf16)v; break;
    case UMAP_I8: static_cast<int8_t *>(p)[i] = (int8_t)rintf(v); break;
    default: static_cast<uint8_t *>(p)[i] = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(v, v, 0, false); break;
    }
}

// Row of id t, or -1 where it lies outside [0, rows).
__device__ __forceinline__ int64_t row_of(const void *ids, int32_t bytes, int64_t t, int64_t rows)
{
    const int64_t v = bytes == 4 ? (int64_t)static_cast<const int32_t *>(ids)[t] : bytes == 8 ? static_cast<const int64_t *>(ids)[t] : t;
    return v >= 0 && v < rows ? v : -1;
}

}  // namespace ul
