// rows_device.hpp -- element types and vectors of elements of the token-row kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "rows_internal.hpp"

namespace ul {

__device__ __forceinline__ int64_t row_block() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// Row of id t, or -1 where it lies outside [0, rows).
__device__ __forceinline__ int64_t row_of(const RowIds &ids, int64_t t, int64_t rows)
{
    const int64_t v = ids.bytes == 4   ? (int64_t)static_cast<const int32_t *>(ids.data)[t]
                      : ids.bytes == 8 ? static_cast<const int64_t *>(ids.data)[t]
                                       : t;
    return v >= 0 && v < rows ? v : -1;
}

template <int T>
struct ElemOf;
template <>
struct ElemOf<UMAP_F32> { using type = float; };
template <>
struct ElemOf<UMAP_F16> { using type = _Float16; };
template <>
struct ElemOf<UMAP_BF16> { using type = uint16_t; };
template <>
struct ElemOf<UMAP_I8> { using type = int8_t; };
template <>
struct ElemOf<UMAP_F8> { using type = uint8_t; };
template <int T>
using Elem = typename ElemOf<T>::type;

template <int T>
__device__ __forceinline__ float elem_float(Elem<T> e)
{
    if constexpr (T == UMAP_BF16) return __uint_as_float((uint32_t)e << 16);
    else if constexpr (T == UMAP_F8) return __builtin_amdgcn_cvt_f32_fp8(e, 0);
    else return (float)e;
}
// To nearest even.  8-bit values come in range, UMAP_I8 ones as whole numbers.
template <int T>
__device__ __forceinline__ Elem<T> float_elem(float v)
{
    if constexpr (T == UMAP_BF16) return __builtin_bit_cast(uint16_t, (__bf16)v);
    else if constexpr (T == UMAP_F8) return (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(v, v, 0, false);
    else return (Elem<T>)v;
}

// V elements as they lie in memory, in 32-bit words where they fill some.  Rows may start
// at any element, so the loads and stores promise no more than its alignment; they are
// full-width ones all the same (dword accesses need no alignment on this architecture).
template <int T, int V>
struct Raw {
    static constexpr bool kWhole = V * sizeof(Elem<T>) % 4 == 0;
    using Unit = std::conditional_t<kWhole, uint32_t, Elem<T>>;
    static constexpr int kUnits = V * sizeof(Elem<T>) / sizeof(Unit);
    Unit w[kUnits];
};
template <int T, int V>
struct __attribute__((packed)) Packed {
    typename Raw<T, V>::Unit w[Raw<T, V>::kUnits];
};

template <int T, int V>
__device__ __forceinline__ Raw<T, V> load_raw(const Elem<T> *p)
{
    const Packed<T, V> m = *reinterpret_cast<const Packed<T, V> *>(p);
    Raw<T, V> r;
#pragma unroll
    for (int i = 0; i < Raw<T, V>::kUnits; ++i) r.w[i] = m.w[i];
    return r;
}
template <int T, int V>
__device__ __forceinline__ void store_raw(Elem<T> *p, const Raw<T, V> &r)
{
    Packed<T, V> m;
#pragma unroll
    for (int i = 0; i < Raw<T, V>::kUnits; ++i) m.w[i] = r.w[i];
    *reinterpret_cast<Packed<T, V> *>(p) = m;
}

// Likewise, for what is not needed again before much else has gone by: the caches give it up
// first, which leaves them to the rows that are (a table's frequent ones, what the next kernel
// reads).  us per call, plain / so: 32,768 x 4096 bf16 looked up 82 / 75, 70,000 x 300 into fp32 30 /
// 20, norm of 32,768 x 4096 into int8 and back 244 / 219, its gradient 194 / 173, gradient of 131,072 x
// 2048 359 / 341.  A lookup, norm and gradient one after the other on the same rows: 8 MB of them
// 14.9 / 13.3, 34 MB 42.8 / 45.2, 67 MB 79.7 / 81.2 (the caches would hold those), 134 MB 168 / 150.  Stores gain by
// 16 bytes only (8-bit rows, written by 8: 209 / 220), loads by 8 too.  Vectors of 32 bytes, fp32's 8 columns,
// go plainly: as two of 16 they lose (70,000 x 784 into fp8 55 / 59, gradient of 200,000 x 300 152 /
// 177, of 65,536 x 1024 149 / 160; of 16,384 x 4096 155 / 153).
template <int T, int V>
__device__ __forceinline__ void store_once(Elem<T> *p, const Raw<T, V> &r)
{
    if constexpr (sizeof(Raw<T, V>) == 16) {
        typedef uint32_t Words __attribute__((ext_vector_type(4), aligned(1)));
        __builtin_nontemporal_store(__builtin_bit_cast(Words, r), reinterpret_cast<Words *>(p));
    } else {
        store_raw<T, V>(p, r);
    }
}
template <int T, int V>
__device__ __forceinline__ Raw<T, V> load_once(const Elem<T> *p)
{
    if constexpr (sizeof(Raw<T, V>) == 16) {
        typedef uint32_t Words __attribute__((ext_vector_type(4), aligned(1)));
        return __builtin_bit_cast(Raw<T, V>, __builtin_nontemporal_load(reinterpret_cast<const Words *>(p)));
    } else if constexpr (sizeof(Raw<T, V>) == 8) {
        typedef uint32_t Words __attribute__((ext_vector_type(2), aligned(1)));
        return __builtin_bit_cast(Raw<T, V>, __builtin_nontemporal_load(reinterpret_cast<const Words *>(p)));
    } else {
        return load_raw<T, V>(p);
    }
}

template <int T, int V>
__device__ __forceinline__ void floats_of(const Raw<T, V> &r, float v[V])
{
    if constexpr (!Raw<T, V>::kWhole) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = elem_float<T>(r.w[i]);
    } else if constexpr (T == UMAP_F32) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = __uint_as_float(r.w[i]);
    } else if constexpr (T == UMAP_F16) {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            v[2 * i] = (float)__builtin_bit_cast(_Float16, (uint16_t)r.w[i]);
            v[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(r.w[i] >> 16));
        }
    } else if constexpr (T == UMAP_BF16) {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            v[2 * i] = __uint_as_float(r.w[i] << 16);
            v[2 * i + 1] = __uint_as_float(r.w[i] & 0xffff0000u);
        }
    } else if constexpr (T == UMAP_I8) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (float)(int8_t)(r.w[i >> 2] >> (8 * (i & 3)));
    } else {
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(r.w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(r.w[i], true);
            v[4 * i] = lo[0];
            v[4 * i + 1] = lo[1];
            v[4 * i + 2] = hi[0];
            v[4 * i + 3] = hi[1];
        }
    }
}

template <int T, int V>
__device__ __forceinline__ Raw<T, V> raw_of(const float v[V])
{
    Raw<T, V> r;
    if constexpr (!Raw<T, V>::kWhole) {
#pragma unroll
        for (int i = 0; i < V; ++i) r.w[i] = float_elem<T>(v[i]);
    } else if constexpr (T == UMAP_F32) {
#pragma unroll
        for (int i = 0; i < V; ++i) r.w[i] = __float_as_uint(v[i]);
    } else if constexpr (T == UMAP_F16) {
        typedef _Float16 half2v __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < V / 2; ++i)
            r.w[i] = __builtin_bit_cast(uint32_t, half2v{(_Float16)v[2 * i], (_Float16)v[2 * i + 1]});
    } else if constexpr (T == UMAP_BF16) {
        typedef __bf16 bf2v __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < V / 2; ++i)
            r.w[i] = __builtin_bit_cast(uint32_t, bf2v{(__bf16)v[2 * i], (__bf16)v[2 * i + 1]});
    } else if constexpr (T == UMAP_I8) {
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
            uint32_t w = 0;
#pragma unroll
            for (int j = 3; j >= 0; --j) w = w << 8 | ((uint32_t)(int)v[4 * i + j] & 0xff);
            r.w[i] = w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
            int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
            r.w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], w, true);
        }
    }
    return r;
}

}  // namespace ul
