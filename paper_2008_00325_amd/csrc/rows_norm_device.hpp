// rows_norm_device.hpp -- how the kernels of the norms lay rows out over lanes, waves and
// workgroups, and what they share.
#pragma once

#include <algorithm>

#include "launch_sizes.hpp"
#include "rows_device.hpp"

namespace ul {

// Lane exchanges inside rows of 16 lanes, without LDS.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;

template <int CTRL>
__device__ __forceinline__ float add_dpp(float v)
{
    return v + __uint_as_float(dpp<CTRL>(__float_as_uint(v)));
}
// Sum over 8, 16, 32 or 64 neighbouring lanes.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v)
{
    v = add_dpp<kXor1>(v);
    v = add_dpp<kXor2>(v);
    v = add_dpp<kHalfMirror>(v);
    if constexpr (LANES >= 16) v = add_dpp<kMirror>(v);
    if constexpr (LANES >= 32) v += __shfl_xor(v, 16);
    if constexpr (LANES >= 64) v += __shfl_xor(v, 32);
    return v;
}

// A row that belongs to a workgroup, not to lanes of a wave.
constexpr int kBlock = 0;

// Whether a sum of squares lost its value to fp32's range: too large, or so small that
// squares vanished and eps does not outweigh them.  Then the row is taken times
// range_step(sum), a power of two.  The smallest rows, one subnormal value of 2^-149 in 32,768
// columns, so get a mean square of 2^-125, still an ordinary number, as the hardware's root needs
// it; the largest of those below 2^-62, sum or eps, one of 2^126.
constexpr float kSmallSum = 0x1p-62f;
__device__ __forceinline__ bool out_of_range(float sum, float eps)
{
    return !(sum < __builtin_inff()) || (sum < kSmallSum && eps < kSmallSum);
}
__device__ __forceinline__ float range_step(float sum) { return sum < 1.0f ? 0x1p94f : 0x1p-80f; }

// Vector i of a thread: columns c = V (thread + i TPR) .. c + V - 1.  Where the row ends inside
// it, the vector is taken from column cols - V on instead, and its first `dup` columns
// are another vector's too: they count in no sum, and are written with the same values.
template <int V>
struct Cols {
    int at;    // first column
    int dup;   // V and more: past the row
    __device__ __forceinline__ Cols(int c, int cols) : at(min(c, cols - V)), dup(c - at) {}
    __device__ __forceinline__ bool live() const { return dup < V; }
    __device__ __forceinline__ bool counts(int j) const { return j >= dup; }
    __device__ __forceinline__ bool shared() const { return dup > 0 && dup < V; }
};

template <int T>
__device__ __forceinline__ const Elem<T> *row_ptr(const umap_rows &m, int64_t t)
{
    return static_cast<const Elem<T> *>(m.data) + t * m.stride;
}
template <int T>
__device__ __forceinline__ Elem<T> *row_out(const umap_rows &m, int64_t t)
{
    return static_cast<Elem<T> *>(m.data) + t * m.stride;
}

template <int V>
__device__ __forceinline__ void load_weight(const RowWeight &weight, int c, float w[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] = 1.0f;
    if (!weight.data) return;
    switch (weight.type) {
    case UMAP_F32: floats_of<UMAP_F32, V>(load_raw<UMAP_F32, V>(static_cast<const float *>(weight.data) + c), w); break;
    case UMAP_F16: floats_of<UMAP_F16, V>(load_raw<UMAP_F16, V>(static_cast<const _Float16 *>(weight.data) + c), w); break;
    default: floats_of<UMAP_BF16, V>(load_raw<UMAP_BF16, V>(static_cast<const uint16_t *>(weight.data) + c), w); break;
    }
}

// LANES lanes of a wave per row, 256 / LANES rows to a workgroup of 256, or a row per
// workgroup of any number of waves.
template <int LANES>
constexpr int kMostThreads = LANES ? 256 : 1024;
template <int LANES>
constexpr int kRowsPerBlock = LANES ? 256 / (LANES ? LANES : 1) : 1;
template <int LANES>
__device__ __forceinline__ int row_threads() { return LANES ? LANES : (int)blockDim.x; }
template <int LANES>
__device__ __forceinline__ int row_in_block()
{
    if constexpr (LANES == kBlock) return 0;
    else if constexpr (LANES == 64) return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    else return threadIdx.x / LANES;
}


// How rows lie in workgroups: threads and rows of one.
struct RowShape {
    int threads;
    int rows;
};
constexpr int kOneThread = -1;
// Lanes of a wave while two vectors per lane hold the row, else a workgroup of as many
// waves as VEC vectors per thread take: one up to `one` columns, two up to 16,384, then
// four; one thread below 8 columns.
template <template <int, int> class Launch, typename... Args>
auto by_cols(int cols, int one, Args... args)
{
    const int vectors = (cols + 7) / 8;
    auto waves = [&](int vec) { return RowShape{64 * ((vectors + 64 * vec - 1) / (64 * vec)), 1}; };
    if (cols < 8) return Launch<kOneThread, 1>::go(RowShape{256, 256}, args...);
    if (cols <= 64) return Launch<8, 1>::go(RowShape{256, 32}, args...);
    if (cols <= 128) return Launch<16, 1>::go(RowShape{256, 16}, args...);
    if (cols <= 256) return Launch<32, 1>::go(RowShape{256, 8}, args...);
    if (cols <= 512) return Launch<64, 1>::go(RowShape{256, 4}, args...);
    if (cols <= 1024) return Launch<64, 2>::go(RowShape{256, 4}, args...);
    if (cols <= one) return Launch<kBlock, 1>::go(waves(1), args...);
    if (cols <= 16384) return Launch<kBlock, 2>::go(waves(2), args...);
    return Launch<kBlock, 4>::go(waves(4), args...);
}

// Where every workgroup ends with a sum to hand over: as many as the card holds at once
// (`waves` of them on a CU), all with the same number of rows, give or take one.
inline int64_t even_grid(int64_t work, int threads, int waves)
{
    const int64_t most = 256 * std::max(1, waves * 64 / threads);
    const int64_t turns = (work + most - 1) / most;
    return (work + turns - 1) / turns;
}

}  // namespace ul
