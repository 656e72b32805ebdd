// kernels_rows.hip -- rows of a table by id, and the root-mean-square norm of rows
// with its gradient (umap_rows.h).
#include "launch_sizes.hpp"
#include "rows_device.hpp"
#include "rows_internal.hpp"

namespace ul {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ int64_t block_id() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

__device__ __forceinline__ float block_sum(float v, float *lds)
{
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    float sum = 0.0f;
    for (int w = 0; w < kThreads / 64; ++w) sum += lds[w];
    return sum;
}
__device__ __forceinline__ float block_max(float v, float *lds)
{
    for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    float m = 0.0f;
    for (int w = 0; w < kThreads / 64; ++w) m = fmaxf(m, lds[w]);
    return m;
}

__global__ __launch_bounds__(kThreads) void k_rows_lookup(umap_rows table, RowIds ids, float scale, umap_rows out)
{
    const int64_t t = block_id();
    if (t >= out.rows) return;
    const int64_t v = row_of(ids.data, ids.bytes, t, table.rows);
    const int64_t groups = table.group ? (table.cols + table.group - 1) / table.group : 1;
    for (int c = threadIdx.x; c < out.cols; c += kThreads) {
        float x = 0.0f;
        if (v >= 0) {
            x = load_elem(table.data, table.type, v * table.stride + c);
            if (table.scales) x *= table.scales[v * groups + (table.group ? c / table.group : 0)];
            x *= scale;
        }
        store_elem(out.data, out.type, t * out.stride + c, x);
    }
}

// 1 / sqrt(mean of the squares of row[0 .. cols) + eps).  Squares whose sum leaves
// fp32's range are formed again from values scaled down by 2^-80.
__device__ float row_rho(const float *row, int cols, float eps, float *lds)
{
    float sum = 0.0f;
    for (int c = threadIdx.x; c < cols; c += kThreads) sum += row[c] * row[c];
    sum = block_sum(sum, lds);
    if (sum < __builtin_inff()) return 1.0f / sqrtf(sum / (float)cols + eps);
    const float down = 0x1p-80f;
    sum = 0.0f;
    for (int c = threadIdx.x; c < cols; c += kThreads) sum += (row[c] * down) * (row[c] * down);
    sum = block_sum(sum, lds);
    return down / sqrtf(sum / (float)cols);
}

__global__ __launch_bounds__(kThreads) void k_rows_norm(umap_rows x, RowIds ids, float scale, umap_rows residual,
                                                        umap_rows h, RowWeight weight, float eps, umap_rows y)
{
    extern __shared__ float row[];
    __shared__ float lds[kThreads / 64];
    const int64_t t = block_id();
    if (t >= y.rows) return;
    const int64_t v = row_of(ids.data, ids.bytes, t, x.rows);
    const int cols = y.cols;
    for (int c = threadIdx.x; c < cols; c += kThreads) {
        float e = v >= 0 ? load_elem(x.data, x.type, v * x.stride + c) * scale : 0.0f;
        if (residual.data) e += load_elem(residual.data, residual.type, t * residual.stride + c);
        if (h.data) store_elem(h.data, h.type, t * h.stride + c, e);
        row[c] = e;
    }
    const float rho = row_rho(row, cols, eps, lds);
    for (int c = threadIdx.x; c < cols; c += kThreads) {
        float e = row[c] * rho;
        if (weight.data) e *= load_elem(weight.data, weight.type, c);
        row[c] = e;
        if (!y.scales) store_elem(y.data, y.type, t * y.stride + c, e);
    }
    if (!y.scales) return;
    __syncthreads();
    const int group = y.group ? y.group : cols, groups = (cols + group - 1) / group;
    const float most = y.type == UMAP_I8 ? 127.0f : 448.0f;
    for (int g = 0; g < groups; ++g) {
        const int end = min(cols, (g + 1) * group);
        float a = 0.0f;
        int bad = 0;
        for (int c = g * group + threadIdx.x; c < end; c += kThreads) {
            a = fmaxf(a, fabsf(row[c]));
            bad |= !(fabsf(row[c]) < __builtin_inff());
        }
        a = block_max(bad ? __builtin_inff() : a, lds);
        const bool fine = a >= 0x1p-100f && a < __builtin_inff();
        const float up = fine ? most / a : 0.0f;
        if (threadIdx.x == 0)
            y.scales[t * groups + g] = fine ? a / most : a < 1.0f ? 0.0f : __builtin_nanf("");
        for (int c = g * group + threadIdx.x; c < end; c += kThreads)
            store_elem(y.data, y.type, t * y.stride + c, fine ? fminf(fmaxf(row[c] * up, -most), most) : 0.0f);
    }
}

__global__ __launch_bounds__(kThreads) void k_rows_norm_grad(umap_rows dy, umap_rows h, umap_rows dh, RowWeight weight,
                                                             float eps, umap_rows dx, float *rhos)
{
    extern __shared__ float row[];
    __shared__ float lds[kThreads / 64];
    const int64_t t = block_id();
    if (t >= dy.rows) return;
    const int cols = dy.cols;
    for (int c = threadIdx.x; c < cols; c += kThreads) row[c] = load_elem(h.data, h.type, t * h.stride + c);
    const float rho = row_rho(row, cols, eps, lds);
    if (rhos) {   // only the norms' reciprocals
        if (threadIdx.x == 0) rhos[t] = rho;
        return;
    }
    float dot = 0.0f;
    for (int c = threadIdx.x; c < cols; c += kThreads) {
        float g = load_elem(dy.data, dy.type, t * dy.stride + c);
        if (weight.data) g *= load_elem(weight.data, weight.type, c);
        dot += g * (row[c] * rho);
    }
    dot = block_sum(dot, lds) / (float)cols;
    for (int c = threadIdx.x; c < cols; c += kThreads) {
        float g = load_elem(dy.data, dy.type, t * dy.stride + c);
        if (weight.data) g *= load_elem(weight.data, weight.type, c);
        float e = rho * (g - row[c] * rho * dot);
        if (dh.data) e += load_elem(dh.data, dh.type, t * dh.stride + c);
        store_elem(dx.data, dx.type, t * dx.stride + c, e);
    }
}

// Columns of dy h rho summed over rows block_id() * per_block ..: partial[block][c].
__global__ __launch_bounds__(kThreads) void k_rows_dweight(umap_rows dy, umap_rows h, const float *rhos,
                                                           int64_t per_block, float *partial)
{
    const int64_t first = blockIdx.x * per_block, last = min(first + per_block, dy.rows);
    for (int c = blockIdx.y * kThreads + threadIdx.x; c < dy.cols; c += gridDim.y * kThreads) {
        float sum = 0.0f;
        for (int64_t t = first; t < last; ++t)
            sum += load_elem(dy.data, dy.type, t * dy.stride + c) *
                   (load_elem(h.data, h.type, t * h.stride + c) * rhos[t]);
        partial[(int64_t)blockIdx.x * dy.cols + c] = sum;
    }
}
__global__ __launch_bounds__(kThreads) void k_rows_join(const float *partial, int64_t count, int cols, float *out)
{
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= cols) return;
    float sum = 0.0f;
    for (int64_t b = 0; b < count; ++b) sum += partial[b * cols + c];
    out[c] = sum;
}

dim3 blocks(int64_t n)
{
    const Grid2 g = grid2(n, kThreads);
    return dim3(g.x, g.y);
}

constexpr int64_t kDweightBlocks = 512;

}  // namespace

hipError_t launch_rows_lookup(const umap_rows &table, RowIds ids, float scale, const umap_rows &out, hipStream_t s)
{
    hipLaunchKernelGGL(k_rows_lookup, blocks(out.rows), dim3(kThreads), 0, s, table, ids, scale, out);
    return hipGetLastError();
}

hipError_t launch_rows_norm(const umap_rows &x, RowIds ids, float scale, const umap_rows *residual, const umap_rows *h,
                            RowWeight weight, float eps, const umap_rows &y, hipStream_t s)
{
    hipLaunchKernelGGL(k_rows_norm, blocks(y.rows), dim3(kThreads), y.cols * sizeof(float), s, x, ids, scale,
                       residual ? *residual : umap_rows{}, h ? *h : umap_rows{}, weight, eps, y);
    return hipGetLastError();
}

int64_t rows_norm_grad_bytes(int64_t n, int32_t cols)
{
    return (n * 4 + 15) / 16 * 16 + kDweightBlocks * cols * 4;
}

hipError_t launch_rows_norm_grad(const umap_rows &dy, const umap_rows &h, const umap_rows *dh, RowWeight weight,
                                 float eps, const umap_rows &dx, float *dweight, void *workspace, hipStream_t s)
{
    const int64_t n = dy.rows;
    float *rhos = static_cast<float *>(workspace), *partial = rhos + (n + 3) / 4 * 4;
    auto rows = [&](float *to) {
        hipLaunchKernelGGL(k_rows_norm_grad, blocks(n), dim3(kThreads), dy.cols * sizeof(float), s, dy, h,
                           dh ? *dh : umap_rows{}, weight, eps, dx, to);
        return hipGetLastError();
    };
    if (dweight) {   // first: dx may take dy's place
        const int64_t per_block = (n + kDweightBlocks - 1) / kDweightBlocks;
        const int64_t count = per_block ? (n + per_block - 1) / per_block : 0;
        const unsigned across = (dy.cols + kThreads - 1) / kThreads;
        if (count) {
            if (hipError_t e = rows(rhos)) return e;
            hipLaunchKernelGGL(k_rows_dweight, dim3((unsigned)count, across), dim3(kThreads), 0, s, dy, h, rhos, per_block,
                               partial);
            if (hipError_t e = hipGetLastError()) return e;
        }
        hipLaunchKernelGGL(k_rows_join, dim3(across), dim3(kThreads), 0, s, partial, count, dy.cols, dweight);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return n > 0 ? rows(nullptr) : hipSuccess;
}

}  // namespace ul
