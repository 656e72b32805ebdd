// kernels_rows.hip -- rows of a table by id, times a scale (umap_rows.h).
//
// Bound by memory: each row is read once and written once, and nothing is computed but
// the product.  A thread takes vectors of V columns, 8 or (where a side is fp32, so that a
// lane's 16 bytes lie next to its neighbours') 4; rows that end inside a vector have
// their last vector start at cols - V, where it writes some columns a second time with
// the same values.
//
// us per call and TB/s of what is read and written, one copy reaching 6.3 TB/s: 131,072 rows of
// 1,024 bf16 58 (9.3: frequent rows come from the caches), 32,768 x 4096 63 (8.4) from one set of
// ids, 72 with new ones at each call; 70,000 x 300 fp16 into fp32 19; one row 2 us of device
// time in a call of 6.
#include "launch_sizes.hpp"
#include "rows_device.hpp"

namespace ul {

namespace {

constexpr int kThreads = 256;

// What a block does: rows_per_block rows of vpr vectors, or (segments > 1) one of the
// segments of kThreads * U vectors of one row.
struct LookupPlan {
    int32_t vpr;
    int32_t rows_per_block;
    int32_t segments;
    uint32_t inv_vpr;   // ceil(2^20 / vpr): i / vpr = i * inv_vpr >> 20 for i < 2^10, vpr <= 2^10
};

template <int TI, int TO, int V, int U>
__global__ __launch_bounds__(kThreads) void k_rows_lookup(umap_rows table, RowIds ids, float scale, umap_rows out,
                                                          LookupPlan plan)
{
    const int64_t b = row_block();
    int64_t first = b * plan.rows_per_block;
    int v0 = 0;
    if (plan.segments > 1) {
        first = b / plan.segments;
        v0 = (int)(b - first * plan.segments) * (kThreads * U);
    }
    if (first >= out.rows) return;
    const int here = plan.segments > 1 ? min(plan.vpr - v0, kThreads * U)
                                       : (int)min((int64_t)plan.rows_per_block, out.rows - first) * plan.vpr;
    int64_t t[U], v[U];
    int c[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = u * kThreads + threadIdx.x;
        const int row = plan.segments > 1 ? 0 : (int)((uint32_t)i * plan.inv_vpr >> 20);
        c[u] = min((v0 + i - row * plan.vpr) * V, table.cols - V);
        t[u] = first + row;
        v[u] = i < here ? row_of(ids, t[u], table.rows) : -1;
    }
    Raw<TI, V> r[U];
    float lo[U], hi[U];   // scales of the vector's first and last column
    const Elem<TI> *const T = static_cast<const Elem<TI> *>(table.data);
    constexpr bool kScaled = TI == UMAP_I8 || TI == UMAP_F8;
    const int groups = table.group ? (table.cols + table.group - 1) / table.group : 1;
    const int shift = table.group ? 31 - __builtin_clz(table.group) : 31;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        lo[u] = hi[u] = 0.0f;
        if (v[u] < 0) continue;
        r[u] = load_raw<TI, V>(T + v[u] * table.stride + c[u]);
        if constexpr (kScaled) {
            lo[u] = table.scales[v[u] * groups + (c[u] >> shift)];
            hi[u] = table.scales[v[u] * groups + ((c[u] + V - 1) >> shift)];
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (u * kThreads + (int)threadIdx.x >= here) continue;
        float x[V] = {};
        if (v[u] >= 0) {
            floats_of<TI, V>(r[u], x);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if constexpr (kScaled) x[i] *= (c[u] + i) >> shift == c[u] >> shift ? lo[u] : hi[u];
                x[i] *= scale;
            }
        }
        store_once<TO, V>(static_cast<Elem<TO> *>(out.data) + t[u] * out.stride + c[u], raw_of<TO, V>(x));
    }
}

// Rows of fewer than 8 columns: a thread per element.
template <int TI, int TO>
__global__ __launch_bounds__(kThreads) void k_rows_lookup_narrow(umap_rows table, RowIds ids, float scale, umap_rows out)
{
    const int64_t i = row_block() * kThreads + threadIdx.x, t = i / out.cols;
    if (t >= out.rows) return;
    const int c = (int)(i - t * out.cols);
    const int64_t v = row_of(ids, t, table.rows);
    float x = 0.0f;
    if (v >= 0) {
        x = elem_float<TI>(static_cast<const Elem<TI> *>(table.data)[v * table.stride + c]);
        if (table.scales) x *= table.scales[v];   // one group
        x *= scale;
    }
    static_cast<Elem<TO> *>(out.data)[t * out.stride + c] = float_elem<TO>(x);
}

dim3 grid_of(int64_t blocks)
{
    const Grid2 g = grid2(blocks, kThreads);
    return dim3(g.x, g.y);
}

template <int TI, int TO, int V, int U>
hipError_t lookup_u(const umap_rows &table, RowIds ids, float scale, const umap_rows &out, hipStream_t s)
{
    LookupPlan plan;
    plan.vpr = (out.cols + V - 1) / V;
    plan.segments = (plan.vpr + kThreads * U - 1) / (kThreads * U);
    plan.rows_per_block = plan.segments > 1 ? 1 : kThreads * U / plan.vpr;
    plan.inv_vpr = ((1u << 20) + plan.vpr - 1) / plan.vpr;
    const int64_t blocks = plan.segments > 1 ? out.rows * plan.segments
                                             : (out.rows + plan.rows_per_block - 1) / plan.rows_per_block;
    hipLaunchKernelGGL((k_rows_lookup<TI, TO, V, U>), grid_of(blocks), dim3(kThreads), 0, s, table, ids, scale, out, plan);
    return hipGetLastError();
}

template <int TI, int TO>
hipError_t lookup(const umap_rows &table, RowIds ids, float scale, const umap_rows &out, hipStream_t s)
{
    if (out.cols < 8) {
        hipLaunchKernelGGL((k_rows_lookup_narrow<TI, TO>), grid_of((out.rows * out.cols + kThreads - 1) / kThreads),
                           dim3(kThreads), 0, s, table, ids, scale, out);
        return hipGetLastError();
    }
    constexpr int V = TI == UMAP_F32 || TO == UMAP_F32 ? 4 : 8;
    if (out.rows * ((out.cols + V - 1) / V) >= (int64_t)1 << 20) return lookup_u<TI, TO, V, 4>(table, ids, scale, out, s);
    return lookup_u<TI, TO, V, 1>(table, ids, scale, out, s);
}

template <int TI>
hipError_t lookup_from(const umap_rows &table, RowIds ids, float scale, const umap_rows &out, hipStream_t s)
{
    switch (out.type) {
    case UMAP_F32: return lookup<TI, UMAP_F32>(table, ids, scale, out, s);
    case UMAP_F16: return lookup<TI, UMAP_F16>(table, ids, scale, out, s);
    default: return lookup<TI, UMAP_BF16>(table, ids, scale, out, s);
    }
}

}  // namespace

hipError_t launch_rows_lookup(const umap_rows &table, RowIds ids, float scale, const umap_rows &out, hipStream_t s)
{
    switch (table.type) {
    case UMAP_F32: return lookup_from<UMAP_F32>(table, ids, scale, out, s);
    case UMAP_F16: return lookup_from<UMAP_F16>(table, ids, scale, out, s);
    case UMAP_BF16: return lookup_from<UMAP_BF16>(table, ids, scale, out, s);
    case UMAP_I8: return lookup_from<UMAP_I8>(table, ids, scale, out, s);
    default: return lookup_from<UMAP_F8>(table, ids, scale, out, s);
    }
}

}  // namespace ul
