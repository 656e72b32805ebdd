// kernels_rows_grad.hip -- gradient of a lookup by sorted ids (umap_rows.h):
// grad[v] = scale * sum over the t with ids[t] = v of dout[t].
//
// The positions t are sorted by id, stably (least significant digit first), so the
// rows that belong to one table row lie one after the other, in the order of t, and
// are added in that order: the same sum in every call, without atomics.
#include "launch_sizes.hpp"
#include "rows_device.hpp"
#include "rows_internal.hpp"

namespace ul {

namespace {

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

constexpr int kThreads = 256;
constexpr int kItems = 16;
constexpr int kTile = kThreads * kItems;
constexpr int kWaves = kThreads / 64;
constexpr int kMaxDigit = 9;   // bits

__device__ __forceinline__ int64_t block_id() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// The sort's key of position t: its table row, or `rows` where it has none.
struct Keys {
    const uint32_t *keys;   // null: from the ids
    RowIds ids;
    int64_t rows;
    __device__ __forceinline__ uint32_t operator()(int64_t t) const
    {
        if (keys) return keys[t];
        const int64_t v = row_of(ids, t, rows);
        return v < 0 ? (uint32_t)rows : (uint32_t)v;
    }
};

// counts[digit * tiles + tile]: keys of the tile with that digit.
__global__ __launch_bounds__(kThreads) void k_digit_counts(Keys keys, int64_t n, int shift, int bits, uint32_t *counts)
{
    __shared__ uint32_t bin[1 << kMaxDigit];
    const int bins = 1 << bits;
    const uint32_t mask = bins - 1;
    for (int d = threadIdx.x; d < bins; d += kThreads) bin[d] = 0;
    __syncthreads();
    for (int i = 0; i < kItems; ++i) {
        const int64_t t = (int64_t)blockIdx.x * kTile + i * kThreads + threadIdx.x;
        if (t < n) atomicAdd(&bin[(keys(t) >> shift) & mask], 1u);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < bins; d += kThreads) counts[(int64_t)d * gridDim.x + blockIdx.x] = bin[d];
}

// Exclusive prefix sums of counts[0 .. size), in place, by one workgroup.
constexpr int kScanThreads = 1024;
__global__ __launch_bounds__(kScanThreads) void k_scan(uint32_t *counts, int64_t size)
{
    __shared__ uint32_t part[kScanThreads / 64];
    uint32_t carry = 0;
    for (int64_t base = 0; base < size; base += kScanThreads) {
        const int64_t i = base + threadIdx.x;
        const uint32_t own = i < size ? counts[i] : 0;
        uint32_t sum = own;
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t up = __shfl_up(sum, o);
            if ((threadIdx.x & 63) >= o) sum += up;
        }
        if ((threadIdx.x & 63) == 63) part[threadIdx.x >> 6] = sum;
        __syncthreads();
        uint32_t before = 0, all = 0;
        for (int w = 0; w < kScanThreads / 64; ++w) {
            if (w < (int)(threadIdx.x >> 6)) before += part[w];
            all += part[w];
        }
        if (i < size) counts[i] = carry + before + sum - own;
        carry += all;
        __syncthreads();
    }
}

// Files the tile's keys and positions behind the counts' prefix sums, in their order:
// wave w has positions w * 64 kItems .. of the tile, 64 at a time, and among
// equal digits a lane comes after the lower lanes and the wave's earlier steps.
__global__ __launch_bounds__(kThreads) void k_file(Keys keys, const uint32_t *from, int64_t n, int shift, int bits,
                                                   const uint32_t *counts, uint32_t *keys_out, uint32_t *pos_out)
{
    __shared__ volatile uint32_t seen[kWaves][1 << kMaxDigit];
    const int bins = 1 << bits, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const uint32_t mask = bins - 1;
    for (int i = threadIdx.x; i < kWaves * bins; i += kThreads) seen[i / bins][i % bins] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * kTile + wave * 64 * kItems + lane;
    uint32_t key[kItems], rank[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const int64_t t = first + i * 64;
        key[i] = t < n ? keys(t) : 0;
        const uint32_t d = (key[i] >> shift) & mask;
        unsigned long long same = __ballot(t < n);
        for (int b = 0; b < bits; ++b) {
            const bool on = (d >> b) & 1;
            const unsigned long long with = __ballot(on);
            same &= on ? with : ~with;
        }
        const uint32_t before = seen[wave][d];
        const uint32_t lower = __popcll(same & ((1ull << lane) - 1));
        rank[i] = before + lower;
        __builtin_amdgcn_wave_barrier();
        if (t < n && lower == 0) seen[wave][d] = before + (uint32_t)__popcll(same);
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    for (int d = threadIdx.x; d < bins; d += kThreads) {
        uint32_t at = counts[(int64_t)d * gridDim.x + blockIdx.x];
        for (int w = 0; w < kWaves; ++w) {
            const uint32_t c = seen[w][d];
            seen[w][d] = at;
            at += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const int64_t t = first + i * 64;
        if (t >= n) continue;
        const uint32_t at = seen[wave][(key[i] >> shift) & mask] + rank[i];
        keys_out[at] = key[i];
        pos_out[at] = from ? from[t] : (uint32_t)t;
    }
}

// One wave per table row and 64 columns.
__global__ __launch_bounds__(kThreads) void k_row_sums(const uint32_t *keys, const uint32_t *pos, umap_rows dout,
                                                       float scale, umap_rows grad, bool accumulate)
{
    const int64_t v = block_id() * kWaves + (threadIdx.x >> 6);
    if (v >= grad.rows) return;
    int64_t lo = 0, hi = dout.rows;   // first position with a key >= v
    while (lo < hi) {
        const int64_t mid = (lo + hi) / 2;
        if (keys[mid] < (uint32_t)v) lo = mid + 1;
        else hi = mid;
    }
    const bool any = lo < dout.rows && keys[lo] == (uint32_t)v;
    if (!any && accumulate) return;
    for (int c = threadIdx.x & 63; c < grad.cols; c += 64) {
        float sum = 0.0f;
        for (int64_t p = lo; p < dout.rows && keys[p] == (uint32_t)v; ++p)
            sum += load_elem(dout.data, dout.type, (int64_t)pos[p] * dout.stride + c);
        sum *= scale;
        if (accumulate) sum += load_elem(grad.data, grad.type, v * grad.stride + c);
        store_elem(grad.data, grad.type, v * grad.stride + c, sum);
    }
}

int64_t align16(int64_t bytes) { return (bytes + 15) / 16 * 16; }
int64_t tile_count(int64_t n) { return (n + kTile - 1) / kTile; }

}  // namespace

// Keys and positions, twice (a pass goes from one pair to the other), and the counts.
int64_t rows_lookup_grad_bytes(int64_t n, int64_t rows, int32_t cols)
{
    (void)rows;
    (void)cols;
    return 16 + 4 * align16(n * 4) + align16(tile_count(n) * (4 << kMaxDigit));
}

hipError_t launch_rows_lookup_grad(const umap_rows &dout, RowIds ids, float scale, const umap_rows &grad,
                                   bool accumulate, void *workspace, hipStream_t s)
{
    const int64_t n = dout.rows;
    char *w = static_cast<char *>(workspace);
    uint32_t *buf[4], *counts;
    for (int i = 0; i < 4; ++i) buf[i] = reinterpret_cast<uint32_t *>(w + i * align16(n * 4));
    counts = reinterpret_cast<uint32_t *>(w + 4 * align16(n * 4));
    const uint32_t *keys = nullptr, *pos = nullptr;
    const unsigned tiles = (unsigned)tile_count(n);
    int key_bits = 1;
    while ((grad.rows >> key_bits) != 0) ++key_bits;   // keys 0 .. rows
    const int passes = (key_bits + kMaxDigit - 1) / kMaxDigit, bits = (key_bits + passes - 1) / passes;
    for (int pass = 0; n > 0 && pass < passes; ++pass) {
        const Keys from{keys, ids, grad.rows};
        uint32_t *keys_out = buf[2 * (pass & 1)], *pos_out = buf[2 * (pass & 1) + 1];
        hipLaunchKernelGGL(k_digit_counts, dim3(tiles), dim3(kThreads), 0, s, from, n, pass * bits, bits, counts);
        if (hipError_t e = hipGetLastError()) return e;
        hipLaunchKernelGGL(k_scan, dim3(1), dim3(kScanThreads), 0, s, counts, (int64_t)tiles << bits);
        if (hipError_t e = hipGetLastError()) return e;
        hipLaunchKernelGGL(k_file, dim3(tiles), dim3(kThreads), 0, s, from, pos, n, pass * bits, bits, counts, keys_out,
                           pos_out);
        if (hipError_t e = hipGetLastError()) return e;
        keys = keys_out;
        pos = pos_out;
    }
    const Grid2 g = grid2((grad.rows + kWaves - 1) / kWaves, kThreads);
    hipLaunchKernelGGL(k_row_sums, dim3(g.x, g.y), dim3(kThreads), 0, s, keys, pos, dout, scale, grad, accumulate);
    return hipGetLastError();
}

}  // namespace ul
