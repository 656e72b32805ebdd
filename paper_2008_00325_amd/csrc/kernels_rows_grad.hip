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

constexpr int kThreads = 256;
constexpr int kItems = 16;
constexpr int kTile = kThreads * kItems;
constexpr int kWaves = kThreads / 64;
constexpr int kMaxDigit = 9;   // bits

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

// ---- sums of equal keys' rows ----
//
// The sorted positions are cut into chunks of equal length, so that a wave's work does
// not depend on how often an id occurs; a wave adds the rows of one chunk for one slab of
// 64 VEC columns.  An id whose positions all lie in the chunk is done then; of one that
// crosses a border the chunk leaves its part, in slot 0 where the id began in an earlier
// chunk, else in slot 1, and k_join_parts adds the parts in order.
constexpr int kMostChunk = 64;   // a lane for each position
constexpr uint32_t kNoKey = 0xffffffffu;

// VEC elements of a row as they lie in memory.
template <int T, int VEC>
struct __attribute__((packed)) Vec {
    Elem<T> e[VEC];
};
template <int T, int VEC>
__device__ __forceinline__ Vec<T, VEC> load_vec(const Elem<T> *p)
{
    return *reinterpret_cast<const Vec<T, VEC> *>(p);
}

// Columns of a lane: VEC from `at` on, the first `dup` of which are another lane's (the
// row ends inside the vector, which then lies at its end); dup >= VEC: none.
template <int VEC>
struct VecCols {
    int at, dup;
    __device__ __forceinline__ VecCols(int c, int cols) : at(max(0, min(c, cols - VEC))), dup(c - at) {}
    __device__ __forceinline__ bool live() const { return dup < VEC; }
};

template <int TG, int VEC>
__device__ __forceinline__ void store_sums(const umap_rows &grad, int64_t row, const VecCols<VEC> &c, const float sum[VEC],
                                           float scale, bool accumulate)
{
    if (!c.live()) return;
    Elem<TG> *const to = static_cast<Elem<TG> *>(grad.data) + row * grad.stride + c.at;
    Vec<TG, VEC> v;
    if (accumulate) {
        v = load_vec<TG, VEC>(to);
#pragma unroll
        for (int j = 0; j < VEC; ++j) v.e[j] = float_elem<TG>(fmaf(scale, sum[j], elem_float<TG>(v.e[j])));
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) v.e[j] = float_elem<TG>(scale * sum[j]);
    }
    if (!c.dup) {
        *reinterpret_cast<Vec<TG, VEC> *>(to) = v;
    } else {
#pragma unroll
        for (int j = 1; j < VEC; ++j)
            if (j >= c.dup) to[j] = v.e[j];
    }
}

struct Sorted {
    const uint32_t *keys, *pos;
    int64_t n;
    int32_t chunk;
};

constexpr int kZeroRows = 16;   // rows that a wave looks up and clears

template <int TD, int TG, int VEC>
__global__ __launch_bounds__(kThreads) void k_chunk_sums(Sorted sorted, int slabs, umap_rows dout, float scale,
                                                         umap_rows grad, bool accumulate, float *parts,
                                                         int64_t chunk_blocks)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t block = row_block();
    if (block >= chunk_blocks) {   // rows that no id points at
        const int64_t first = ((block - chunk_blocks) * kWaves + wave) * kZeroRows;
        const int64_t v = first + (lane & (kZeroRows - 1));
        bool clear = v < grad.rows;
        if (clear) {
            int64_t lo = 0, hi = sorted.n;   // first position with a key >= v
            while (lo < hi) {
                const int64_t mid = (lo + hi) / 2;
                if (sorted.keys[mid] < (uint32_t)v) lo = mid + 1;
                else hi = mid;
            }
            clear = lo == sorted.n || sorted.keys[lo] != (uint32_t)v;
        }
        uint64_t rows = __ballot(clear) & ((1ull << kZeroRows) - 1);
        const float zero[VEC] = {};
        for (; rows; rows &= rows - 1) {
            const int64_t row = first + __builtin_ctzll(rows);
            for (int s = 0; s < slabs; ++s)
                store_sums<TG, VEC>(grad, row, VecCols<VEC>((s * 64 + lane) * VEC, grad.cols), zero, 0.0f, false);
        }
        return;
    }
    const int64_t unit = block * kWaves + wave, chunk = unit / slabs;
    const int slab = (int)(unit - chunk * slabs);
    const int64_t p0 = chunk * sorted.chunk;
    if (p0 >= sorted.n) return;
    const int64_t p = p0 + lane;
    const bool mine = lane < sorted.chunk && p < sorted.n;
    const uint32_t key = mine ? sorted.keys[p] : kNoKey;
    const uint32_t next = mine && p + 1 < sorted.n ? sorted.keys[p + 1] : kNoKey;
    const uint32_t from = mine ? sorted.pos[p] : 0;
    const uint32_t before = p0 > 0 ? sorted.keys[p0 - 1] : kNoKey;
    const int count = __popcll(__ballot(mine && key < (uint32_t)grad.rows));   // positions without a row come last
    if (count == 0) return;
    const uint64_t ends = __ballot(key != next);
    bool open = before == (uint32_t)__builtin_amdgcn_readfirstlane(key);   // the id began in an earlier chunk
    const VecCols<VEC> cols((slab * 64 + lane) * VEC, grad.cols);
    const Elem<TD> *const base = static_cast<const Elem<TD> *>(dout.data);
    float *const part = parts + chunk * 2 * grad.cols;
    float sum[VEC] = {};
    auto leave = [&](int slot) {
        float *const to = part + (int64_t)slot * grad.cols + cols.at;
        if (cols.live()) {
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (j >= cols.dup) to[j] = sum[j];
        }
    };
    constexpr int kAhead = 8;
    for (int i0 = 0; i0 < count; i0 += kAhead) {
        Vec<TD, VEC> row[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (i0 + u < count && cols.live())
                row[u] = load_vec<TD, VEC>(base + (int64_t)(uint32_t)__builtin_amdgcn_readlane(from, i0 + u) * dout.stride + cols.at);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int i = i0 + u;
            if (i >= count) break;
#pragma unroll
            for (int j = 0; j < VEC; ++j) sum[j] += elem_float<TD>(row[u].e[j]);
            if (ends >> i & 1) {
                if (open) leave(0);
                else store_sums<TG, VEC>(grad, (uint32_t)__builtin_amdgcn_readlane(key, i), cols, sum, scale, accumulate);
                open = false;
#pragma unroll
                for (int j = 0; j < VEC; ++j) sum[j] = 0.0f;
            }
        }
    }
    if (!(ends >> (count - 1) & 1)) leave(open ? 0 : 1);
}

// The ids that cross a chunk's end and begin in it: slot 1 of the chunk and slot 0 of those
// that follow.  1,024 columns to a workgroup of 1,024 threads, a quarter of the parts to
// each 256 of them; the quarters are added in order.
constexpr int kJoinThreads = 1024, kJoinCols = 1024;

template <int TG>
__global__ __launch_bounds__(kJoinThreads) void k_join_parts(Sorted sorted, float scale, umap_rows grad, bool accumulate,
                                                             const float *parts)
{
    __shared__ float quarter[3][kJoinCols];
    const int64_t chunk = row_block(), p0 = chunk * sorted.chunk, p1 = p0 + sorted.chunk;
    if (p1 >= sorted.n) return;
    const uint32_t key = sorted.keys[p1 - 1];
    if (key >= (uint32_t)grad.rows || sorted.keys[p1] != key || (p0 > 0 && sorted.keys[p0 - 1] == key)) return;
    // the chunks after this one that begin with the key
    const int lane = threadIdx.x & 63;
    int64_t more = 0;
    for (;;) {
        const int64_t p = (chunk + 1 + more + lane) * sorted.chunk;
        const uint64_t same = __ballot(p < sorted.n && sorted.keys[p] == key);
        const int here = ~same ? __builtin_ctzll(~same) : 64;
        more += here;
        if (here < 64) break;
    }
    const int q = threadIdx.x >> 8, cols = grad.cols;
    const int64_t each = (more + 3) / 4, first = min(each * q, more), last = min(first + each, more);
    for (int c0 = blockIdx.z * kJoinCols; c0 < cols; c0 += gridDim.z * kJoinCols) {
        float sum[4] = {};
        const float *const at = parts + (chunk + 1) * 2 * cols;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = c0 + j * 256 + (threadIdx.x & 255);
            if (c >= cols) continue;
            if (q == 0) sum[j] = parts[(chunk * 2 + 1) * cols + c];
#pragma unroll 4
            for (int64_t m = first; m < last; ++m) sum[j] += at[m * 2 * cols + c];
            if (q > 0) quarter[q - 1][j * 256 + (threadIdx.x & 255)] = sum[j];
        }
        __syncthreads();
        if (q == 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int i = j * 256 + (int)threadIdx.x, c = c0 + i;
                if (c >= cols) continue;
                const float total = scale * (((sum[j] + quarter[0][i]) + quarter[1][i]) + quarter[2][i]);
                Elem<TG> *const to = static_cast<Elem<TG> *>(grad.data) + (int64_t)key * grad.stride + c;
                *to = float_elem<TG>(accumulate ? elem_float<TG>(*to) + total : total);
            }
        }
        __syncthreads();
    }
}

int64_t align16(int64_t bytes) { return (bytes + 15) / 16 * 16; }
int64_t tile_count(int64_t n) { return (n + kTile - 1) / kTile; }

// Columns per lane: as many as leave no lane of a wave without any.
int vec_for(int cols) { return cols <= 64 ? 1 : cols <= 128 ? 2 : cols <= 256 ? 4 : 8; }

// Positions per chunk: about 8,192 waves where there are enough of them.
struct ChunkPlan {
    int32_t slabs, chunk;
    int64_t chunks;
    ChunkPlan(int64_t n, int32_t cols)
    {
        const int width = 64 * vec_for(cols);
        slabs = (cols + width - 1) / width;
        chunk = kMostChunk;
        while (chunk > 8 && (n + chunk - 1) / chunk * slabs < 8192) chunk /= 2;
        chunks = (n + chunk - 1) / chunk;
    }
};

struct Workspace {
    int64_t sorted, counts, parts, bytes;
    Workspace(int64_t n, int32_t cols)
    {
        const ChunkPlan plan(n, cols);
        sorted = align16(n * 4);
        counts = 4 * sorted;
        parts = counts + align16(tile_count(n) * (4 << kMaxDigit));
        bytes = parts + align16(plan.chunks * 2 * cols * 4) + 16;
    }
};

template <int TD, int TG, int VEC>
hipError_t sum_chunks(const Sorted &sorted, const ChunkPlan &plan, const umap_rows &dout, float scale,
                      const umap_rows &grad, bool accumulate, float *parts, hipStream_t s)
{
    const int64_t chunk_blocks = (plan.chunks * plan.slabs + kWaves - 1) / kWaves;
    const int64_t zero_blocks = accumulate ? 0 : (grad.rows + kZeroRows * kWaves - 1) / (kZeroRows * kWaves);
    const Grid2 g = grid2(chunk_blocks + zero_blocks, kThreads);
    hipLaunchKernelGGL((k_chunk_sums<TD, TG, VEC>), dim3(g.x, g.y), dim3(kThreads), 0, s, sorted, plan.slabs, dout,
                       scale, grad, accumulate, parts, chunk_blocks);
    if (hipError_t e = hipGetLastError()) return e;
    if (plan.chunks < 2) return hipSuccess;
    const Grid2 j = grid2(plan.chunks, kJoinThreads);
    const int across = (grad.cols + kJoinCols - 1) / kJoinCols;
    hipLaunchKernelGGL((k_join_parts<TG>), dim3(j.x, j.y, across < 16 ? across : 16), dim3(kJoinThreads), 0, s, sorted,
                       scale, grad, accumulate, parts);
    return hipGetLastError();
}

template <int TD, int TG>
hipError_t sum_by_cols(const Sorted &sorted, const ChunkPlan &plan, const umap_rows &dout, float scale,
                       const umap_rows &grad, bool accumulate, float *parts, hipStream_t s)
{
    switch (vec_for(grad.cols)) {
    case 1: return sum_chunks<TD, TG, 1>(sorted, plan, dout, scale, grad, accumulate, parts, s);
    case 2: return sum_chunks<TD, TG, 2>(sorted, plan, dout, scale, grad, accumulate, parts, s);
    case 4: return sum_chunks<TD, TG, 4>(sorted, plan, dout, scale, grad, accumulate, parts, s);
    default: return sum_chunks<TD, TG, 8>(sorted, plan, dout, scale, grad, accumulate, parts, s);
    }
}

template <int TD>
hipError_t sum_into(const Sorted &sorted, const ChunkPlan &plan, const umap_rows &dout, float scale,
                    const umap_rows &grad, bool accumulate, float *parts, hipStream_t s)
{
    switch (grad.type) {
    case UMAP_F32: return sum_by_cols<TD, UMAP_F32>(sorted, plan, dout, scale, grad, accumulate, parts, s);
    case UMAP_F16: return sum_by_cols<TD, UMAP_F16>(sorted, plan, dout, scale, grad, accumulate, parts, s);
    default: return sum_by_cols<TD, UMAP_BF16>(sorted, plan, dout, scale, grad, accumulate, parts, s);
    }
}

}  // namespace

int64_t rows_lookup_grad_bytes(int64_t n, int64_t rows, int32_t cols)
{
    (void)rows;
    return Workspace(n, cols).bytes;
}

hipError_t launch_rows_lookup_grad(const umap_rows &dout, RowIds ids, float scale, const umap_rows &grad,
                                   bool accumulate, void *workspace, hipStream_t s)
{
    const int64_t n = dout.rows;
    const Workspace at(n, grad.cols);
    char *w = static_cast<char *>(workspace);
    uint32_t *buf[4], *counts = reinterpret_cast<uint32_t *>(w + at.counts);
    for (int i = 0; i < 4; ++i) buf[i] = reinterpret_cast<uint32_t *>(w + i * at.sorted);
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
    const ChunkPlan plan(n, grad.cols);
    const Sorted sorted{keys, pos, n, plan.chunk};
    float *const parts = reinterpret_cast<float *>(w + at.parts);
    switch (dout.type) {
    case UMAP_F32: return sum_into<UMAP_F32>(sorted, plan, dout, scale, grad, accumulate, parts, s);
    case UMAP_F16: return sum_into<UMAP_F16>(sorted, plan, dout, scale, grad, accumulate, parts, s);
    default: return sum_into<UMAP_BF16>(sorted, plan, dout, scale, grad, accumulate, parts, s);
    }
}

}  // namespace ul
