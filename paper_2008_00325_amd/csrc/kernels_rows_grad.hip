// kernels_rows_grad.hip -- gradient of a lookup by sorted ids (umap_rows.h):
// grad[v] = scale * sum over the t with ids[t] = v of dout[t].
//
// The positions t are sorted by id, stably (least significant digit first), so the
// rows that belong to one table row lie one after the other, in the order of t, and
// are added in that order: the same sum in every call, without atomics.
//
// Bound by memory: every row of dout is read once and every row of grad written once, by
// waves that all have the same number of rows however often an id occurs; the sort (of 4-byte
// keys and positions) and the joins are latency, launch by launch.  Sums are fp32, rounded
// once.  us per call: 131,072 bf16 rows into fp32 128,000 x 2048 338 (1.58 GB, 251 us at a
// copy's rate: sums and zeros 287, sort 32, joins 19), 8,192 into 32,000 x 1024 40 (0.15 GB, 24: sort
// and zeros 27, sums 9, joins 6), 77 into 2,000 x 64 14 (three launches).
#include <algorithm>

#include "launch_sizes.hpp"
#include "rows_device.hpp"
#include "rows_internal.hpp"

namespace ul {

namespace {
constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// ---- the sort ----
//
// Least significant digit first, up to 9 bits at a time.  A tile of 1,024 ITEMS keys belongs to
// a workgroup: a launch counts the tile's digits, another files its keys behind those
// of the tiles before.  Up to 8,192 keys one workgroup does all of it in one launch.
// What bounds it is latency, launch by launch.
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kMaxDigit = 9;   // bits
constexpr int kMaxBins = 1 << kMaxDigit;

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

// counts[tile][digit]: keys of the tile with that digit.  The first pass also clears the
// number of joins.
template <int ITEMS>
__global__ __launch_bounds__(kSortThreads) void k_digit_counts(Keys keys, int64_t n, int shift, int bits,
                                                               uint32_t *counts, uint32_t *joins)
{
    __shared__ uint32_t bin[kMaxBins];
    const int bins = 1 << bits;
    const uint32_t mask = bins - 1;
    const int64_t first = (int64_t)blockIdx.x * (kSortThreads * ITEMS) + threadIdx.x;
    uint32_t key[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
        if (first + i * kSortThreads < n) key[i] = keys(first + i * kSortThreads);
    for (int d = threadIdx.x; d < bins; d += kSortThreads) bin[d] = 0;
    if (joins && blockIdx.x == 0 && threadIdx.x == 0) *joins = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
        if (first + i * kSortThreads < n) atomicAdd(&bin[(key[i] >> shift) & mask], 1u);
    __syncthreads();
    for (int d = threadIdx.x; d < bins; d += kSortThreads) counts[(int64_t)blockIdx.x * bins + d] = bin[d];
}

// Many tiles: counts[tile][d] becomes the number in the tiles before, counts[tiles][d] that in
// all of them.  A thread per digit.
__global__ __launch_bounds__(64) void k_tile_sums(uint32_t *counts, int64_t tiles, int bins)
{
    const int d = blockIdx.x * 64 + threadIdx.x;
    if (d >= bins) return;
    uint32_t sum = 0;
    constexpr int kAhead = 16;
    for (int64_t t0 = 0; t0 < tiles; t0 += kAhead) {
        uint32_t c[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) c[u] = t0 + u < tiles ? counts[(t0 + u) * bins + d] : 0;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (t0 + u < tiles) counts[(t0 + u) * bins + d] = sum;
            sum += c[u];
        }
    }
    counts[tiles * bins + d] = sum;
}

struct SortLds {
    uint32_t seen[kSortWaves][kMaxBins];
    uint32_t wave_total[kSortWaves];
};

// Ranks of a tile's keys: wave w has positions 64 ITEMS w .. of the tile, 64 at a time, and
// among equal digits a key comes after those of lower lanes, of the wave's earlier steps
// and of lower waves.  `there`: how many of the thread's keys exist.
template <int ITEMS>
__device__ __forceinline__ void rank_in_wave(const uint32_t key[ITEMS], int there, int shift, uint32_t mask, SortLds &lds,
                                             uint32_t rank[ITEMS])
{
    volatile uint32_t *const seen = lds.seen[threadIdx.x >> 6];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const uint32_t d = (key[i] >> shift) & mask;
        // the lanes with this digit: those that agree in every bit
        const uint64_t any = __ballot(i < there);
        uint32_t lo = (uint32_t)any, hi = (uint32_t)(any >> 32);
#pragma unroll
        for (int b = 0; b < kMaxDigit; ++b) {
            const int32_t on = (int32_t)(d << (31 - b)) >> 31;   // the bit, 32 times
            const uint64_t with = __ballot(on < 0);
            lo &= ~((uint32_t)with ^ (uint32_t)on);
            hi &= ~((uint32_t)(with >> 32) ^ (uint32_t)on);
        }
        const uint64_t same = (uint64_t)hi << 32 | lo;
        const uint32_t before = seen[d];
        const uint32_t lower = __builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0));   // of them, below this one
        rank[i] = before + lower;
        __builtin_amdgcn_wave_barrier();
        if (i < there && lower == 0) seen[d] = before + (uint32_t)__popcll(same);
        __builtin_amdgcn_wave_barrier();
    }
}

// Exclusive prefix sums over the digits of all[threadIdx.x]; a barrier's work.
__device__ __forceinline__ uint32_t digit_start(uint32_t all, SortLds &lds)
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    uint32_t up = all;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t v = __shfl_up(up, o);
        if (lane >= o) up += v;
    }
    if (lane == 63) lds.wave_total[wave] = up;
    __syncthreads();
    up -= all;
    for (int w = 0; w < wave && w < kMaxBins / 64; ++w) up += lds.wave_total[w];
    return up;
}

// The waves' counts of a digit, and their sum; then where each wave's keys of it start.
__device__ __forceinline__ uint32_t counts_of(int d, const SortLds &lds, uint32_t c[kSortWaves])
{
    uint32_t all = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) c[w] = lds.seen[w][d];
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) all += c[w];
    return all;
}
__device__ __forceinline__ void starts_of(int d, uint32_t at, const uint32_t c[kSortWaves], SortLds &lds)
{
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
        lds.seen[w][d] = at;
        at += c[w];
    }
}

// Files the tile's keys and positions where their digit's turn is.  SUMMED: k_tile_sums
// has run; else each workgroup adds up the tiles' counts itself.
template <int ITEMS, bool SUMMED>
__global__ __launch_bounds__(kSortThreads) void k_file(Keys keys, const uint32_t *from, int64_t n, int shift, int bits,
                                                       const uint32_t *counts, int tiles, uint32_t *keys_out,
                                                       uint32_t *pos_out)
{
    __shared__ SortLds lds;
    const int bins = 1 << bits, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const uint32_t mask = bins - 1;
    const int64_t first = (int64_t)blockIdx.x * (kSortThreads * ITEMS) + wave * 64 * ITEMS + lane;
    uint32_t key[ITEMS], pos[ITEMS], rank[ITEMS];
    int there = 0;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int64_t t = first + i * 64;
        key[i] = t < n ? keys(t) : 0;
        pos[i] = from && t < n ? from[t] : (uint32_t)t;
        there += t < n;
    }
    // this thread's digit: its keys in the tiles before this one, and in all
    uint32_t mine = 0, all = 0;
    const int d = threadIdx.x;
    if (d < bins) {
        if constexpr (SUMMED) {
            mine = counts[(int64_t)blockIdx.x * bins + d];
            all = counts[(int64_t)tiles * bins + d];
        } else {
#pragma unroll 16
            for (int t = 0; t < tiles; ++t) {
                const uint32_t c = counts[t * bins + d];
                all += c;
                mine += t < (int)blockIdx.x ? c : 0;
            }
        }
    }
    for (int i = lane; i < bins; i += 64) lds.seen[wave][i] = 0;
    __builtin_amdgcn_wave_barrier();
    rank_in_wave<ITEMS>(key, there, shift, mask, lds, rank);
    const uint32_t at = digit_start(all, lds) + mine;   // behind its barrier all waves have counted
    if (d < bins) {
        uint32_t c[kSortWaves];
        counts_of(d, lds, c);
        starts_of(d, at, c, lds);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        if (i >= there) continue;
        const uint32_t to = lds.seen[wave][(key[i] >> shift) & mask] + rank[i];
        keys_out[to] = key[i];
        pos_out[to] = pos[i];
    }
}

// Zeros for a row by `lanes` lanes of which this is number `lane`.
__device__ __forceinline__ void clear_row(const umap_rows &grad, int bytes_per, int64_t row, int lane, int lanes)
{
    const int bytes = grad.cols * bytes_per;
    char *const to = static_cast<char *>(grad.data) + row * grad.stride * bytes_per;
    if (bytes >= 16) {   // the last 16 bytes may be written twice
        const Raw<UMAP_F32, 4> zero{};
        for (int b = lane * 16; b < bytes; b += lanes * 16) {
            float *const at = reinterpret_cast<float *>(to + min(b, bytes - 16));
            if (lanes == 64) store_once<UMAP_F32, 4>(at, zero);
            else store_raw<UMAP_F32, 4>(at, zero);   // neighbours of one lane meet in the cache
        }
    } else {
        for (int b = lane * 2; b < bytes; b += lanes * 2) *reinterpret_cast<uint16_t *>(to + b) = 0;
    }
}

// Rows that no id points at, where the ids are few: a workgroup marks the ids of its stretch
// of rows in LDS, then clears the others.  The sort beside it takes one CU.
constexpr int kMostMarked = 32768;
__device__ __forceinline__ void clear_unmarked(const Keys &keys, int n, const umap_rows &grad, int bytes_per, int64_t first,
                                               int rows)
{
    __shared__ uint32_t marked[kMostMarked / 32];
    for (int i = threadIdx.x; i < (rows + 31) / 32; i += kSortThreads) marked[i] = 0;
    __syncthreads();
    for (int t = threadIdx.x; t < n; t += kSortThreads) {
        const int64_t r = (int64_t)keys(t) - first;
        if (r >= 0 && r < rows) atomicOr(&marked[r >> 5], 1u << (r & 31));
    }
    __syncthreads();
    for (int r = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); r < rows; r += kSortWaves)
        if (!(marked[r >> 5] >> (r & 31) & 1) && first + r < grad.rows) clear_row(grad, bytes_per, first + r, threadIdx.x & 63, 64);
}

// The whole sort of up to 1,024 ITEMS keys by one workgroup; the others clear stretches of
// clear_rows rows.
template <int ITEMS>
__global__ __launch_bounds__(kSortThreads) void k_sort_few(Keys keys, int n, int passes, int bits, uint32_t *keys_out,
                                                           uint32_t *pos_out, uint32_t *joins, umap_rows grad,
                                                           int bytes_per, int clear_rows)
{
    if (blockIdx.x > 0) {
        clear_unmarked(keys, n, grad, bytes_per, (int64_t)(blockIdx.x - 1) * clear_rows, clear_rows);
        return;
    }
    __shared__ SortLds lds;
    __shared__ uint32_t key_at[kSortThreads * ITEMS];
    __shared__ uint16_t pos_at[kSortThreads * ITEMS];
    const int bins = 1 << bits, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const uint32_t mask = bins - 1;
    const int first = wave * 64 * ITEMS + lane;
    uint32_t key[ITEMS], pos[ITEMS], rank[ITEMS];
    int there = 0;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int t = first + i * 64;
        key[i] = t < n ? keys(t) : 0;
        pos[i] = t;
        there += t < n;
    }
    if (threadIdx.x == 0) *joins = 0;
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = pass * bits;
        for (int i = lane; i < bins; i += 64) lds.seen[wave][i] = 0;
        __builtin_amdgcn_wave_barrier();
        rank_in_wave<ITEMS>(key, there, shift, mask, lds, rank);
        __syncthreads();
        const int d = threadIdx.x;
        uint32_t all = 0, c[kSortWaves];
        if (d < bins) all = counts_of(d, lds, c);
        const uint32_t at = digit_start(all, lds);
        if (d < bins) starts_of(d, at, c, lds);
        __syncthreads();
        const bool last = pass == passes - 1;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if (i >= there) continue;
            const uint32_t to = lds.seen[wave][(key[i] >> shift) & mask] + rank[i];
            if (last) {
                keys_out[to] = key[i];
                pos_out[to] = pos[i];
            } else {
                key_at[to] = key[i];
                pos_at[to] = (uint16_t)pos[i];
            }
        }
        if (last) break;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if (i >= there) continue;
            key[i] = key_at[first + i * 64];
            pos[i] = pos_at[first + i * 64];
        }
    }
}

// ---- sums of equal keys' rows ----
//
// The sorted positions are cut into chunks of equal length, so that the work does not
// depend on how often an id occurs; a wave (LANES lanes of it for narrow rows) adds the
// rows of one chunk for one slab of LANES VEC columns.  An id that begins in a chunk and
// ends in it or in the next one is the chunk's own.  Of a longer one each chunk leaves its
// part, in slot 1 where the id begins, else in slot 0, and k_join_parts adds the parts in
// order.
constexpr uint32_t kNoKey = 0xffffffffu;

// Columns of a lane: VEC from `at` on, the first `dup` of which are another lane's (the
// row ends inside the vector, which then lies at its end); dup >= VEC: none.
template <int VEC>
struct VecCols {
    int at, dup;
    __device__ __forceinline__ VecCols(int c, int cols) : at(min(c, cols - VEC)), dup(c - at) {}   // cols >= VEC
    __device__ __forceinline__ bool live() const { return dup < VEC; }
};

template <int TG, int VEC>
__device__ __forceinline__ void store_sums(const umap_rows &grad, int64_t row, const VecCols<VEC> &c, const float sum[VEC],
                                           float scale, bool accumulate)
{
    if (!c.live()) return;
    Elem<TG> *const to = static_cast<Elem<TG> *>(grad.data) + row * grad.stride + c.at;
    float v[VEC];
    if (accumulate) {
        floats_of<TG, VEC>(load_raw<TG, VEC>(to), v);
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[j] = fmaf(scale, sum[j], v[j]);
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[j] = scale * sum[j];
    }
    if (!c.dup) {
        store_raw<TG, VEC>(to, raw_of<TG, VEC>(v));
    } else {
#pragma unroll
        for (int j = 1; j < VEC; ++j)
            if (j >= c.dup) to[j] = float_elem<TG>(v[j]);
    }
}

struct Sorted {
    const uint32_t *keys, *pos;
    int64_t n;
    int32_t chunk;
};
// Chunks in which an id that needs joining begins.
struct Joins {
    uint32_t *count, *chunks;
};

// LANES lanes that work on one chunk: all values below are the same in each of them.
template <int LANES>
struct Group {
    int base = threadIdx.x & 63 & ~(LANES - 1);
    __device__ __forceinline__ uint64_t ballot(bool v) const
    {
        const uint64_t all = __ballot(v);
        if constexpr (LANES == 64) return all;
        else return all >> base & ((1ull << LANES) - 1);
    }
    __device__ __forceinline__ uint32_t at(uint32_t v, int i) const
    {
        if constexpr (LANES == 64) return (uint32_t)__builtin_amdgcn_readlane((int)v, i);
        else return (uint32_t)__shfl((int)v, base + i);
    }
};

// The keys and rows of a chunk, one to a lane.
template <int LANES>
struct Chunk {
    uint32_t key, from;
    int count;        // positions that have a row (those without come last)
    uint64_t ends;    // positions that are their key's last
    __device__ __forceinline__ Chunk(const Sorted &sorted, int64_t p0, int64_t rows, const Group<LANES> &group)
    {
        const int lane = threadIdx.x & (LANES - 1);
        const int64_t p = p0 + lane;
        const bool mine = lane < sorted.chunk && p < sorted.n;
        key = mine ? sorted.keys[p] : kNoKey;
        from = mine ? sorted.pos[p] : 0;
        const uint32_t next = mine && p + 1 < sorted.n ? sorted.keys[p + 1] : kNoKey;
        count = __popcll(group.ballot(mine && key < (uint32_t)rows));
        ends = group.ballot(mine && key != next);
    }
};

// Rows that a wave looks up and clears: some 64 KB of them, at most one to a lane.
__host__ __device__ inline int rows_to_clear(int row_bytes)
{
    int rows = 64;
    while (rows > 8 && (int64_t)rows * row_bytes > 65536) rows /= 2;
    return rows;
}

template <int TD, int TG, int LANES, int VEC, int PARTS>
__global__ __launch_bounds__(kThreads) void k_chunk_sums(Sorted sorted, int slabs, umap_rows dout, float scale,
                                                         umap_rows grad, bool accumulate, float *parts, Joins joins,
                                                         int64_t chunk_blocks)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t block = row_block();
    if (block >= chunk_blocks) {   // rows that no id points at
        const int per_wave = rows_to_clear(grad.cols * sizeof(Elem<TG>));
        const int64_t first = ((block - chunk_blocks) * kWaves + wave) * per_wave;
        const int64_t v = first + lane;
        bool clear = lane < per_wave && v < grad.rows;
        if (clear) {
            int64_t lo = 0, hi = sorted.n;   // first position with a key >= v
            while (lo < hi) {
                const int64_t mid = (lo + hi) / 2;
                if (sorted.keys[mid] < (uint32_t)v) lo = mid + 1;
                else hi = mid;
            }
            clear = lo == sorted.n || sorted.keys[lo] != (uint32_t)v;
        }
        if (per_wave == 64) {   // narrow rows: a lane clears its own
            if (clear) clear_row(grad, sizeof(Elem<TG>), v, 0, 1);
        } else {
            for (uint64_t rows = __ballot(clear); rows; rows &= rows - 1)
                clear_row(grad, sizeof(Elem<TG>), first + __builtin_ctzll(rows), lane, 64);
        }
        return;
    }
    const Group<LANES> group;
    int64_t unit = block * kWaves + wave;
    if constexpr (LANES < 64) unit = unit * (64 / LANES) + lane / LANES;
    const int64_t chunk = unit / slabs;
    const int slab = (int)(unit - chunk * slabs);
    const int64_t p0 = chunk * sorted.chunk;
    if (p0 >= sorted.n) return;
    const Chunk<LANES> here(sorted, p0, grad.rows, group);
    if (here.count == 0) return;
    const Chunk<LANES> next(sorted, p0 + sorted.chunk, grad.rows, group);
    const uint32_t first_key = group.at(here.key, 0);
    // the chunk's first id may have begun before it: in the last chunk (then that one has
    // all of it, if it ends here), or earlier
    bool open = p0 > 0 && sorted.keys[p0 - 1] == first_key;
    int begin = 0;
    if (open && here.ends && (p0 == sorted.chunk || sorted.keys[p0 - sorted.chunk - 1] != first_key)) {
        begin = __builtin_ctzll(here.ends) + 1;
        open = false;
    }
    const int me = threadIdx.x & (LANES - 1);
    auto cols = [&](int h) { return VecCols<VEC>(((slab * PARTS + h) * LANES + me) * VEC, grad.cols); };
    const Elem<TD> *const base = static_cast<const Elem<TD> *>(dout.data);
    float sum[PARTS][VEC] = {};
    auto leave = [&](int slot) {
        float *const to = parts + (chunk * 2 + slot) * grad.cols;
#pragma unroll
        for (int h = 0; h < PARTS; ++h) {
            const VecCols<VEC> c = cols(h);
            if (!c.live()) continue;
            if (!c.dup) {
                store_raw<UMAP_F32, VEC>(to + c.at, raw_of<UMAP_F32, VEC>(sum[h]));
            } else {
#pragma unroll
                for (int j = 1; j < VEC; ++j)
                    if (j >= c.dup) to[c.at + j] = sum[h][j];
            }
        }
    };
    // rows in flight while those before them are added (us per call with 4 / 6 / 8 rows of 16-bit
    // types: 131,072 x 2048 into 128,000 rows 351 / 346 / 341, 65,536 x 2048 135 / 127 / 123; with 8 / 16: 343 /
    // 339, 32,768 x 4096 194 / 189, 300 columns 87 / 84; 70,000 x 784 fp32 with 4 / 8 120 / 117; more gives
    // nothing)
    constexpr int kAhead = PARTS * VEC * sizeof(Elem<TD>) > 16 ? 8 : 16;
    struct Row {
        Raw<TD, VEC> part[PARTS];
    };
    auto add = [&](const Chunk<LANES> &of, int i0, int end) {
        Row row[kAhead], ahead[kAhead];
        auto read = [&](int from, Row to[kAhead]) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (from + u >= end) break;
                const Elem<TD> *const at = base + (int64_t)group.at(of.from, from + u) * dout.stride;   // by all lanes
#pragma unroll
                for (int h = 0; h < PARTS; ++h)
                    if (cols(h).live()) to[u].part[h] = load_once<TD, VEC>(at + cols(h).at);
            }
        };
        read(i0, row);
        for (; i0 < end; i0 += kAhead) {
            read(i0 + kAhead, ahead);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int i = i0 + u;
                if (i >= end) break;
#pragma unroll
                for (int h = 0; h < PARTS; ++h) {
                    float v[VEC];
                    floats_of<TD, VEC>(row[u].part[h], v);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) sum[h][j] += v[j];
                }
                if (of.ends >> i & 1) {
                    const uint32_t key = group.at(of.key, i);
                    if (open) leave(0);
#pragma unroll
                    for (int h = 0; h < PARTS; ++h) {
                        if (!open) store_sums<TG, VEC>(grad, key, cols(h), sum[h], scale, accumulate);
#pragma unroll
                        for (int j = 0; j < VEC; ++j) sum[h][j] = 0.0f;
                    }
                    open = false;
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) row[u] = ahead[u];
        }
    };
    add(here, begin, here.count);
    if (begin >= here.count || here.ends >> (here.count - 1) & 1) return;   // the last id ends with the chunk
    if (open) {
        leave(0);
    } else if (next.ends) {   // it ends in the next chunk
        add(next, 0, __builtin_ctzll(next.ends) + 1);
    } else {
        leave(1);
        if (slab == 0 && me == 0) joins.chunks[atomicAdd(joins.count, 1u)] = (uint32_t)chunk;
    }
}

// The ids over several chunks: slot 1 of the chunk in which one begins and slot 0 of those
// that follow.  64 VEC columns to a workgroup and a stretch of the parts to each of its waves,
// whose sums are added in order.  (The order of the list changes nothing in the sums.)
constexpr int kJoinWaves = 16;
constexpr int join_vec(int cols) { return cols >= 4 ? 4 : 1; }   // a vector's columns must exist

template <int TG, int VEC>
__global__ __launch_bounds__(64 * kJoinWaves) void k_join_parts(Sorted sorted, float scale, umap_rows grad, bool accumulate,
                                                                const float *parts, Joins joins)
{
    constexpr int kJoinCols = 64 * VEC;
    __shared__ float stretch[kJoinWaves][kJoinCols];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, cols = grad.cols;
    const uint32_t count = *joins.count;
    for (uint32_t j = blockIdx.x; j < count; j += gridDim.x) {
        const int64_t chunk = joins.chunks[j];
        const uint32_t key = sorted.keys[(chunk + 1) * sorted.chunk];
        // the chunks after this one that begin with the key
        int64_t more = 0;
        for (;;) {
            const int64_t p = (chunk + 1 + more + lane) * sorted.chunk;
            const uint64_t same = __ballot(p < sorted.n && sorted.keys[p] == key);
            const int here = ~same ? __builtin_ctzll(~same) : 64;
            more += here;
            if (here < 64) break;
        }
        const int64_t each = (more + kJoinWaves - 1) / kJoinWaves;
        const int64_t first = min(each * wave, more), last = min(first + each, more);
        for (int c0 = blockIdx.y * kJoinCols; c0 < cols; c0 += gridDim.y * kJoinCols) {
            const VecCols<VEC> c(c0 + lane * VEC, cols);
            const float *const begun = parts + (chunk * 2 + 1) * cols + c.at, *const after = parts + (chunk + 1) * 2 * cols + c.at;
            float sum[VEC] = {};
            auto add = [&](const float *p) {
                float v[VEC];
                floats_of<UMAP_F32, VEC>(load_raw<UMAP_F32, VEC>(p), v);
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum[i] += v[i];
            };
            if (wave == 0) add(begun);
#pragma unroll 16
            for (int64_t m = first; m < last; ++m) add(after + m * 2 * cols);
#pragma unroll
            for (int i = 0; i < VEC; ++i) stretch[wave][lane * VEC + i] = sum[i];
            __syncthreads();
            if (wave == 0 && c.live()) {
                float total[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    total[i] = stretch[0][lane * VEC + i];
                    for (int w = 1; w < kJoinWaves; ++w) total[i] += stretch[w][lane * VEC + i];
                }
                store_sums<TG, VEC>(grad, key, c, total, scale, accumulate);
            }
            __syncthreads();
        }
    }
}

// Up to 8,192 keys are sorted in one launch; us per call so / by tiles in four: 5,000 of 64 columns added
// to a table 24 / 33, 8,192 28 / 36, but with 16 keys per thread 16,384 45 / 39.  Then tiles of 4,096
// keys, whose workgroups add up the tiles' counts themselves, up to 256 tiles; beyond that tiles of
// 8,192, with a launch for the sums.  4,096 / 8,192 keys, 64 columns: 10,000 ids 36 / 47, 65,536 49 / 64,
// 131,072 61 / 76, 262,144 67 / 80, 524,288 94 / 103, 1,048,576 150 / 153; 700,000 of 16 columns into
// 300,000 rows 160 / 166; four million of 16 (4,096 with a launch for the sums) 812 / 752.
struct SortPlan {
    int items;   // per thread
    int64_t tiles;
    bool summed;
    explicit SortPlan(int64_t n)
    {
        summed = n > 256 * 4096;
        items = summed ? 8 : 4;
        if (few(n)) items = n <= 1024 ? 1 : n <= 4096 ? 4 : 8;
        tiles = (n + kSortThreads * items - 1) / (kSortThreads * items);
    }
    static bool few(int64_t n) { return n <= 8192; }
};

struct SortPass {
    Keys from;
    const uint32_t *pos;
    int64_t n;
    int shift, bits;
    uint32_t *counts;
    int tiles;
    uint32_t *keys_out, *pos_out, *joins;
    hipStream_t s;

    template <int ITEMS, bool SUMMED>
    hipError_t run() const
    {
        const dim3 grid((unsigned)tiles), threads(kSortThreads);
        hipLaunchKernelGGL((k_digit_counts<ITEMS>), grid, threads, 0, s, from, n, shift, bits, counts, joins);
        if (hipError_t e = hipGetLastError()) return e;
        if constexpr (SUMMED) {
            hipLaunchKernelGGL(k_tile_sums, dim3(((1u << bits) + 63) / 64), dim3(64), 0, s, counts, (int64_t)tiles, 1 << bits);
            if (hipError_t e = hipGetLastError()) return e;
        }
        hipLaunchKernelGGL((k_file<ITEMS, SUMMED>), grid, threads, 0, s, from, pos, n, shift, bits, counts, tiles,
                           keys_out, pos_out);
        return hipGetLastError();
    }
};

int64_t align16(int64_t bytes) { return (bytes + 15) / 16 * 16; }

// Lanes and columns per lane: as many columns as leave no lane of a wave without any, and
// where a wave's lanes are more than the columns, several chunks to a wave.
struct RowShape {
    int lanes, slab;   // columns of a slab
    explicit RowShape(int cols)
    {
        lanes = cols <= 16 ? 16 : cols <= 32 ? 32 : 64;
        slab = cols <= 16 ? 16 : cols <= 32 ? 32 : cols <= 64 ? 64 : cols <= 128 ? 128 : cols <= 256 ? 256 : 512;
    }
};

// Positions per chunk: 64 where that leaves 2,048 waves, else fewer.  us per call with at least
// 2,048 / 4,096 / 8,192 / 16,384 waves: 131,072 rows of 300 columns 75 / 85 / 95 / 111, of 2,048
// columns 354 / 354 / 355 / 364, 32,768 of 4,096 196 / 195 / 204 / 231, 131,072 of 1,024 with one id
// 112 / 111 / 154 / 255.
struct ChunkPlan {
    int32_t slabs, chunk;
    int64_t chunks;
    ChunkPlan(int64_t n, int32_t cols)
    {
        const RowShape shape(cols);
        slabs = (cols + shape.slab - 1) / shape.slab;
        chunk = shape.lanes;
        while (chunk > 8 && (n + chunk - 1) / chunk * slabs * shape.lanes / 64 < 2048) chunk /= 2;
        chunks = (n + chunk - 1) / chunk;
    }
};

struct Workspace {
    int64_t sorted, counts, joins, parts, bytes;
    Workspace(int64_t n, int32_t cols)
    {
        const ChunkPlan plan(n, cols);
        sorted = align16(n * 4);   // keys and positions, twice: a pass goes from one pair to the other
        counts = 4 * sorted;
        joins = counts + align16((SortPlan(n).tiles + 1) * (4 << kMaxDigit));
        parts = joins + 16 + align16(plan.chunks * 4);
        bytes = parts + align16(plan.chunks * 2 * cols * 4);
    }
};

// What the launches of one call share.
struct Call {
    Sorted sorted;
    ChunkPlan plan;
    umap_rows dout, grad;
    float scale;
    bool accumulate;
    bool cleared;   // rows without ids are zero already
    float *parts;
    Joins joins;
    hipStream_t s;
};

template <int TD, int TG, int LANES, int VEC, int PARTS = 1>
hipError_t sum_chunks(const Call &c)
{
    const int per_block = kThreads / LANES;
    const int64_t chunk_blocks = (c.plan.chunks * c.plan.slabs + per_block - 1) / per_block;
    const int64_t per_clear = (int64_t)rows_to_clear(c.grad.cols * sizeof(Elem<TG>)) * kWaves;
    const int64_t zero_blocks = c.accumulate || c.cleared ? 0 : (c.grad.rows + per_clear - 1) / per_clear;
    const Grid2 g = grid2(chunk_blocks + zero_blocks, kThreads);
    hipLaunchKernelGGL((k_chunk_sums<TD, TG, LANES, VEC, PARTS>), dim3(g.x, g.y), dim3(kThreads), 0, c.s, c.sorted, c.plan.slabs,
                       c.dout, c.scale, c.grad, c.accumulate, c.parts, c.joins, chunk_blocks);
    if (hipError_t e = hipGetLastError()) return e;
    if (c.plan.chunks < 3) return hipSuccess;   // no id needs joining
    const int join_cols = 64 * join_vec(c.grad.cols), across = (c.grad.cols + join_cols - 1) / join_cols;
    const dim3 grid((unsigned)std::min<int64_t>(c.plan.chunks, 256), std::min(across, 64)), threads(64 * kJoinWaves);
    if (join_vec(c.grad.cols) == 1)
        hipLaunchKernelGGL((k_join_parts<TG, 1>), grid, threads, 0, c.s, c.sorted, c.scale, c.grad, c.accumulate, c.parts, c.joins);
    else
        hipLaunchKernelGGL((k_join_parts<TG, 4>), grid, threads, 0, c.s, c.sorted, c.scale, c.grad, c.accumulate, c.parts, c.joins);
    return hipGetLastError();
}

template <int TD, int TG>
hipError_t sum_by_cols(const Call &c)
{
    const RowShape shape(c.grad.cols);
    // a lane's 16 bytes lie next to its neighbours': 8 columns of 16 bits, or twice 4 where a
    // side is fp32
    constexpr bool wide = TD == UMAP_F32 || TG == UMAP_F32;
    switch (shape.slab) {
    case 16: return sum_chunks<TD, TG, 16, 1>(c);
    case 32: return sum_chunks<TD, TG, 32, 1>(c);
    case 64: return sum_chunks<TD, TG, 64, 1>(c);
    case 128: return sum_chunks<TD, TG, 64, 2>(c);
    case 256: return sum_chunks<TD, TG, 64, 4>(c);
    default: return sum_chunks<TD, TG, 64, wide ? 4 : 8, wide ? 2 : 1>(c);
    }
}

template <int TD>
hipError_t sum_into(const Call &c)
{
    switch (c.grad.type) {
    case UMAP_F32: return sum_by_cols<TD, UMAP_F32>(c);
    case UMAP_F16: return sum_by_cols<TD, UMAP_F16>(c);
    default: return sum_by_cols<TD, UMAP_BF16>(c);
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
    uint32_t *const join_count = reinterpret_cast<uint32_t *>(w + at.joins);
    int key_bits = 1;
    while ((grad.rows >> key_bits) != 0) ++key_bits;   // keys 0 .. rows
    const int passes = (key_bits + kMaxDigit - 1) / kMaxDigit, bits = (key_bits + passes - 1) / passes;
    const uint32_t *keys = nullptr, *pos = nullptr;
    const SortPlan sort(n);
    if (n > 0 && SortPlan::few(n)) {
        const Keys from{nullptr, ids, grad.rows};
        // about two workgroups to a CU clear rows meanwhile
        const int clear_rows = (int)std::min<int64_t>(kMostMarked, (grad.rows + 510) / 511);
        const dim3 grid(accumulate ? 1 : 1 + (unsigned)((grad.rows + clear_rows - 1) / clear_rows)), threads(kSortThreads);
        const int bytes_per = grad.type == UMAP_F32 ? 4 : 2;
        if (sort.items == 1)
            hipLaunchKernelGGL((k_sort_few<1>), grid, threads, 0, s, from, (int)n, passes, bits, buf[0], buf[1], join_count, grad, bytes_per, clear_rows);
        else if (sort.items == 4)
            hipLaunchKernelGGL((k_sort_few<4>), grid, threads, 0, s, from, (int)n, passes, bits, buf[0], buf[1], join_count, grad, bytes_per, clear_rows);
        else
            hipLaunchKernelGGL((k_sort_few<8>), grid, threads, 0, s, from, (int)n, passes, bits, buf[0], buf[1], join_count, grad, bytes_per, clear_rows);
        if (hipError_t e = hipGetLastError()) return e;
        keys = buf[0];
        pos = buf[1];
    } else {
        for (int pass = 0; n > 0 && pass < passes; ++pass) {
            const SortPass p{Keys{keys, ids, grad.rows}, pos, n, pass * bits, bits, counts, (int)sort.tiles,
                             buf[2 * (pass & 1)], buf[2 * (pass & 1) + 1], pass ? nullptr : join_count, s};
            const hipError_t e = sort.summed ? p.run<8, true>() : p.run<4, false>();
            if (e != hipSuccess) return e;
            keys = p.keys_out;
            pos = p.pos_out;
        }
    }
    const ChunkPlan plan(n, grad.cols);
    const Call call{Sorted{keys, pos, n, plan.chunk}, plan, dout, grad, scale, accumulate, n > 0 && SortPlan::few(n),
                    reinterpret_cast<float *>(w + at.parts), Joins{join_count, join_count + 4}, s};
    switch (dout.type) {
    case UMAP_F32: return sum_into<UMAP_F32>(call);
    case UMAP_F16: return sum_into<UMAP_F16>(call);
    default: return sum_into<UMAP_BF16>(call);
    }
}

}  // namespace ul
