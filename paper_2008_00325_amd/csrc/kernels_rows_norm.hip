// kernels_rows_norm.hip -- root-mean-square norm of rows and its gradient (umap_rows.h).
//
//   norm      h = scale x + residual, rho = 1 / sqrt(mean h^2 + eps), y = h rho weight
//   gradient  dx = rho (dy weight - h rho^2 mean(dy weight h)) + dh, dweight = sum dy h rho
//
// Bound by memory: a row is read once and stays in registers between its sums and its
// result, so every input is read and every output written once.  A row belongs to some
// lanes of a wave (up to 1,024 columns) or to a workgroup, whose waves add their sums over
// LDS with one barrier; a thread holds a few vectors of its columns, and reads its share of
// the next row before it works on this one.  The gradient's workgroups stay and keep
// dweight's sums of their rows in registers or LDS; a second launch joins them in order.
// All arithmetic is fp32; h, y and dx are rounded once, on the way out.
//
// us per call and TB/s of what is read and written, one copy reaching 6.3 TB/s: 32,768 x 4096
// bf16, residual added, into bf16 h and int8 156 (6.0), gradient with upstream gradient and
// dweight 167 (6.5), the join 5 more; 131,072 x 1024 bf16 without residual 85 (6.3); 70,000 x 784
// fp32 into fp8 with a scale per 128 columns 57 (4.9).  Weaker: rows a little longer than a
// power of two vectors (300 columns into int8 4.7: 38 of 64 lanes have any), and rows that a
// workgroup's registers, 128 per thread, do not hold, part of which goes through scratch memory: all beyond
// 16,384 columns (norm 4.0 to 4.9, gradient 3.2 to 3.8, with dweight 2.0 to 2.5) and gradients from 8,193
// columns on (bf16 with dweight 4.3 to 5.0, fp32 4.5 to 4.7, with dweight 2.1 to 2.7).
#include <algorithm>

#include "launch_sizes.hpp"
#include "rows_device.hpp"

namespace ul {

namespace {

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
__device__ __forceinline__ uint32_t max_u(uint32_t a, uint32_t b) { return a > b ? a : b; }
// Largest of 4, 8, 16 or 32 neighbouring lanes.
__device__ __forceinline__ uint32_t lanes_max(uint32_t v, int lanes)
{
    v = max_u(v, dpp<kXor1>(v));
    v = max_u(v, dpp<kXor2>(v));
    if (lanes >= 8) v = max_u(v, dpp<kHalfMirror>(v));
    if (lanes >= 16) v = max_u(v, dpp<kMirror>(v));
    if (lanes >= 32) v = max_u(v, (uint32_t)__shfl_xor((int)v, 16));
    return v;
}

// Sums and maxima over a row's threads: LANES of a wave, or (kBlock) a workgroup.  Two
// buffers take turns, so that one barrier per value is enough: a buffer is written again
// only after the next value's barrier.
constexpr int kBlock = 0;
struct RowLds {
    float v[2][2][16];
};
template <int LANES>
struct RowThreads {
    RowLds *lds;
    int turn = 0;
    __device__ __forceinline__ void sum2(float &a, float &b)
    {
        a = lanes_sum<LANES ? LANES : 64>(a);
        b = lanes_sum<LANES ? LANES : 64>(b);
        if constexpr (LANES == kBlock) {
            if ((threadIdx.x & 63) == 0) {
                lds->v[turn][0][threadIdx.x >> 6] = a;
                lds->v[turn][1][threadIdx.x >> 6] = b;
            }
            __syncthreads();
            a = b = 0.0f;
            for (int w = 0; w < (int)(blockDim.x >> 6); ++w) {
                a += lds->v[turn][0][w];
                b += lds->v[turn][1][w];
            }
            turn ^= 1;
        }
    }
    __device__ __forceinline__ float sum(float a)
    {
        a = lanes_sum<LANES ? LANES : 64>(a);
        if constexpr (LANES == kBlock) {
            if ((threadIdx.x & 63) == 0) lds->v[turn][0][threadIdx.x >> 6] = a;
            __syncthreads();
            a = 0.0f;
            for (int w = 0; w < (int)(blockDim.x >> 6); ++w) a += lds->v[turn][0][w];
            turn ^= 1;
        }
        return a;
    }
    __device__ __forceinline__ uint32_t max(uint32_t a)
    {
        constexpr int kLanes = LANES ? LANES : 64;
        a = lanes_max(a, kLanes);
        if constexpr (kLanes >= 64) a = max_u(a, (uint32_t)__shfl_xor((int)a, 32));
        if constexpr (LANES == kBlock) {
            if ((threadIdx.x & 63) == 0) lds->v[turn][0][threadIdx.x >> 6] = __uint_as_float(a);
            __syncthreads();
            for (int w = 0; w < (int)(blockDim.x >> 6); ++w) a = max_u(a, __float_as_uint(lds->v[turn][0][w]));
            turn ^= 1;
        }
        return a;
    }
};

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
// Columns of the norm's vectors: 8, or 4 from fp32 to fp32, so that a lane's 16 bytes lie
// next to its neighbours' (256 MB of fp32 rows, us with 8 / 4: into fp32 300 columns 107 / 94,
// 784 100 / 93, 2,048 93 / 90, but 32,768, where registers are short, 126 / 152; into bf16 784 71
// / 72; into int8 784 67 / 75).  The gradient takes 8 (784 columns 202 / 208).
template <int TX, int TY, int VEC>
constexpr int kNormVec = TX == UMAP_F32 && TY == UMAP_F32 && VEC < 4 ? 4 : 8;
constexpr int kGradVec = 8;

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

template <int V>
__device__ __forceinline__ float square_sum(const float e[V], const Cols<V> &c)
{
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j) sum = fmaf(e[j], e[j], sum);
    if (c.shared()) {
        sum = 0.0f;
#pragma unroll
        for (int j = 0; j < V; ++j) sum = c.counts(j) ? fmaf(e[j], e[j], sum) : sum;
    }
    return c.live() ? sum : 0.0f;
}
template <int V>
__device__ __forceinline__ float product_sum(const float e[V], const float g[V], const float w[V], const Cols<V> &c)
{
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j) sum = fmaf(g[j] * w[j], e[j], sum);
    if (c.shared()) {
        sum = 0.0f;
#pragma unroll
        for (int j = 0; j < V; ++j) sum = c.counts(j) ? fmaf(g[j] * w[j], e[j], sum) : sum;
    }
    return c.live() ? sum : 0.0f;
}

// The scale of a group whose largest magnitude has these bits, and its values divided by it.
// All quotients are fp32's, to nearest even, by Markstein's method: from a reciprocal that is
// itself rounded to nearest, q = v / s with one correction by the exact remainder v - q s.  The
// scale lies between 2^-109 and 2^121, so that its reciprocal is an ordinary number (a largest
// magnitude beyond 2^126 has a subnormal one, which the hardware takes for 0).
template <int TY>
struct Quant {
    static constexpr float kMost = TY == UMAP_I8 ? 127.0f : 448.0f;
    bool fine;
    float scale, up;
    static __device__ __forceinline__ float quotient(float v, float s, float over_s)
    {
        const float q = v * over_s;
        return fmaf(fmaf(-q, s, v), over_s, q);
    }
    __device__ __forceinline__ explicit Quant(uint32_t bits)
    {
        const float m = __uint_as_float(bits);
        fine = bits >= __float_as_uint(0x1p-100f) && bits < 0x7f800000u;
        scale = fine ? quotient(m, kMost, 1.0f / kMost) : bits < 0x7f800000u ? 0.0f : __builtin_nanf("");
        const float near = __builtin_amdgcn_rcpf(scale);   // within a unit of its last place
        up = fmaf(fmaf(-near, scale, 1.0f), near, near);
    }
    // A value in its 8-bit type's range; what a group that is not fine holds is for the caller to drop.
    __device__ __forceinline__ float of(float v) const { return quotient(v, scale, up); }
    __device__ __forceinline__ float operator()(float v) const
    {
        if constexpr (TY == UMAP_I8) return fine ? rintf(of(v)) : 0.0f;
        else return fine ? of(v) : 0.0f;
    }
    // 8 of them.  UMAP_I8: adding 1.5 2^23 leaves the nearest whole number in the sum's low
    // bits.  The group's largest value is at most a unit of its last place above 127 or 448 and
    // rounds to it.
    __device__ __forceinline__ Raw<TY, 8> pack(const float v[8]) const
    {
        Raw<TY, 8> r;
        if constexpr (TY == UMAP_I8) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint32_t b[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) b[j] = __float_as_uint(of(v[4 * i + j]) + 0x1.8p23f);
                const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400), hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000c0c);
                r.w[i] = lo | hi;
            }
        } else {
            float s[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] = of(v[j]);
            r = raw_of<TY, 8>(s);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) r.w[i] = fine ? r.w[i] : 0;
        return r;
    }
};

// Bits of the largest magnitude of V values, above all finite ones where one is not finite.
template <int V>
__device__ __forceinline__ uint32_t most_bits(const float e[V], const Cols<V> &c)
{
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) most = max_u(most, __float_as_uint(e[j]) & 0x7fffffffu);
    if (c.shared()) {
        most = 0;
#pragma unroll
        for (int j = 0; j < V; ++j) most = max_u(most, c.counts(j) ? __float_as_uint(e[j]) & 0x7fffffffu : 0);
    }
    return c.live() ? most : 0;
}

// 8 VEC columns per thread; cols >= 8.  MORE: a thread keeps its weights over
// its rows and reads a row ahead.
template <int TX, int TY, int LANES, int VEC, bool MORE>
__global__ __launch_bounds__(kMostThreads<LANES>) void k_rows_norm(umap_rows x, RowIds ids, float scale, umap_rows residual,
                                                             umap_rows h, RowWeight weight, float eps, umap_rows y)
{
    constexpr int kRows = kRowsPerBlock<LANES>, V = kNormVec<TX, TY, VEC>, N = VEC * 8 / V;
    constexpr bool kEight = TY == UMAP_I8 || TY == UMAP_F8;
    __shared__ RowLds lds;
    RowThreads<LANES> row{&lds};
    const int TPR = row_threads<LANES>(), me = LANES ? threadIdx.x & (LANES - 1) : threadIdx.x, cols = y.cols;
    const float over_cols = 1.0f / (float)cols;
    float w[MORE ? N : 1][V];
    if constexpr (MORE) {
#pragma unroll
        for (int i = 0; i < N; ++i) load_weight<V>(weight, Cols<V>(V * (me + i * TPR), cols).at, w[i]);
    }
    Raw<TX, V> a[N], b[N];
    auto read = [&](int64_t t) {
        const int64_t v = row_of(ids, t, x.rows);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = Cols<V>(V * (me + i * TPR), cols).at;
            if (v >= 0) a[i] = load_once<TX, V>(row_ptr<TX>(x, v) + at);
            else a[i] = Raw<TX, V>{};   // a missing row stands for zeros
            if (residual.data) b[i] = load_once<TX, V>(row_ptr<TX>(residual, t) + at);
        }
    };
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t t = (int64_t)blockIdx.x * kRows + row_in_block<LANES>();
    if (MORE && t < y.rows) read(t);
    for (; t < y.rows; t += step) {
        if (!MORE) read(t);
        float e[N][V];
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            floats_of<TX, V>(a[i], e[i]);
            if (scale != 1.0f) {
#pragma unroll
                for (int j = 0; j < V; ++j) e[i][j] *= scale;
            }
            if (residual.data) {
                float r[V];
                floats_of<TX, V>(b[i], r);
#pragma unroll
                for (int j = 0; j < V; ++j) e[i][j] += r[j];
            }
            sum += square_sum<V>(e[i], Cols<V>(V * (me + i * TPR), cols));
        }
        if (MORE && t + step < y.rows) read(t + step);
        sum = row.sum(sum);
        if (h.data) {   // behind the sum's barrier: h may lie where other waves read
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const Cols<V> c(V * (me + i * TPR), cols);
                if (c.live()) store_once<TX, V>(row_out<TX>(h, t) + c.at, raw_of<TX, V>(e[i]));
            }
        }
        float add = eps;
        if (out_of_range(sum, eps)) {
            const float k = range_step(sum);
            sum = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
#pragma unroll
                for (int j = 0; j < V; ++j) e[i][j] *= k;
                sum += square_sum<V>(e[i], Cols<V>(V * (me + i * TPR), cols));
            }
            sum = row.sum(sum);
            add = eps * k * k;
        }
        const float rho = __builtin_amdgcn_rsqf(fmaf(sum, over_cols, add));
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (!MORE) load_weight<V>(weight, Cols<V>(V * (me + i * TPR), cols).at, w[0]);
#pragma unroll
            for (int j = 0; j < V; ++j) e[i][j] = e[i][j] * rho * w[MORE ? i : 0][j];
        }

        if constexpr (!kEight) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const Cols<V> c(V * (me + i * TPR), cols);
                if (c.live()) store_once<TY, V>(row_out<TY>(y, t) + c.at, raw_of<TY, V>(e[i]));
            }
        } else {
            // magnitudes compare as their bits do, infinities and NaN above all others
            uint32_t most[N], all = 0;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                most[i] = most_bits<V>(e[i], Cols<V>(V * (me + i * TPR), cols));
                all = max_u(all, most[i]);
            }
            if (y.group == 0) all = row.max(all);
            const int lanes = y.group / V, groups = y.group ? (cols + y.group - 1) / y.group : 1;
            float *const scales = y.scales + t * groups;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int v = me + i * TPR;
                const Cols<V> c(V * v, cols);
                const Quant<TY> quant(y.group ? lanes_max(most[i], lanes) : all);
                if (!c.live()) continue;
                if (y.group ? (v & (lanes - 1)) == 0 : v == 0) scales[y.group ? v / lanes : 0] = quant.scale;
                Elem<TY> *const to = row_out<TY>(y, t) + c.at;
                if (!c.dup) {
                    store_raw<TY, V>(to, quant.pack(e[i]));
                } else {   // only its own columns: the others may be another group's
#pragma unroll
                    for (int j = 1; j < V; ++j)
                        if (c.counts(j)) to[j] = float_elem<TY>(quant(e[i][j]));
                }
            }
        }
    }
}

template <int TX, int LANES, int VEC, bool DW, bool MORE>
__global__ __launch_bounds__(kMostThreads<LANES>) void k_rows_norm_grad(umap_rows dy, umap_rows h, umap_rows dh,
                                                                  RowWeight weight, float eps, umap_rows dx,
                                                                  float *partial)
{
    constexpr int kRows = kRowsPerBlock<LANES>, V = kGradVec, N = VEC * 8 / V;
    __shared__ RowLds lds;
    RowThreads<LANES> row{&lds};
    const int TPR = row_threads<LANES>(), me = LANES ? threadIdx.x & (LANES - 1) : threadIdx.x, cols = dy.cols;
    const float over_cols = 1.0f / (float)cols;
    // dweight's sums of this thread's columns, in LDS where registers are short
    constexpr bool kInLds = DW && LANES == kBlock && VEC > 1;
    extern __shared__ float dw_lds[];
    float w[MORE ? N : 1][V], dw[DW && !kInLds ? N : 1][V];
    auto dw_at = [&](int i, int j) -> float & { return dw_lds[(i * V + j) * TPR + me]; };
    if constexpr (MORE) {
#pragma unroll
        for (int i = 0; i < N; ++i) load_weight<V>(weight, Cols<V>(V * (me + i * TPR), cols).at, w[i]);
    }
#pragma unroll
    for (int i = 0; i < (DW ? N : 1); ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if constexpr (kInLds) dw_at(i, j) = 0.0f;
            else dw[i][j] = 0.0f;
        }
    Raw<TX, V> a[N], b[N], u[N];
    auto read = [&](int64_t t) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = Cols<V>(V * (me + i * TPR), cols).at;
            a[i] = load_once<TX, V>(row_ptr<TX>(h, t) + at);
            b[i] = load_once<TX, V>(row_ptr<TX>(dy, t) + at);
            if (dh.data) u[i] = load_once<TX, V>(row_ptr<TX>(dh, t) + at);
        }
    };
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t t = (int64_t)blockIdx.x * kRows + row_in_block<LANES>();
    if (MORE && t < dy.rows) read(t);
    for (; t < dy.rows; t += step) {
        if (!MORE) read(t);
        Raw<TX, V> ha[N], db[N], ua[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            ha[i] = a[i];
            db[i] = b[i];
            if (dh.data) ua[i] = u[i];
        }
        if (MORE && t + step < dy.rows) read(t + step);
        auto sums = [&](float k, float &sum, float &dot) {
            sum = dot = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const Cols<V> c(V * (me + i * TPR), cols);
                float e[V], g[V];
                floats_of<TX, V>(ha[i], e);
                floats_of<TX, V>(db[i], g);
#pragma unroll
                for (int j = 0; j < V; ++j) e[j] *= k;
                if constexpr (!MORE) load_weight<V>(weight, c.at, w[0]);
                sum += square_sum<V>(e, c);
                dot += product_sum<V>(e, g, w[MORE ? i : 0], c);
            }
            row.sum2(sum, dot);
        };
        float sum, dot, add = eps, k = 1.0f;
        sums(1.0f, sum, dot);
        if (out_of_range(sum, eps)) {
            k = range_step(sum);
            sums(k, sum, dot);
            add = eps * k * k;
        }
        if constexpr (kInLds && VEC == 2) {   // the floats are formed anew below: kept, they would spill
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int j = 0; j < Raw<TX, V>::kUnits; ++j) asm volatile("" : "+v"(ha[i].w[j]), "+v"(db[i].w[j]));
        }
        // of the row times k: unit = h k rho, dx = k (rho (g - unit (dot rho / cols))), in this order:
        // k rho may be beyond fp32's range where dx is not
        const float rho = __builtin_amdgcn_rsqf(fmaf(sum, over_cols, add));
        const float along = dot * rho * over_cols;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const Cols<V> c(V * (me + i * TPR), cols);
            float e[V], g[V], r[V];
            floats_of<TX, V>(ha[i], e);
            floats_of<TX, V>(db[i], g);
            if constexpr (!MORE) load_weight<V>(weight, c.at, w[0]);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float unit = e[j] * k * rho;
                if constexpr (kInLds) dw_at(i, j) = fmaf(g[j], unit, dw_at(i, j));
                else if constexpr (DW) dw[i][j] = fmaf(g[j], unit, dw[i][j]);
                r[j] = k * (rho * (g[j] * w[MORE ? i : 0][j] - unit * along));
            }
            if (dh.data) {
                floats_of<TX, V>(ua[i], e);
#pragma unroll
                for (int j = 0; j < V; ++j) r[j] += e[j];
            }
            if (c.live()) store_once<TX, V>(row_out<TX>(dx, t) + c.at, raw_of<TX, V>(r));
        }
    }
    if constexpr (DW) {
        float *const to = partial + (int64_t)blockIdx.x * cols;
        constexpr int kShared = LANES ? VEC * 8 * 64 : 1;
        __shared__ float total[kShared];
        if constexpr (LANES) {   // the wave's rows, then the block's waves, in order
            const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
            for (int o = LANES; o < 64; o <<= 1)
#pragma unroll
                for (int i = 0; i < N; ++i)
#pragma unroll
                    for (int j = 0; j < V; ++j) dw[i][j] += __shfl_xor(dw[i][j], o);
            for (int s = 0; s < 4; ++s) {
                if (wave == s) {
#pragma unroll
                    for (int i = 0; i < N; ++i)
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            float &at = total[(i * V + j) * 64 + lane];
                            if (s) dw[i][j] += at;
                            at = dw[i][j];
                        }
                }
                __syncthreads();
            }
            if (wave != 3 || lane >= LANES) return;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const Cols<V> c(V * (me + i * TPR), cols);
            float sums[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if constexpr (kInLds) sums[j] = dw_at(i, j);
                else sums[j] = dw[i][j];
            }
            if (!c.dup) {
                store_raw<UMAP_F32, V>(to + c.at, raw_of<UMAP_F32, V>(sums));
            } else {
#pragma unroll
                for (int j = 1; j < V; ++j)
                    if (c.counts(j)) to[c.at + j] = sums[j];
            }
        }
    }
}

// ---- rows of fewer than 8 columns: a thread per row ----
constexpr int kNarrow = 7;

__device__ __forceinline__ float weight_at(const RowWeight &weight, int c)
{
    if (!weight.data) return 1.0f;
    switch (weight.type) {
    case UMAP_F32: return static_cast<const float *>(weight.data)[c];
    case UMAP_F16: return elem_float<UMAP_F16>(static_cast<const _Float16 *>(weight.data)[c]);
    default: return elem_float<UMAP_BF16>(static_cast<const uint16_t *>(weight.data)[c]);
    }
}

template <int TX, int TY>
__global__ __launch_bounds__(256) void k_rows_norm_narrow(umap_rows x, RowIds ids, float scale, umap_rows residual,
                                                          umap_rows h, RowWeight weight, float eps, umap_rows y)
{
    const int cols = y.cols;
    const int64_t step = (int64_t)gridDim.x * 256;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < y.rows; t += step) {
        const int64_t v = row_of(ids, t, x.rows);
        float e[kNarrow], sum = 0.0f, add = eps;
#pragma unroll
        for (int c = 0; c < kNarrow; ++c) {
            e[c] = 0.0f;
            if (c >= cols) continue;
            if (v >= 0) e[c] = elem_float<TX>(row_ptr<TX>(x, v)[c]) * scale;
            if (residual.data) e[c] += elem_float<TX>(row_ptr<TX>(residual, t)[c]);
            if (h.data) row_out<TX>(h, t)[c] = float_elem<TX>(e[c]);
            sum = fmaf(e[c], e[c], sum);
        }
        if (out_of_range(sum, eps)) {
            const float k = range_step(sum);
            sum = 0.0f;
#pragma unroll
            for (int c = 0; c < kNarrow; ++c) {
                e[c] *= k;
                sum = fmaf(e[c], e[c], sum);
            }
            add = eps * k * k;
        }
        const float rho = __builtin_amdgcn_rsqf(sum / (float)cols + add);
        uint32_t most = 0;
#pragma unroll
        for (int c = 0; c < kNarrow; ++c) {
            if (c >= cols) continue;
            e[c] = e[c] * rho * weight_at(weight, c);
            most = max_u(most, __float_as_uint(e[c]) & 0x7fffffffu);
        }
        if constexpr (TY == UMAP_I8 || TY == UMAP_F8) {
            const Quant<TY> quant(most);
            y.scales[t] = quant.scale;   // one group
#pragma unroll
            for (int c = 0; c < kNarrow; ++c)
                if (c < cols) row_out<TY>(y, t)[c] = float_elem<TY>(quant(e[c]));
        } else {
#pragma unroll
            for (int c = 0; c < kNarrow; ++c)
                if (c < cols) row_out<TY>(y, t)[c] = float_elem<TY>(e[c]);
        }
    }
}

template <int TX>
__global__ __launch_bounds__(256) void k_rows_norm_grad_narrow(umap_rows dy, umap_rows h, umap_rows dh, RowWeight weight,
                                                               float eps, umap_rows dx, float *partial)
{
    __shared__ float part[4][kNarrow];
    const int cols = dy.cols;
    const int64_t step = (int64_t)gridDim.x * 256;
    float dw[kNarrow] = {};
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < dy.rows; t += step) {
        float e[kNarrow], g[kNarrow], sum = 0.0f, dot = 0.0f, add = eps, k = 1.0f;
#pragma unroll
        for (int c = 0; c < kNarrow; ++c) {
            e[c] = c < cols ? elem_float<TX>(row_ptr<TX>(h, t)[c]) : 0.0f;
            g[c] = c < cols ? elem_float<TX>(row_ptr<TX>(dy, t)[c]) : 0.0f;
            sum = fmaf(e[c], e[c], sum);
        }
        if (out_of_range(sum, eps)) {
            k = range_step(sum);
            sum = 0.0f;
#pragma unroll
            for (int c = 0; c < kNarrow; ++c) {
                e[c] *= k;
                sum = fmaf(e[c], e[c], sum);
            }
            add = eps * k * k;
        }
        const float rho = __builtin_amdgcn_rsqf(sum / (float)cols + add);
#pragma unroll
        for (int c = 0; c < kNarrow; ++c) {
            if (c >= cols) continue;
            e[c] *= rho;
            dw[c] = fmaf(g[c], e[c], dw[c]);
            g[c] *= weight_at(weight, c);
            dot = fmaf(g[c], e[c], dot);
        }
        const float along = dot / (float)cols;
#pragma unroll
        for (int c = 0; c < kNarrow; ++c) {
            if (c >= cols) continue;
            float r = k * (rho * (g[c] - e[c] * along));
            if (dh.data) r += elem_float<TX>(row_ptr<TX>(dh, t)[c]);
            row_out<TX>(dx, t)[c] = float_elem<TX>(r);
        }
    }
    if (!partial) return;
#pragma unroll
    for (int c = 0; c < kNarrow; ++c) {
        const float sum = lanes_sum<64>(dw[c]);
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6][c] = sum;
    }
    __syncthreads();
    const int c = threadIdx.x;
    if (c < cols) partial[(int64_t)blockIdx.x * cols + c] = part[0][c] + part[1][c] + part[2][c] + part[3][c];
}

// out[c] = partial[0][c] + .. + partial[count - 1][c]: 64 columns per workgroup, each of its
// waves adding a stretch of the rows, then the stretches in order.
constexpr int kJoinWaves = 16;
__global__ __launch_bounds__(64 * kJoinWaves) void k_rows_join(const float *partial, int count, int cols, float *out)
{
    __shared__ float part[kJoinWaves][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = blockIdx.x * 64 + lane;
    const int per = (count + kJoinWaves - 1) / kJoinWaves, first = wave * per, last = min(first + per, count);
    float sum = 0.0f;
    if (c < cols) {
#pragma unroll 8
        for (int b = first; b < last; ++b) sum += partial[(int64_t)b * cols + c];
    }
    part[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && c < cols) {
        for (int w = 1; w < kJoinWaves; ++w) sum += part[w][lane];
        out[c] = sum;
    }
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
int64_t even_grid(int64_t work, int threads, int waves)
{
    const int64_t most = 256 * std::max(1, waves * 64 / threads);
    const int64_t turns = (work + most - 1) / most;
    return (work + turns - 1) / turns;
}
// us per call with upstream gradient and dweight at 8 / 12 / 16 / 20 waves on a CU: 256 MB of bf16
// rows of 300 columns 350 / 272 / 250 / 239, 784 204 / 209 / 230 / 210, 1,024 198 / 195 / 207 / 206, 2,048 226 / 186 / 191 /
// 202, 4,096 207 / 207 / 180 / 180, 8,192 and more the same (one workgroup); 128 MB, three sets in turn, at
// 8 / 12 / 16: 128 columns 88 / 97 / 97, 256 89 / 94 / 98, fp32 196 / 210 / 209 at both.  Lanes in eights, which short
// rows leave partly idle, at 8 / 16: bf16 16 columns 216 / 160, 32 125 / 100, 40 110 / 95, 48 99 / 97, 56 92 / 95, 64 88 / 96;
// fp32, which the same bound costs 7 % from 32 to 48 columns, 16 312 / 233, 24 233 / 213, 32 200 / 215, 48 198 / 214, 64 197 /
// 210.
constexpr int grad_waves(int lanes, int vec, int cols)
{
    return (lanes == 64 && vec == 2) || lanes == 16 || lanes == 32 || (lanes == 8 && cols > 48) ? 8 : 16;
}

template <int TX, int TY>
struct Norm {
    template <int LANES, int VEC>
    struct With {
        static hipError_t go(RowShape shape, const umap_rows *x, RowIds ids, float scale, const umap_rows *residual,
                             const umap_rows *h, RowWeight weight, float eps, const umap_rows *y, hipStream_t s)
        {
            const int64_t work = (y->rows + shape.rows - 1) / shape.rows;
            const dim3 grid(VEC == 4 ? (unsigned)even_grid(work, shape.threads, 16) : (unsigned)norm_grid(work, y->cols, shape.threads));
            const dim3 threads(shape.threads);
            const umap_rows r = residual ? *residual : umap_rows{}, to = h ? *h : umap_rows{};
            if constexpr (LANES == kOneThread)
                hipLaunchKernelGGL((k_rows_norm_narrow<TX, TY>), grid, threads, 0, s, *x, ids, scale, r, to, weight, eps, *y);
            else
                hipLaunchKernelGGL((k_rows_norm<TX, TY, LANES, VEC, (VEC < 4)>), grid, threads, 0, s, *x, ids, scale, r, to, weight, eps, *y);
            return hipGetLastError();
        }
    };
};

template <int LANES, int VEC>
struct GradBlocks {
    static int64_t go(RowShape shape, int64_t n, int cols)
    {
        return even_grid((n + shape.rows - 1) / shape.rows, shape.threads, grad_waves(LANES, VEC, cols));
    }
};
constexpr int kGradOne = 8192, kNormOne = 4096;   // columns up to which one vector per thread measured best

template <int TX>
struct Grad {
    template <int LANES, int VEC>
    struct With {
        static hipError_t go(RowShape shape, const umap_rows *dy, const umap_rows *h, const umap_rows *dh,
                             RowWeight weight, float eps, const umap_rows *dx, float *partial, int64_t *count, hipStream_t s)
        {
            const int64_t work = (dy->rows + shape.rows - 1) / shape.rows;
            *count = partial || VEC == 4 ? GradBlocks<LANES, VEC>::go(shape, dy->rows, dy->cols) : norm_grid(work, dy->cols, shape.threads);
            const dim3 grid((unsigned)*count), threads(shape.threads);
            const size_t sums = LANES == kBlock && VEC > 1 ? (size_t)shape.threads * VEC * 32 : 0;
            const umap_rows up = dh ? *dh : umap_rows{};
            if constexpr (LANES == kOneThread)
                hipLaunchKernelGGL((k_rows_norm_grad_narrow<TX>), grid, threads, 0, s, *dy, *h, up, weight, eps, *dx, partial);
            else if (partial)
                hipLaunchKernelGGL((k_rows_norm_grad<TX, LANES, VEC, true, (VEC < 4)>), grid, threads, sums, s, *dy, *h, up, weight, eps, *dx, partial);
            else
                hipLaunchKernelGGL((k_rows_norm_grad<TX, LANES, VEC, false, (VEC < 4)>), grid, threads, 0, s, *dy, *h, up, weight, eps, *dx, nullptr);
            return hipGetLastError();
        }
    };
};

template <int TX, typename... Args>
hipError_t norm_from(int32_t type, int cols, Args... args)
{
    switch (type) {
    case UMAP_F32: return by_cols<Norm<TX, UMAP_F32>::template With>(cols, kNormOne, args...);
    case UMAP_F16: return by_cols<Norm<TX, UMAP_F16>::template With>(cols, kNormOne, args...);
    case UMAP_BF16: return by_cols<Norm<TX, UMAP_BF16>::template With>(cols, kNormOne, args...);
    case UMAP_I8: return by_cols<Norm<TX, UMAP_I8>::template With>(cols, kNormOne, args...);
    default: return by_cols<Norm<TX, UMAP_F8>::template With>(cols, kNormOne, args...);
    }
}

}  // namespace

hipError_t launch_rows_norm(const umap_rows &x, RowIds ids, float scale, const umap_rows *residual, const umap_rows *h,
                            RowWeight weight, float eps, const umap_rows &to, hipStream_t s)
{
    umap_rows y = to;
    if (y.group >= y.cols) y.group = 0;   // one group: the kernels take a group to lie in one vector of its lanes
    switch (x.type) {
    case UMAP_F32: return norm_from<UMAP_F32>(y.type, y.cols, &x, ids, scale, residual, h, weight, eps, &y, s);
    case UMAP_F16: return norm_from<UMAP_F16>(y.type, y.cols, &x, ids, scale, residual, h, weight, eps, &y, s);
    default: return norm_from<UMAP_BF16>(y.type, y.cols, &x, ids, scale, residual, h, weight, eps, &y, s);
    }
}

int64_t rows_norm_grad_bytes(int64_t n, int32_t cols)
{
    if (n < 1) return 16;
    return by_cols<GradBlocks>(cols, kGradOne, n, cols) * cols * 4;   // one sum of dweight per workgroup
}

hipError_t launch_rows_norm_grad(const umap_rows &dy, const umap_rows &h, const umap_rows *dh, RowWeight weight,
                                 float eps, const umap_rows &dx, float *dweight, void *workspace, hipStream_t s)
{
    int64_t count = 0;
    // one workgroup's sums are dweight itself
    const bool one = dweight && dy.rows > 0 && by_cols<GradBlocks>(dy.cols, kGradOne, dy.rows, dy.cols) == 1;
    float *const partial = one ? dweight : dweight ? static_cast<float *>(workspace) : nullptr;
    if (dy.rows > 0) {
        hipError_t e;
        switch (dy.type) {
        case UMAP_F32: e = by_cols<Grad<UMAP_F32>::With>(dy.cols, kGradOne, &dy, &h, dh, weight, eps, &dx, partial, &count, s); break;
        case UMAP_F16: e = by_cols<Grad<UMAP_F16>::With>(dy.cols, kGradOne, &dy, &h, dh, weight, eps, &dx, partial, &count, s); break;
        default: e = by_cols<Grad<UMAP_BF16>::With>(dy.cols, kGradOne, &dy, &h, dh, weight, eps, &dx, partial, &count, s); break;
        }
        if (e != hipSuccess) return e;
    }
    if (dweight && !one) {
        hipLaunchKernelGGL(k_rows_join, dim3((dy.cols + 63) / 64), dim3(64 * kJoinWaves), 0, s, partial, (int)count,
                           dy.cols, dweight);
        return hipGetLastError();
    }
    return hipSuccess;
}

}  // namespace ul
