// kernels_rows_layer.hip -- mean and variance norm of rows and its gradient (umap_rows.h).
//
//   norm      h = x + residual, off = h - mean h, rho = 1 / sqrt(mean off^2 + eps), y = off rho weight + bias
//   gradient  u = off rho, g = dy weight, dx = rho (g - mean g - u mean(g u)) + dh, dweight = sum dy u, dbias = sum dy
//
// Bound by memory: as in the root-mean-square norm a row is read once and stays in
// registers, in the same lanes, waves and workgroups.  All its sums are taken at once, of differences from the row's
// first value h0: e = h - h0, mean h = h0 + mean e, mean off^2 = mean e^2 - (mean e)^2, and mean(g off) likewise.  That
// loses at most the factor 1 + (mean e)^2 / mean off^2 in precision, however far the mean is from zero; rows for which it
// is over 17 (h0 four deviations off), or whose squares leave fp32's range, are read again and taken in two turns, the
// mean first.  The gradient keeps the sums of dweight and dbias of a workgroup's rows in registers or
// LDS; a second launch joins the workgroups in order.  Beyond 16,384 columns neither holds them: there each row's
// mean and rho are written down, and a launch of its own forms the two sums, reading dy and h a second time.
//
// us per call and TB/s of what is read and written, three sets of inputs in turn: 32,768 x 4,096 bf16 with residual 172 (6.2),
// its gradient with upstream gradient, dweight and dbias 177 (6.1); 70,000 x 784 fp32 into bf16 57 (5.8); gradients of 65,536 x
// 2,048 141 (5.7), 131,072 x 768 112 (5.4), 131,072 x 300 61 (3.8: 38 of 64 lanes have any).  With the mean taken first and the
// sums in two or three turns the gradient of 32,768 x 4,096 took 202.  Weaker: from 4,097 to 8,192 columns a workgroup of up to
// 16 waves is alone on its CU (norm of 16,384 x 8,192 133, 4.1; with residual 188, 5.7; its gradient 210, 5.1), and beyond registers are short (8,192 x 20,000:
// 207, 3.2; gradient 417, 2.4).
#include "rows_norm_device.hpp"

namespace ul {

namespace {

// v plus its value 16 or 32 lanes away, in both: the hardware swaps the halves of two registers, here of one and the same.
__device__ __forceinline__ float add_16(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float add_32(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Sums over a row's threads, K values at once; the two buffers take turns, so that one barrier is
// enough: a buffer is written again only after the next sum's barrier.
struct LayerLds {
    float v[2][16][4];
};
template <int LANES>
struct LayerSums {
    LayerLds *lds;
    int turn = 0;
    template <int K>
    __device__ __forceinline__ void operator()(float (&v)[K])
    {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = add_dpp<kXor1>(v[k]);
            v[k] = add_dpp<kXor2>(v[k]);
            v[k] = add_dpp<kHalfMirror>(v[k]);
            if constexpr (LANES != 8) v[k] = add_dpp<kMirror>(v[k]);
            if constexpr (LANES == 32 || LANES == 64 || LANES == kBlock) v[k] = add_16(v[k]);
            if constexpr (LANES == 64 || LANES == kBlock) v[k] = add_32(v[k]);
        }
        if constexpr (LANES == kBlock) {
            typedef float F4 __attribute__((ext_vector_type(4)));
            F4(&at)[16] = reinterpret_cast<F4(&)[16]>(lds->v[turn]);
            if ((threadIdx.x & 63) == 0) {
                F4 mine = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int k = 0; k < K; ++k) mine[k] = v[k];
                at[threadIdx.x >> 6] = mine;
            }
            __syncthreads();
            F4 all = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int w = 0; w < (int)(blockDim.x >> 6); ++w) all += at[w];
#pragma unroll
            for (int k = 0; k < K; ++k) v[k] = all[k];
            turn ^= 1;
        }
    }
};

// Sums over a row of what `terms` adds for column j of the thread's vector i.
template <int LANES, int V, int N, int K, typename Terms>
__device__ __forceinline__ void row_sums(LayerSums<LANES> &row, int me, int TPR, int cols, float (&sums)[K], Terms terms)
{
#pragma unroll
    for (int k = 0; k < K; ++k) sums[k] = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const Cols<V> c(V * (me + i * TPR), cols);
        float s[K] = {};
#pragma unroll
        for (int j = 0; j < V; ++j) terms(i, j, s);
        if (c.shared()) {
#pragma unroll
            for (int k = 0; k < K; ++k) s[k] = 0.0f;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float more[K];
#pragma unroll
                for (int k = 0; k < K; ++k) more[k] = s[k];
                terms(i, j, more);
#pragma unroll
                for (int k = 0; k < K; ++k) s[k] = c.counts(j) ? more[k] : s[k];
            }
        }
#pragma unroll
        for (int k = 0; k < K; ++k) sums[k] += c.live() ? s[k] : 0.0f;
    }
    row(sums);
}

// What centres a row: e - shift = k (h - mean h), rho = 1 / sqrt(mean of its square + k^2 eps).  k is a power of two, 1 but
// where squares would leave fp32's range.
struct Spread {
    float rho, k;
    float mean, left;   // k (h - mean h) = (k h - mean) - left, or k (h - mean) - left where k > 1
};
// With a gradient g: mean g, and the mean of g times k (h - mean h) rho.
struct Along {
    float mean_g, along;
};

// In two turns, for any row; e: h on the way in, centred on the way out.
template <int LANES, int V, int N, bool kGrad>
__device__ __forceinline__ Spread centre(LayerSums<LANES> &row, float (&e)[N][V], const float (&g)[kGrad ? N : 1][V], float sum_g,
                                         int me, int TPR, int cols, float eps, Along *along)
{
    const float over_cols = 1.0f / (float)cols;
    constexpr int K = kGrad ? 3 : 2;
    float sums[K], k = 1.0f, mean, left = 0.0f;
    auto times = [&](float by) {
        k *= by;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) e[i][j] *= by;
    };
    auto less = [&](float by) {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) e[i][j] -= by;
    };
    auto squares = [&] {
        row_sums<LANES, V, N>(row, me, TPR, cols, sums, [&](int i, int j, float (&s)[K]) {
            s[0] += e[i][j];
            s[1] = fmaf(e[i][j], e[i][j], s[1]);
            if constexpr (kGrad) s[2] = fmaf(g[i][j], e[i][j], s[2]);
        });
    };
    squares();
    if (!(sums[1] < __builtin_inff())) {
        times(0x1p-80f);
        squares();
    }
    mean = sums[0] * over_cols;
    less(mean);
    squares();
    // Values within some 2^-10 of their mean: their differences from it are exact, and so are those from the first
    // one's, which are zeros where the values are equal (differences from a rounded mean would be noise).
    auto from_first = [&] {
        float first[1] = {me == 0 ? e[0][0] : 0.0f};
        row(first);
        less(first[0]);
        left += first[0];
        squares();
    };
    if (sums[1] < 0x1p-20f * (mean * mean) * (float)cols) from_first();
    if (k < 1.0f && sums[1] < 0x1p-40f) {   // large, but nearly alike
        times(0x1p80f);
        mean *= 0x1p80f;
        left *= 0x1p80f;
        squares();
    }
    if (k == 1.0f && sums[1] < kSmallSum && eps < kSmallSum) {
        times(0x1p94f);
        left *= 0x1p94f;
        from_first();
    }
    const float rest = sums[0] * over_cols;   // of the mean's rounding
    less(rest);
    float var = fmaf(sums[1], over_cols, -rest * rest);
    var = var < 0.0f ? 0.0f : var;
    const float rho = __builtin_amdgcn_rsqf(var + eps * k * k);
    if constexpr (kGrad) *along = {sum_g * over_cols, fmaf(-rest, sum_g, sums[K - 1]) * rho * over_cols};
    return {rho, k, mean, left + rest};
}

// In one turn where that is precise.  e: h - h0 on the way in (and out, `shift` above zero mean), or centred on the way out;
// `again` forms h once more.
template <int LANES, int V, int N, bool kGrad, typename Again>
__device__ __forceinline__ Spread spread(LayerSums<LANES> &row, float (&e)[N][V], const float (&g)[kGrad ? N : 1][V], float h0,
                                         int me, int TPR, int cols, float eps, float &shift, Along *along, Again again)
{
    const float over_cols = 1.0f / (float)cols;
    constexpr int K = kGrad ? 4 : 2;
    float sums[K];
    row_sums<LANES, V, N>(row, me, TPR, cols, sums, [&](int i, int j, float (&s)[K]) {
        s[0] += e[i][j];
        s[1] = fmaf(e[i][j], e[i][j], s[1]);
        if constexpr (kGrad) {
            s[2] += g[i][j];
            s[3] = fmaf(g[i][j], e[i][j], s[3]);
        }
    });
    const float sum_g = kGrad ? sums[K - 2] : 0.0f;
    shift = sums[0] * over_cols;
    const float var = fmaf(sums[1], over_cols, -shift * shift);
    if (sums[1] < __builtin_inff() && 16.0f * var >= shift * shift && (sums[1] >= kSmallSum || eps >= kSmallSum)) {
        const float rho = __builtin_amdgcn_rsqf(var + eps);
        if constexpr (kGrad) *along = {sum_g * over_cols, fmaf(-shift, sum_g, sums[K - 1]) * rho * over_cols};
        return {rho, 1.0f, h0, shift};
    }
    shift = 0.0f;
    again();
    return centre<LANES, V, N, kGrad>(row, e, g, sum_g, me, TPR, cols, eps, along);
}

// N vectors of V columns per thread.  MORE: a thread keeps its weights over its rows and reads a row ahead.
template <int TX, int TY, int LANES, int V, int N, bool MORE>
__global__ __launch_bounds__(kMostThreads<LANES>) void k_rows_layer(umap_rows x, umap_rows residual, umap_rows h,
                                                                    RowWeight weight, RowWeight bias, float eps, umap_rows y)
{
    constexpr int kRows = kRowsPerBlock<LANES>;
    __shared__ LayerLds lds;
    LayerSums<LANES> row{&lds};
    const int TPR = row_threads<LANES>(), me = LANES ? threadIdx.x & (LANES - 1) : threadIdx.x, cols = y.cols;
    float w[MORE ? N : 1][V], b[MORE ? N : 1][V];
    auto read_weight = [&](int i, float (&w)[V], float (&b)[V]) {
        const int at = Cols<V>(V * (me + i * TPR), cols).at;
        load_weight<V>(weight, at, w);
        load_weight<V>(bias, at, b);
        if (!bias.data) {
#pragma unroll
            for (int j = 0; j < V; ++j) b[j] = 0.0f;
        }
    };
    if constexpr (MORE) {
#pragma unroll
        for (int i = 0; i < N; ++i) read_weight(i, w[i], b[i]);
    }
    Raw<TX, V> a[N], r[N];
    Elem<TX> a0, r0;   // the row's first value
    auto read = [&](int64_t t) {
        a0 = row_ptr<TX>(x, t)[0];
        if (residual.data) r0 = row_ptr<TX>(residual, t)[0];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = Cols<V>(V * (me + i * TPR), cols).at;
            a[i] = load_once<TX, V>(row_ptr<TX>(x, t) + at);
            if (residual.data) r[i] = load_once<TX, V>(row_ptr<TX>(residual, t) + at);
        }
    };
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t t = (int64_t)blockIdx.x * kRows + row_in_block<LANES>();
    if (MORE && t < y.rows) read(t);
    for (; t < y.rows; t += step) {
        if (!MORE) read(t);
        float e[N][V];
        const float h0 = residual.data ? elem_float<TX>(a0) + elem_float<TX>(r0) : elem_float<TX>(a0);
        Raw<TX, V> keep[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            floats_of<TX, V>(a[i], e[i]);
            if (residual.data) {
                float more[V];
                floats_of<TX, V>(r[i], more);
#pragma unroll
                for (int j = 0; j < V; ++j) e[i][j] += more[j];
            }
            if (h.data) keep[i] = raw_of<TX, V>(e[i]);
#pragma unroll
            for (int j = 0; j < V; ++j) e[i][j] -= h0;
        }
        if (MORE && t + step < y.rows) read(t + step);
        const float none[1][V] = {};
        float shift;
        const Spread s = spread<LANES, V, N, false>(row, e, none, h0, me, TPR, cols, eps, shift, nullptr, [&] {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int at = Cols<V>(V * (me + i * TPR), cols).at;
                floats_of<TX, V>(load_raw<TX, V>(row_ptr<TX>(x, t) + at), e[i]);
                if (residual.data) {
                    float more[V];
                    floats_of<TX, V>(load_raw<TX, V>(row_ptr<TX>(residual, t) + at), more);
#pragma unroll
                    for (int j = 0; j < V; ++j) e[i][j] += more[j];
                }
            }
        });
        const float less = -shift * s.rho;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const Cols<V> c(V * (me + i * TPR), cols);
            if constexpr (!MORE) read_weight(i, w[0], b[0]);
#pragma unroll
            for (int j = 0; j < V; ++j)
                e[i][j] = fmaf(fmaf(e[i][j], s.rho, less), w[MORE ? i : 0][j], b[MORE ? i : 0][j]);
            if (!c.live()) continue;
            // behind the sums' barriers: h may lie where other waves read
            if (h.data) store_once<TX, V>(row_out<TX>(h, t) + c.at, keep[i]);
            store_once<TY, V>(row_out<TY>(y, t) + c.at, raw_of<TY, V>(e[i]));
        }
    }
}

// DW: sums of dweight and dbias, 2 cols per workgroup.  stats: null, or receives each row's Spread.  dx's data may be
// null: the statistics alone.
template <int TX, int LANES, int V, int N, bool DW, bool MORE>
__global__ __launch_bounds__(kMostThreads<LANES>) void k_rows_layer_grad(umap_rows dy, umap_rows h, umap_rows dh,
                                                                         RowWeight weight, float eps, umap_rows dx,
                                                                         float *partial, Spread *stats)
{
    constexpr int kRows = kRowsPerBlock<LANES>;
    __shared__ LayerLds lds;
    LayerSums<LANES> row{&lds};
    const int TPR = row_threads<LANES>(), me = LANES ? threadIdx.x & (LANES - 1) : threadIdx.x, cols = dy.cols;
    const float over_cols = 1.0f / (float)cols;
    // the sums of this thread's columns, in LDS where registers are short
    constexpr bool kInLds = DW && LANES == kBlock && N > 1;
    extern __shared__ float sums_lds[];
    float w[MORE ? N : 1][V], dw[DW && !kInLds ? N : 1][V], db[DW && !kInLds ? N : 1][V];
    auto lds_at = [&](int which, int i, int j) -> float & { return sums_lds[((which * N + i) * V + j) * TPR + me]; };
    if constexpr (MORE) {
#pragma unroll
        for (int i = 0; i < N; ++i) load_weight<V>(weight, Cols<V>(V * (me + i * TPR), cols).at, w[i]);
    }
#pragma unroll
    for (int i = 0; i < (DW ? N : 1); ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if constexpr (kInLds) lds_at(0, i, j) = lds_at(1, i, j) = 0.0f;
            else dw[i][j] = db[i][j] = 0.0f;
        }
    Raw<TX, V> a[N], b[N], u[N];
    Elem<TX> a0;   // the row's first value
    auto read = [&](int64_t t) {
        a0 = row_ptr<TX>(h, t)[0];
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
        Raw<TX, V> db_raw[N], ua[N];
        float e[N][V], g[N][V];
        const float h0 = elem_float<TX>(a0);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            floats_of<TX, V>(a[i], e[i]);
            floats_of<TX, V>(b[i], g[i]);
            db_raw[i] = b[i];
            if (dh.data) ua[i] = u[i];
            if constexpr (!MORE) load_weight<V>(weight, Cols<V>(V * (me + i * TPR), cols).at, w[0]);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                e[i][j] -= h0;
                g[i][j] *= w[MORE ? i : 0][j];
            }
        }
        if (MORE && t + step < dy.rows) read(t + step);
        Along means;
        float shift;
        const Spread s = spread<LANES, V, N, true>(row, e, g, h0, me, TPR, cols, eps, shift, &means, [&] {
#pragma unroll
            for (int i = 0; i < N; ++i)
                floats_of<TX, V>(load_raw<TX, V>(row_ptr<TX>(h, t) + Cols<V>(V * (me + i * TPR), cols).at), e[i]);
        });
        const float less = -shift * s.rho;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float y[V];   // dy
            if constexpr (DW) floats_of<TX, V>(db_raw[i], y);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                e[i][j] = fmaf(e[i][j], s.rho, less);   // u
                if constexpr (kInLds) {
                    lds_at(0, i, j) = fmaf(y[j], e[i][j], lds_at(0, i, j));
                    lds_at(1, i, j) += y[j];
                } else if constexpr (DW) {
                    dw[i][j] = fmaf(y[j], e[i][j], dw[i][j]);
                    db[i][j] += y[j];
                }
            }
        }
        if (stats && me == 0) stats[t] = s;
        const float off = -means.mean_g * s.rho, along = -means.along * s.rho;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const Cols<V> c(V * (me + i * TPR), cols);
            if (s.k == 1.0f) {
#pragma unroll
                for (int j = 0; j < V; ++j) g[i][j] = fmaf(e[i][j], along, fmaf(g[i][j], s.rho, off));
            } else {   // in this order: k rho may be beyond fp32's range where dx is not
#pragma unroll
                for (int j = 0; j < V; ++j) g[i][j] = s.k * (s.rho * ((g[i][j] - means.mean_g) - e[i][j] * means.along));
            }
            if (dh.data) {
                float more[V];
                floats_of<TX, V>(ua[i], more);
#pragma unroll
                for (int j = 0; j < V; ++j) g[i][j] += more[j];
            }
            if (c.live() && dx.data) store_once<TX, V>(row_out<TX>(dx, t) + c.at, raw_of<TX, V>(g[i]));
        }
    }
    if constexpr (DW) {
        float *const to = partial + (int64_t)blockIdx.x * 2 * cols;
        if constexpr (LANES) {   // the wave's rows, then the block's waves, in order
            __shared__ float total[N * V * 64];
            const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
            for (int which = 0; which < 2; ++which) {
                float(&d)[N][V] = which ? db : dw;
                for (int o = LANES; o < 64; o <<= 1)
#pragma unroll
                    for (int i = 0; i < N; ++i)
#pragma unroll
                        for (int j = 0; j < V; ++j) d[i][j] += __shfl_xor(d[i][j], o);
                for (int s = 0; s < 4; ++s) {
                    if (wave == s) {
#pragma unroll
                        for (int i = 0; i < N; ++i)
#pragma unroll
                            for (int j = 0; j < V; ++j) {
                                float &at = total[(i * V + j) * 64 + lane];
                                if (s) d[i][j] += at;
                                at = d[i][j];
                            }
                    }
                    __syncthreads();
                }
            }
            if (wave != 3 || lane >= LANES) return;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const Cols<V> c(V * (me + i * TPR), cols);
#pragma unroll
            for (int which = 0; which < 2; ++which)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float sum;
                    if constexpr (kInLds) sum = lds_at(which, i, j);
                    else sum = which ? db[i][j] : dw[i][j];
                    if (c.live() && c.counts(j)) to[which * cols + c.at + j] = sum;
                }
        }
    }
}

// dweight's and dbias's sums of a stretch of rows from their statistics, 8 columns per lane.
template <int TX>
__global__ __launch_bounds__(256) void k_rows_layer_sums(umap_rows dy, umap_rows h, const Spread *stats, int64_t stretch,
                                                         float *partial)
{
    constexpr int V = 8;
    const int cols = dy.cols;
    const Cols<V> c(V * ((int)blockIdx.x * 256 + (int)threadIdx.x), cols);
    if (!c.live()) return;
    const int64_t first = blockIdx.y * stretch, last = min(first + stretch, dy.rows);
    float dw[V] = {}, db[V] = {};
#pragma unroll 4
    for (int64_t t = first; t < last; ++t) {
        const Spread s = stats[t];
        float e[V], g[V];
        floats_of<TX, V>(load_once<TX, V>(row_ptr<TX>(h, t) + c.at), e);
        floats_of<TX, V>(load_once<TX, V>(row_ptr<TX>(dy, t) + c.at), g);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float off = (s.k > 1.0f ? (e[j] - s.mean) * s.k : e[j] * s.k - s.mean) - s.left;
            dw[j] = fmaf(g[j], off * s.rho, dw[j]);
            db[j] += g[j];
        }
    }
    float *const to = partial + (int64_t)blockIdx.y * 2 * cols;
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (c.counts(j)) {
            to[c.at + j] = dw[j];
            to[cols + c.at + j] = db[j];
        }
}

// Columns 0 .. cols - 1 of the partial sums' rows into dweight, the rest into dbias (either may be null): 64 columns per
// workgroup, each of its waves adding a stretch of the rows, then the stretches in order.
constexpr int kLayerJoinWaves = 16;
__global__ __launch_bounds__(64 * kLayerJoinWaves) void k_rows_layer_join(const float *partial, int64_t count, int cols,
                                                                          float *dweight, float *dbias)
{
    __shared__ float part[kLayerJoinWaves][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = blockIdx.x * 64 + lane;
    const int64_t per = (count + kLayerJoinWaves - 1) / kLayerJoinWaves, first = wave * per, last = min(first + per, count);
    float sum = 0.0f;
    if (c < 2 * cols) {
#pragma unroll 8
        for (int64_t b = first; b < last; ++b) sum += partial[b * 2 * cols + c];
    }
    part[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && c < 2 * cols) {
        for (int w = 1; w < kLayerJoinWaves; ++w) sum += part[w][lane];
        if (c < cols && dweight) dweight[c] = sum;
        if (c >= cols && dbias) dbias[c - cols] = sum;
    }
}

// Rows of fewer than 8 columns: a lane per column, 8 lanes per row.
template <int LANES, int VEC, int TX, int TY>
struct LayerShape {
    static constexpr bool kNarrow = LANES == kOneThread;
    static constexpr int kLanes = kNarrow ? 8 : LANES;
    // as in the root-mean-square norm: 16 bytes of fp32 next to each other
    static constexpr int V = kNarrow ? 1 : TX == UMAP_F32 && TY == UMAP_F32 && VEC < 4 ? 4 : 8;
    static constexpr int N = kNarrow ? 1 : VEC * 8 / V;
    static RowShape shape(RowShape s) { return kNarrow ? RowShape{256, 32} : s; }
};
constexpr int kLayerOne = 8192;   // columns up to which a workgroup's threads have one vector

template <int TX, int TY>
struct Layer {
    template <int LANES, int VEC>
    struct With {
        static hipError_t go(RowShape of, const umap_rows *x, const umap_rows *residual, const umap_rows *h, RowWeight weight,
                             RowWeight bias, float eps, const umap_rows *y, hipStream_t s)
        {
            using L = LayerShape<LANES, VEC, TX, TY>;
            const RowShape shape = L::shape(of);
            const int64_t work = (y->rows + shape.rows - 1) / shape.rows;
            const int64_t grid = VEC == 4 ? even_grid(work, shape.threads, 16) : norm_grid(work, y->cols, shape.threads);
            hipLaunchKernelGGL((k_rows_layer<TX, TY, L::kLanes, L::V, L::N, (VEC < 4)>), dim3((unsigned)grid), dim3(shape.threads), 0,
                               s, *x, residual ? *residual : umap_rows{}, h ? *h : umap_rows{}, weight, bias, eps, *y);
            return hipGetLastError();
        }
    };
};

// Workgroups of the gradient, each of which hands over sums of its rows: as many as make this number of waves on a CU.
// us per call at 8 / 12 / 16 / 24, three sets of inputs in turn: 131,072 x 300 bf16 79 / 68 / 61 / 73, 512 74 / 72 / 73 / 91, 768
// 112 / 106 / 128 / 116, 1,024 139 / 146 / 156 / 151, 65,536 x 2,048 169 / 141 / 149 / 174, 32,768 x 4,096 with upstream
// gradient 227 / 227 / 177 / 221 (one workgroup, one, two, two uneven ones), 131,072 x 200 fp16 44 / 45 / 42 / 51, 50,000 x
// 1,024 fp32 121 / 128 / 128 / 134, 16,384 x 4,096 fp32 154 / 154 / 158 / 168.
constexpr int layer_waves(int lanes, int vec, int threads) { return lanes == 64 && vec == 2 ? 8 : lanes == kBlock && threads <= 256 ? 12 : 16; }
template <int LANES, int VEC>
struct LayerBlocks {
    static int64_t go(RowShape of, int64_t n)
    {
        const RowShape shape = LayerShape<LANES, VEC, UMAP_BF16, UMAP_BF16>::shape(of);
        return even_grid((n + shape.rows - 1) / shape.rows, shape.threads, layer_waves(LANES, VEC, shape.threads));
    }
};
constexpr int kLayerLdsCols = 16384;   // beyond these the sums have a launch of their own
// Stretches of rows of that launch: about 1,024 workgroups.
int64_t stretches(int64_t n, int cols)
{
    const int64_t strips = (cols + 2047) / 2048;
    return std::min(n, std::max<int64_t>(1, 1024 / strips));
}

template <int TX>
struct LayerGrad {
    template <int LANES, int VEC>
    struct With {
        static hipError_t go(RowShape of, const umap_rows *dy, const umap_rows *h, const umap_rows *dh, RowWeight weight,
                             float eps, const umap_rows *dx, float *partial, Spread *stats, hipStream_t s)
        {
            using L = LayerShape<LANES, VEC, UMAP_BF16, UMAP_BF16>;
            const RowShape shape = L::shape(of);
            const int64_t work = (dy->rows + shape.rows - 1) / shape.rows;
            const int64_t grid = partial || VEC == 4 ? LayerBlocks<LANES, VEC>::go(of, dy->rows) : norm_grid(work, dy->cols, shape.threads);
            const dim3 blocks((unsigned)grid), threads(shape.threads);
            const umap_rows up = dh ? *dh : umap_rows{};
            if constexpr (VEC < 4) {
                if (partial) {
                    const size_t sums = LANES == kBlock && VEC > 1 ? (size_t)shape.threads * VEC * 64 : 0;
                    hipLaunchKernelGGL((k_rows_layer_grad<TX, L::kLanes, L::V, L::N, true, true>), blocks, threads, sums, s, *dy, *h, up,
                                       weight, eps, *dx, partial, nullptr);
                    return hipGetLastError();
                }
            }
            hipLaunchKernelGGL((k_rows_layer_grad<TX, L::kLanes, L::V, L::N, false, (VEC < 4)>), blocks, threads, 0, s, *dy, *h, up,
                               weight, eps, *dx, nullptr, stats);
            return hipGetLastError();
        }
    };
};

template <int TX>
hipError_t layer_from(const umap_rows *x, const umap_rows *residual, const umap_rows *h, RowWeight weight, RowWeight bias,
                      float eps, const umap_rows *y, hipStream_t s)
{
    switch (y->type) {
    case UMAP_F32: return by_cols<Layer<TX, UMAP_F32>::template With>(y->cols, kLayerOne, x, residual, h, weight, bias, eps, y, s);
    case UMAP_F16: return by_cols<Layer<TX, UMAP_F16>::template With>(y->cols, kLayerOne, x, residual, h, weight, bias, eps, y, s);
    default: return by_cols<Layer<TX, UMAP_BF16>::template With>(y->cols, kLayerOne, x, residual, h, weight, bias, eps, y, s);
    }
}

template <int TX>
hipError_t layer_grad(const umap_rows &dy, const umap_rows &h, const umap_rows *dh, RowWeight weight, float eps,
                      const umap_rows &dx, bool sums, void *workspace, int64_t *count, hipStream_t s)
{
    const int64_t n = dy.rows;
    const int cols = dy.cols;
    if (!sums || cols <= kLayerLdsCols) {
        *count = sums ? by_cols<LayerBlocks>(cols, kLayerOne, n) : 0;
        return by_cols<LayerGrad<TX>::template With>(cols, kLayerOne, &dy, &h, dh, weight, eps, &dx,
                                                     sums ? static_cast<float *>(workspace) : nullptr, static_cast<Spread *>(nullptr), s);
    }
    const int64_t most = stretches(n, cols), stretch = (n + most - 1) / most;
    *count = (n + stretch - 1) / stretch;
    auto *const partial = static_cast<float *>(workspace);
    auto *const stats = reinterpret_cast<Spread *>(partial + most * 2 * cols);
    auto rows = [&](const umap_rows &to) {
        return by_cols<LayerGrad<TX>::template With>(cols, kLayerOne, &dy, &h, dh, weight, eps, &to, static_cast<float *>(nullptr), stats, s);
    };
    // where dx replaces dy, the sums have to read dy before
    const bool replaced = dx.data == dy.data;
    hipError_t e = rows(replaced ? umap_rows{} : dx);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_rows_layer_sums<TX>), dim3((cols + 2047) / 2048, (unsigned)*count), dim3(256), 0, s, dy, h, stats, stretch,
                       partial);
    e = hipGetLastError();
    return e == hipSuccess && replaced ? rows(dx) : e;
}

}  // namespace

hipError_t launch_rows_layer_norm(const umap_rows &x, const umap_rows *residual, const umap_rows *h, RowWeight weight,
                                  RowWeight bias, float eps, const umap_rows &y, hipStream_t s)
{
    switch (x.type) {
    case UMAP_F32: return layer_from<UMAP_F32>(&x, residual, h, weight, bias, eps, &y, s);
    case UMAP_F16: return layer_from<UMAP_F16>(&x, residual, h, weight, bias, eps, &y, s);
    default: return layer_from<UMAP_BF16>(&x, residual, h, weight, bias, eps, &y, s);
    }
}

int64_t rows_layer_norm_grad_bytes(int64_t n, int32_t cols)
{
    if (n < 1) return 16;
    if (cols <= kLayerLdsCols) return by_cols<LayerBlocks>(cols, kLayerOne, n) * 2 * cols * 4;
    return stretches(n, cols) * 2 * cols * 4 + n * (int64_t)sizeof(Spread);
}

hipError_t launch_rows_layer_norm_grad(const umap_rows &dy, const umap_rows &h, const umap_rows *dh, RowWeight weight, float eps,
                                       const umap_rows &dx, float *dweight, float *dbias, void *workspace, hipStream_t s)
{
    const bool sums = dweight || dbias;
    int64_t count = 0;
    if (dy.rows > 0) {
        hipError_t e;
        switch (dy.type) {
        case UMAP_F32: e = layer_grad<UMAP_F32>(dy, h, dh, weight, eps, dx, sums, workspace, &count, s); break;
        case UMAP_F16: e = layer_grad<UMAP_F16>(dy, h, dh, weight, eps, dx, sums, workspace, &count, s); break;
        default: e = layer_grad<UMAP_BF16>(dy, h, dh, weight, eps, dx, sums, workspace, &count, s); break;
        }
        if (e != hipSuccess) return e;
    }
    if (!sums) return hipSuccess;
    hipLaunchKernelGGL(k_rows_layer_join, dim3((2 * dy.cols + 63) / 64), dim3(64 * kLayerJoinWaves), 0, s,
                       static_cast<const float *>(workspace), count, dy.cols, dweight, dbias);
    return hipGetLastError();
}

}  // namespace ul
