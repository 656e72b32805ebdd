// kernels_rows_layer.hip -- mean and variance norm of rows and its gradient (umap_rows.h).
//
//   norm      h = x + residual, off = h - mean h, rho = 1 / sqrt(mean off^2 + eps), y = off rho weight + bias
//   gradient  u = off rho, g = dy weight, dx = rho (g - mean g - u mean(g u)) + dh, dweight = sum dy u, dbias = sum dy
//
// Bound by memory: as in the root-mean-square norm a row is read once and stays in
// registers, in the same lanes, waves and workgroups.  The sums take two turns: the mean first, then the
// sums of h - mean and of its square, the first of which corrects the mean's own rounding (a row of 1000 +- 1
// keeps its digits).  The gradient keeps the sums of dweight and dbias of a workgroup's rows in registers or
// LDS; a second launch joins the workgroups in order.  Beyond 16,384 columns neither holds them: there each row's
// mean and rho are written down, and a launch of its own forms the two sums, reading dy and h a second time.
#include "rows_norm_device.hpp"

namespace ul {

namespace {

// Sums over a row's threads, K values at once; the two buffers take turns, so that one barrier is
// enough: a buffer is written again only after the next sum's barrier.
struct LayerLds {
    float v[2][2][16];
};
template <int LANES>
struct LayerSums {
    LayerLds *lds;
    int turn = 0;
    __device__ __forceinline__ void operator()(float (&v)[2])
    {
        v[0] = lanes_sum<LANES ? LANES : 64>(v[0]);
        v[1] = lanes_sum<LANES ? LANES : 64>(v[1]);
        if constexpr (LANES == kBlock) {
            if ((threadIdx.x & 63) == 0) {
                lds->v[turn][0][threadIdx.x >> 6] = v[0];
                lds->v[turn][1][threadIdx.x >> 6] = v[1];
            }
            __syncthreads();
            v[0] = v[1] = 0.0f;
            for (int w = 0; w < (int)(blockDim.x >> 6); ++w) {
                v[0] += lds->v[turn][0][w];
                v[1] += lds->v[turn][1][w];
            }
            turn ^= 1;
        }
    }
};

// Sums of a[i][j] and of a[i][j] b[i][j] over a row.
template <int LANES, int V, int N>
__device__ __forceinline__ void row_sums(LayerSums<LANES> &row, const float (&a)[N][V], const float (&b)[N][V], int me, int TPR,
                                         int cols, float (&sums)[2])
{
    sums[0] = sums[1] = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const Cols<V> c(V * (me + i * TPR), cols);
        float s = 0.0f, q = 0.0f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            s += a[i][j];
            q = fmaf(a[i][j], b[i][j], q);
        }
        if (c.shared()) {
            s = q = 0.0f;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                s = c.counts(j) ? s + a[i][j] : s;
                q = c.counts(j) ? fmaf(a[i][j], b[i][j], q) : q;
            }
        }
        sums[0] += c.live() ? s : 0.0f;
        sums[1] += c.live() ? q : 0.0f;
    }
    row(sums);
}

// What centres a row: e = k (h - mean), rho = 1 / sqrt(mean e^2 + k^2 eps).  k is a power of two, 1 but where
// squares would leave fp32's range: of h, before the mean is taken, or of h - mean, where they would vanish.
struct Spread {
    float rho, k;
    float mean, left;   // e = (k h - mean) - left, or k (h - mean) - left where k > 1
};
template <int LANES, int V, int N>
__device__ __forceinline__ Spread centre(LayerSums<LANES> &row, float (&e)[N][V], int me, int TPR, int cols, float eps)
{
    const float over_cols = 1.0f / (float)cols;
    float sums[2], k = 1.0f, mean;
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
    row_sums<LANES, V, N>(row, e, e, me, TPR, cols, sums);
    if (!(sums[1] < __builtin_inff())) {
        times(0x1p-80f);
        row_sums<LANES, V, N>(row, e, e, me, TPR, cols, sums);
    }
    mean = sums[0] * over_cols;
    less(mean);
    row_sums<LANES, V, N>(row, e, e, me, TPR, cols, sums);
    float left = 0.0f;
    // Values within some 2^-10 of their mean: their differences from it are exact, and so are those from the first
    // one's, which are zeros where the values are equal (differences from a rounded mean would be noise).
    auto from_first = [&] {
        float first[2] = {me == 0 ? e[0][0] : 0.0f, 0.0f};
        row(first);
        less(first[0]);
        left += first[0];
        row_sums<LANES, V, N>(row, e, e, me, TPR, cols, sums);
    };
    if (sums[1] < 0x1p-20f * (mean * mean) * (float)cols) from_first();
    if (k < 1.0f && sums[1] < 0x1p-40f) {   // large, but nearly alike
        times(0x1p80f);
        mean *= 0x1p80f;
        left *= 0x1p80f;
        row_sums<LANES, V, N>(row, e, e, me, TPR, cols, sums);
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
    return {__builtin_amdgcn_rsqf(var + eps * k * k), k, mean, left + rest};
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
    auto read = [&](int64_t t) {
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
#pragma unroll
        for (int i = 0; i < N; ++i) {
            floats_of<TX, V>(a[i], e[i]);
            if (residual.data) {
                float more[V];
                floats_of<TX, V>(r[i], more);
#pragma unroll
                for (int j = 0; j < V; ++j) e[i][j] += more[j];
            }
        }
        if (MORE && t + step < y.rows) read(t + step);
        Raw<TX, V> keep[N];
        if (h.data) {
#pragma unroll
            for (int i = 0; i < N; ++i) keep[i] = raw_of<TX, V>(e[i]);
        }
        const Spread s = centre<LANES, V, N>(row, e, me, TPR, cols, eps);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const Cols<V> c(V * (me + i * TPR), cols);
            if constexpr (!MORE) read_weight(i, w[0], b[0]);
#pragma unroll
            for (int j = 0; j < V; ++j) e[i][j] = fmaf(e[i][j] * s.rho, w[MORE ? i : 0][j], b[MORE ? i : 0][j]);
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
        Raw<TX, V> db_raw[N], ua[N];
        float e[N][V];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            floats_of<TX, V>(a[i], e[i]);
            db_raw[i] = b[i];
            if (dh.data) ua[i] = u[i];
        }
        if (MORE && t + step < dy.rows) read(t + step);
        const Spread s = centre<LANES, V, N>(row, e, me, TPR, cols, eps);
        float g[N][V], sums[2];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const Cols<V> c(V * (me + i * TPR), cols);
            floats_of<TX, V>(db_raw[i], g[i]);
            if constexpr (!MORE) load_weight<V>(weight, c.at, w[0]);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                e[i][j] *= s.rho;   // u
                if constexpr (kInLds) {
                    lds_at(0, i, j) = fmaf(g[i][j], e[i][j], lds_at(0, i, j));
                    lds_at(1, i, j) += g[i][j];
                } else if constexpr (DW) {
                    dw[i][j] = fmaf(g[i][j], e[i][j], dw[i][j]);
                    db[i][j] += g[i][j];
                }
                g[i][j] *= w[MORE ? i : 0][j];
            }
        }
        row_sums<LANES, V, N>(row, g, e, me, TPR, cols, sums);
        const float mean_g = sums[0] * over_cols, along = sums[1] * over_cols;
        if (stats && me == 0) stats[t] = s;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const Cols<V> c(V * (me + i * TPR), cols);
            // in this order: k rho may be beyond fp32's range where dx is not
#pragma unroll
            for (int j = 0; j < V; ++j) g[i][j] = s.k * (s.rho * ((g[i][j] - mean_g) - e[i][j] * along));
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

// Workgroups of the gradient, each of which hands over sums of its rows.
template <int LANES, int VEC>
struct LayerBlocks {
    static int64_t go(RowShape of, int64_t n)
    {
        const RowShape shape = LayerShape<LANES, VEC, UMAP_BF16, UMAP_BF16>::shape(of);
        return even_grid((n + shape.rows - 1) / shape.rows, shape.threads, 16);
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
