// kernels_rows_head.hip -- the head over a table of tokens (umap_rows.h): softmax cross entropy
// and the divergence from a teacher's largest logits, and their gradient.
//
//   z_tv = scale h_t . W_v,  lse_t = log sum_v exp z_tv,  shares q_tv of the row's own tokens v
//   loss_t = sum_v q_tv (log q_tv + lse_t - z_tv)          (cross entropy: one token, q = 1)
//   D_tv = g_t (exp(z_tv - lse_t) - q_tv),  dh = D W,  dW = D^T h,  g_t = dscale scale dloss_t
//
// The logits are never kept.  Forward: a tile of them (rows of the table times rows of h) leaves a maximum and a sum of
// exponentials for each row of h, and its one token's logit; a second launch joins the tiles, and forms the logits of rows of more
// tokens, as dot products.  Gradient: for a piece of the table at a time (D of 256 MB, what the last cache holds) the logits
// are formed anew and D is written in the inputs' type, its entries at the rows' own tokens from those tokens' unrounded p
// and q, which may nearly cancel; then come the two products.  That p is the tile's own or, in 16 bits with more tokens than
// one, comes of the same instructions in the same order: lse comes of the same sums, and what rounding did to them cancels.  With
// p from a dot product in another order, 16-bit entries of 300 rows with partial sums up to 2,300, where p = q, were off by 1.7e-4 to
// 3.7e-4 (medians), so not at all; dh and dW of 77 rows against 2,000 x 64 in fp32 by 8.1e-7 and 9.3e-7 of their norms, so, with the
// lse of the forward call, by 3.2e-7 and 3.1e-7 (medians of 39 inputs).
//
// Precision of D in 16 bits: an entry is off by up to half a unit in its last place, and sums of many entries average that
// out: dW is off by 1.22 (median) to 1.44 times what its own type's rounding alone costs (60 cases of 257 to 700 rows).  Where it
// does not average out it is avoided: up to 256 rows D has two parts, a value and what its rounding left; and a row of dh, most of which often comes from one
// token, gets back what that token's entry lost.  Where all g_t are alike they are left to the very end: D is then p - q, whose
// largest entries, those of the rows' tokens, lie just below 1 and so are rounded least.  Else g_t is a number in [1/2, 1) times
// 2^e_t.  D holds the number; dh gets 2^e_t on the way out, exactly, and dW takes h_t times 2^(e_t - E), E the largest of the rows
// that take part, instead: exact too, down to the smallest exponent of fp32 and bf16.  fp16, which has few exponents, leaves h_t
// as it is: D, 2^15 times as large so that the probabilities of rare tokens are not among its smallest values, holds the number
// times 2^-((E - e_t) mod 6), and the rows of D and of h's copy are put in order of (E - e_t) / 6, their bands, whose sums dW takes one
// after the other from the smallest weights on, times 2^-6 from band to band.  (With h_t times 2^(e_t - E) in fp16, dW of tokens
// that only rows with 2^-20 of the largest weight know was off by 1.7e-2 of its norm, so by 2.8e-4, of which 2.2e-4 is its own
// rounding.)  Weights within 2^6 are one band, in their order, and take no longer (2,048 rows against 32,000 x 4,096 1,413 and 1,423 us,
// 8,000 against 3,000 x 256 171 and 159); weights over 2^40, seven bands, 1,394 -> 1,548 us for the former, 49 -> 65 for 300 rows against
// 10,007 x 300.
//
// Bound by the matrix cores for many rows, by the table's bytes for few.  bf16: 8,192 rows against 128,000 x 4,096: loss 6.1 ms
// (1,400 TFLOP/s; the library's product of the same size 5.8 ms, without the exponentials), gradient 20.2 ms (1,280: D 0.84,
// dh 0.82 and dW 0.84 ms of each of 8 pieces); one row against 32,000 x 2,048: 22 us of the tiles (6.0 TB/s) and 4 of
// their join.  Fewer columns leave a tile less to multiply before its end: 2,048 rows against 32,000 reach 1,350 TFLOP/s at 4,096
// columns, 910 at 512.
#include <math.h>

#include <algorithm>

#include "launch_sizes.hpp"
#include "rows_product.hpp"

namespace ul {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
__device__ __forceinline__ float minus_inf() { return -__builtin_inff(); }

// What the tiles' exponentials are of, and to what base: 16-bit types' logits are in units of log 2, so that a product
// and a sum with one rounding lead to the hardware's 2^x; fp32's are in natural units and go through expf, since their
// results are not rounded any further.
template <int T>
struct Logit {
    float unit;   // times a dot product: a logit
    __device__ __forceinline__ explicit Logit(float scale) : unit(T == UMAP_F32 ? scale : scale * kLog2e) {}
    static __device__ __forceinline__ float exp(float x) { return T == UMAP_F32 ? expf(x) : __builtin_amdgcn_exp2f(x); }
    static __device__ __forceinline__ float log(float x) { return T == UMAP_F32 ? logf(x) : __builtin_amdgcn_logf(x); }
    static __device__ __forceinline__ float natural(float x) { return T == UMAP_F32 ? x : x * kLn2; }
    static __device__ __forceinline__ float of_natural(float x) { return T == UMAP_F32 ? x : x * kLog2e; }
    // exp(dot's logit - less)
    __device__ __forceinline__ float exp_less(float dot, float less) const
    {
        return T == UMAP_F32 ? expf(dot * unit - less) : __builtin_amdgcn_exp2f(fmaf(dot, unit, -less));
    }
};

// Largest logit and sum of exp(logit - largest).
struct MaxSum {
    float m, s;
    // Values to subtract from: a largest of -inf (no value yet, or all of them) subtracts nothing.
    static __device__ __forceinline__ float base(float m) { return m == minus_inf() ? 0.0f : m; }
    template <int T>
    __device__ __forceinline__ void join(MaxSum o)
    {
        const float most = fmaxf(m, o.m), b = base(most);
        s = fmaf(s, Logit<T>::exp(m - b), o.s * Logit<T>::exp(o.m - b));
        m = most;
    }
};

__device__ __forceinline__ float wave_sum(float v)
{
    for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
    return v;
}

// ---- the logits' tiles: forward -------------------------------------------------------------

// The one tokens of a wave's 16 FN rows of B, a row to a lane, in the wave's part of a tile.  Few waves have one there, and the
// others see it at once.
template <class P>
struct OwnPlaces {
    static_assert(P::kFN <= 4, "a lane to a row");
    int at = -1;   // rows of A from the wave's first
    uint64_t rows;
    // This lane's row, from the tile's first; behind the wave's rows: no row.
    static __device__ __forceinline__ int row(int none)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        return lane < 16 * P::kFN ? wave % P::kWN * 16 * P::kFN + lane : none;
    }
    // own: rows of A from the tile's first, negative: none
    __device__ __forceinline__ explicit OwnPlaces(int64_t own)
    {
        const int64_t in = own - P::m_first(0);
        if (own >= 0 && in >= 0 && in < 16 * P::kFM) at = (int)in;
        rows = __ballot(at >= 0);
    }
    __device__ __forceinline__ bool any(int j) const { return (rows >> (16 * j) & 0xffff) != 0; }
    // acc[i][j][r] is a row's own token's where this is 16 i + r.
    __device__ __forceinline__ int place(int j) const { return __shfl(at, 16 * j + (threadIdx.x & 15)) - (int)(threadIdx.x >> 4 & 3) * 4; }
    // Its acc, or 0.
    static __device__ __forceinline__ float pick(int place, const Acc4 (&acc)[P::kFM][P::kFN], int j)
    {
        float x = 0.0f;
#pragma unroll
        for (int i = 0; i < P::kFM; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) x = place == 16 * i + r ? acc[i][j][r] : x;
        return x;
    }
    // Whether this lane has it.
    static __device__ __forceinline__ bool here(int place) { return place >= 0 && (place & 15) < 4; }
};

// Rows of one token each: its logit, as it is among the exponentials, in their units.
struct OwnLogits {
    RowIds ids;
    int64_t first;   // row of h's first
    int64_t vocab, piece;   // rows of the table, and which of them w's first is
    float *z;        // null: rows of more tokens
    // An id as it lies in memory, for a load that nobody waits for before id().
    struct Words {
        int32_t low, high;
    };
    __device__ __forceinline__ Words fetch(int64_t t) const
    {
        const auto *const at = reinterpret_cast<const int32_t *>(static_cast<const char *>(ids.data) + (first + t) * ids.bytes);
        return {at[0], at[ids.bytes / 4 - 1]};
    }
    __device__ __forceinline__ int64_t id(const Words &w) const
    {
        const int64_t v = ids.bytes == 4 ? (int64_t)w.low : (int64_t)w.high << 32 | (uint32_t)w.low;
        return v >= 0 && v < vocab ? v : -1;
    }
};

template <int T, class P>
__global__ __launch_bounds__(P::kThreads) void k_head_lse(ProductSide w, ProductSide h, float scale, Tiles tiles, int64_t first_tile,
                                                          int64_t all_tiles, MaxSum *partial, OwnLogits one)
{
    __shared__ __align__(16) Piece lds[P::kLds / 16];
    constexpr int FM = P::kFM, FN = P::kFN;
    const TileAt at = tile_at(tiles, blockIdx.x);
    const int64_t m0 = (int64_t)at.m * P::M, n0 = (int64_t)at.n * P::N;
    Acc4 acc[FM][FN];
    P::run(w, h, m0, n0, 0, w.cols, lds, acc);
    OwnLogits::Words own = {};   // on its way while the exponentials are formed
    if (one.z) own = one.fetch(min(n0 + OwnPlaces<P>::row(0), h.rows - 1));
    MaxSum(*const part)[P::N] = reinterpret_cast<MaxSum(*)[P::N]>(lds);   // behind the product's last barrier
    const int live = (int)min((int64_t)P::M, w.rows - m0);
    Logit<T> logit(scale);
    if (live < P::M || logit.unit < 0.0f) {   // the largest is the largest product's but here
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[i][j][r] = P::m_of(i) + r < live ? acc[i][j][r] * logit.unit : minus_inf();
        logit.unit = 1.0f;
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        float most = minus_inf();
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) most = fmaxf(most, acc[i][j][r]);
        if (most != minus_inf()) most *= logit.unit;
        const float b = MaxSum::base(most);
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) sum += logit.exp_less(acc[i][j][r], b);
        MaxSum all{most, sum};
#pragma unroll
        for (int o = 16; o < 64; o <<= 1) all.template join<T>({__shfl_xor(all.m, o), __shfl_xor(all.s, o)});
        if ((threadIdx.x & 63) < 16) part[(threadIdx.x >> 6) / P::kWN][P::n_of(j)] = all;
    }
    if (one.z) {
        const int row = OwnPlaces<P>::row(-1);
        const OwnPlaces<P> places(row >= 0 && n0 + row < h.rows ? one.id(own) - one.piece - m0 : -1);
        if (places.rows) {
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                if (!places.any(j)) continue;
                const int place = places.place(j);
                const float z = OwnPlaces<P>::pick(place, acc, j) * logit.unit;
                if (OwnPlaces<P>::here(place)) one.z[n0 + P::n_of(j)] = z;
            }
        }
    }
    __syncthreads();
    for (int n = threadIdx.x; n < P::N; n += P::kThreads) {
        if (n0 + n >= h.rows) continue;
        MaxSum all = part[0][n];
#pragma unroll
        for (int i = 1; i < P::kWM; ++i) all.template join<T>(part[i][n]);
        partial[(n0 + n) * all_tiles + first_tile + at.m] = all;
    }
}

// ---- a row's own tokens ----------------------------------------------------------------------

constexpr int kMostTokens = 256;   // of a row

struct Taught {
    RowIds ids;
    int32_t k;
    const void *teacher;   // null: one token a row
    int64_t stride;
    int32_t type;
    float scale;
};

__device__ __forceinline__ float teacher_at(const Taught &x, int64_t t, int e)
{
    switch (x.type) {
    case UMAP_F32: return static_cast<const float *>(x.teacher)[t * x.stride + e];
    case UMAP_F16: return elem_float<UMAP_F16>(static_cast<const _Float16 *>(x.teacher)[t * x.stride + e]);
    default: return elem_float<UMAP_BF16>(static_cast<const uint16_t *>(x.teacher)[t * x.stride + e]);
    }
}

// A row has a wave (up to 64 tokens) or a workgroup of 4 or 16; each thread one of its tokens.
template <int WAVES>
struct RowTeam {
    static constexpr int kThreads = 64 * WAVES, kRows = WAVES == 1 ? 4 : 1, kBlock = kThreads * kRows;   // of a workgroup
    struct Lds {
        float part[WAVES];
        int id[kMostTokens];
        float share[kMostTokens], z[kMostTokens];
    };
    Lds *lds;
    int me, wave;   // in the row
    __device__ __forceinline__ explicit RowTeam(Lds *l)
        : lds(l), me(threadIdx.x % kThreads), wave(WAVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6))
    {
    }
    template <typename Op>
    __device__ __forceinline__ float all(float v, Op op) const
    {
        for (int o = 1; o < 64; o <<= 1) v = op(v, __shfl_xor(v, o));
        if constexpr (WAVES > 1) {
            __syncthreads();
            if ((me & 63) == 0) lds->part[wave] = v;
            __syncthreads();
            v = lds->part[0];
#pragma unroll
            for (int i = 1; i < WAVES; ++i) v = op(v, lds->part[i]);
        }
        return v;
    }
    __device__ __forceinline__ float sum(float v) const { return all(v, [](float a, float b) { return a + b; }); }
    __device__ __forceinline__ float max(float v) const { return all(v, [](float a, float b) { return fmaxf(a, b); }); }
    // Token e's value, for all threads.
    __device__ __forceinline__ int of(int v, const int *shared, int e) const
    {
        return WAVES == 1 ? __builtin_amdgcn_readlane(v, e) : __builtin_amdgcn_readfirstlane(shared[e]);
    }
    __device__ __forceinline__ float of(float v, const float *shared, int e) const
    {
        return WAVES == 1 ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), e)) : shared[e];
    }
};

// This thread's token: id (-1: none) and share.
template <int WAVES>
struct OwnToken {
    int id = -1;
    float share, log_share = minus_inf();
    bool any;
    bool alone = false;   // all threads have the row's one token
    __device__ __forceinline__ OwnToken(const RowTeam<WAVES> &team, const Taught &x, int64_t t, int64_t rows)
    {
        if (!x.teacher) {   // one token, which all threads know
            id = (int)row_of(x.ids, t, rows);
            share = 1.0f;
            log_share = 0.0f;
            any = id >= 0;
            alone = true;
            return;
        }
        if (team.me < x.k) id = (int)row_of(x.ids, t * x.k + team.me, rows);
        float logit = minus_inf();   // the largest of these counts 1
        if (id >= 0) {
            const float a = teacher_at(x, t, team.me);
            if (a == minus_inf()) id = -1;
            else logit = x.scale < 0.0f ? -a : a;
        }
        if (WAVES > 1 && team.me < kMostTokens) team.lds->id[team.me] = id;   // read behind the reductions' barriers
        // the difference first: it is in fp32's range, or far below, where a product with the scale may not be
        const float less = logit - MaxSum::base(team.max(logit));
        log_share = (less == minus_inf() ? -__FLT_MAX__ : less) * fabsf(x.scale);   // the scale may be 0
        share = id >= 0 ? expf(log_share) : 0.0f;   // not rounded any further in fp32, nor in the loss
        const float sum = team.sum(share);
        any = !(sum == 0.0f);   // the largest counts 1
        share = id >= 0 ? share / sum : 0.0f;
        log_share -= logf(sum);
        if constexpr (WAVES > 1) {
            if (team.me < kMostTokens) team.lds->share[team.me] = share;
            __syncthreads();
        }
    }
};

// All shares of a thread's token in its row: of a token that comes twice the first place has them, the others none.
template <int WAVES>
__device__ __forceinline__ float all_shares(const RowTeam<WAVES> &team, const OwnToken<WAVES> &own, int k)
{
    if (own.alone) return own.share;
    float share = 0.0f;
    bool again = false;
#pragma unroll 8
    for (int o = 0; o < k; ++o) {
        const int other = team.of(own.id, team.lds->id, o);
        const float more = team.of(own.share, team.lds->share, o);
        if (other != own.id) continue;
        share += more;
        again |= o < team.me;
    }
    return again ? -1.0f : share;
}

template <int T>
__device__ __forceinline__ void fetch8(const Elem<T> *row, int c, int cols, float v[8])
{
    if (c + 8 <= cols) {
        floats_of<T, 8>(load_raw<T, 8>(row + c), v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c + j < cols ? elem_float<T>(row[c + j]) : 0.0f;
    }
}

// Logits of a row's k tokens, as dot products with the table's rows: each thread's token's.
template <int T, int WAVES>
__device__ __forceinline__ float own_logit(const RowTeam<WAVES> &team, const Elem<T> *h, const ProductSide &w,
                                           const OwnToken<WAVES> &own, int k, float scale)
{
    constexpr int kAtOnce = 4;
    const int cols = (int)w.cols, lane = team.me & 63;
    float z = 0.0f;
    // a wave to a token, whose number and row all its lanes know
    for (int e0 = kAtOnce * team.wave; cols > 256 && e0 < k; e0 += kAtOnce * WAVES) {
        const Elem<T> *row[kAtOnce];
        float sum[kAtOnce] = {};
        int id[kAtOnce];
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
            id[q] = e0 + q < k ? team.of(own.id, team.lds->id, e0 + q) : -1;
            row[q] = static_cast<const Elem<T> *>(w.data) + (int64_t)max(id[q], 0) * w.stride;
        }
        for (int c = lane * 8; c < cols; c += 512) {
            float a[8];
            fetch8<T>(h, c, cols, a);
#pragma unroll
            for (int q = 0; q < kAtOnce; ++q) {
                if (id[q] < 0) continue;
                float b[8];
                fetch8<T>(row[q], c, cols, b);
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[q] = fmaf(a[j], b[j], sum[q]);
            }
        }
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
            const float all = wave_sum(sum[q]) * scale;
            if constexpr (WAVES == 1) z = lane == e0 + q ? all : z;
            else if (lane == 0) team.lds->z[e0 + q] = all;
        }
    }
    // few columns: `lanes` lanes to a token, as many tokens side by side as a wave then has, kAtOnce times
    const int lanes = cols <= 64 ? 8 : cols <= 128 ? 16 : 32, side = 64 / lanes, sub = lane / lanes;
    for (int e0 = kAtOnce * side * team.wave; cols <= 256 && e0 < k; e0 += kAtOnce * side * WAVES) {
        const Elem<T> *row[kAtOnce];
        float sum[kAtOnce] = {};
        bool there[kAtOnce];
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
            const int e = e0 + q * side + sub;
            const int id = WAVES == 1 ? __shfl(own.id, min(e, 63)) : team.lds->id[min(e, kMostTokens - 1)];
            there[q] = e < k && id >= 0;
            row[q] = static_cast<const Elem<T> *>(w.data) + (int64_t)(there[q] ? id : 0) * w.stride;
        }
        for (int c = (lane % lanes) * 8; c < cols; c += 8 * lanes) {
            float a[8];
            fetch8<T>(h, c, cols, a);
#pragma unroll
            for (int q = 0; q < kAtOnce; ++q) {
                if (!there[q]) continue;
                float b[8];
                fetch8<T>(row[q], c, cols, b);
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[q] = fmaf(a[j], b[j], sum[q]);
            }
        }
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
            for (int o = 1; o < lanes; o <<= 1) sum[q] += __shfl_xor(sum[q], o);
            const int e = e0 + q * side + sub;
            if constexpr (WAVES == 1) {
                for (int s = 0; s < side; ++s) {
                    const float other = __shfl(sum[q], s * lanes);
                    z = lane == e0 + q * side + s ? other * scale : z;
                }
            } else if (lane % lanes == 0 && e < kMostTokens) {
                team.lds->z[e] = sum[q] * scale;
            }
        }
    }
    if constexpr (WAVES > 1) {
        __syncthreads();
        z = team.me < k ? team.lds->z[team.me] : 0.0f;
    }
    return z;
}

template <int T>
__device__ __forceinline__ Piece piece_at(const Elem<T> *p)
{
    return __builtin_bit_cast(Piece, load_raw<T, 16 / (int)sizeof(Elem<T>)>(p));
}

// The same in 16 bits, without the scale, by the tiles' instructions in the tiles' order, 16 tokens by a wave: they round as the
// tiles' do.  (fp32's instruction takes 16 times the cycles of the products that are wanted: a loss of 1,000 rows with 33 tokens
// each against 3,000 x 3,000 would take 230 us instead of 187.)
template <int T, int WAVES>
__device__ __forceinline__ float own_dot(const RowTeam<WAVES> &team, const Elem<T> *h, const ProductSide &w, const OwnToken<WAVES> &own, int k)
{
    constexpr int kPer = 8, kHalf = 4 * kPer;   // columns of a piece, and of a half step
    const int cols = (int)w.cols, lane = team.me & 63, g = lane >> 4;
    const Elem<T> *const mine = h + g * kPer;
    float z = 0.0f;
    for (int e0 = 16 * team.wave; e0 < k; e0 += 16 * WAVES) {
        const int e = e0 + (lane & 15), id = WAVES == 1 ? __shfl(own.id, min(e, 63)) : team.lds->id[min(e, kMostTokens - 1)];
        const Elem<T> *const row = static_cast<const Elem<T> *>(w.data) + (int64_t)(e < k ? max(id, 0) : 0) * w.stride + g * kPer;
        Acc4 dot = {0.0f, 0.0f, 0.0f, 0.0f};
        int c = 0;
        auto pieces = [&](auto count) {
            constexpr int N = decltype(count)::value;
            for (; c + N * kHalf <= cols; c += N * kHalf) {
                Piece a[N], b[N] = {};
#pragma unroll
                for (int q = 0; q < N; ++q) a[q] = piece_at<T>(row + c + q * kHalf);
                if ((lane & 15) == 0) {   // of the product's 16 columns one is looked at
#pragma unroll
                    for (int q = 0; q < N; ++q) b[q] = piece_at<T>(mine + c + q * kHalf);
                }
#pragma unroll
                for (int q = 0; q < N; ++q) dot = multiply<T>(a[q], b[q], dot);
            }
        };
        pieces(std::integral_constant<int, 4>{});
        pieces(std::integral_constant<int, 1>{});
        if (c < cols) {   // past the last column: zeros
            float a[kPer], b[kPer];
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const bool there = c + g * kPer + j < cols;
                a[j] = there ? elem_float<T>(row[c + j]) : 0.0f;
                b[j] = there ? elem_float<T>(mine[c + j]) : 0.0f;
            }
            dot = multiply<T>(__builtin_bit_cast(Piece, raw_of<T, kPer>(a)), __builtin_bit_cast(Piece, raw_of<T, kPer>(b)), dot);
        }
        // lanes 16 g have tokens e0 + 4 g .. + 3
        if constexpr (WAVES == 1) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float other = __shfl(dot[r], (lane & 12) * 4);
                z = lane >> 4 == e0 >> 4 && (lane & 3) == r ? other : z;
            }
        } else if ((lane & 15) == 0) {
#pragma unroll
            for (int r = 0; r < 4; ++r) team.lds->z[e0 + 4 * g + r] = dot[r];
        }
    }
    if constexpr (WAVES > 1) {
        __syncthreads();
        z = team.me < k ? team.lds->z[team.me] : 0.0f;
    }
    return z;
}

// A copy of rows for the products, in whole pieces of 16 bytes: `pitch` columns, zeros past the last.
template <int T>
__global__ __launch_bounds__(256) void k_head_pack(ProductSide from, Elem<T> *to, int pitch)
{
    const int64_t total = from.rows * (pitch / 8);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / (pitch / 8);
        const int c = (int)(i % (pitch / 8)) * 8;
        float v[8] = {};
        if (c < from.cols) fetch8<T>(static_cast<const Elem<T> *>(from.data) + r * from.stride, c, (int)from.cols, v);
        store_raw<T, 8>(to + r * pitch + c, raw_of<T, 8>(v));
    }
}

// Joins a row's tiles, and sums its loss.
template <int T, int WAVES>
__global__ __launch_bounds__(RowTeam<WAVES>::kBlock) void k_head_loss(ProductSide w, ProductSide h, float scale, Taught taught, int64_t first,
                                                   int64_t tiles, const MaxSum *partial, const float *one, float *loss, float *lse)
{
    __shared__ typename RowTeam<WAVES>::Lds lds;
    const RowTeam<WAVES> team(&lds);
    const int64_t t = (int64_t)blockIdx.x * RowTeam<WAVES>::kRows + threadIdx.x / RowTeam<WAVES>::kThreads;
    if (t >= h.rows) return;
    MaxSum mine{minus_inf(), 0.0f};
    for (int64_t i = team.me; i < tiles; i += RowTeam<WAVES>::kThreads) mine.template join<T>(partial[t * tiles + i]);
    const OwnToken<WAVES> own(team, taught, first + t, w.rows);
    float z;
    if (one) z = Logit<T>::natural(one[t]);
    else z = own_logit<T, WAVES>(team, static_cast<const Elem<T> *>(h.data) + t * h.stride, w, own, taught.k, scale);
    const float most = team.max(mine.m);
    const float sum = Logit<T>::natural(most + Logit<T>::log(team.sum(mine.s * Logit<T>::exp(mine.m - MaxSum::base(most)))));
    const float share = all_shares(team, own, taught.k);   // > 0, or NaN, where there is one
    const float log_share = share == own.share ? own.log_share : logf(share);
    float all = own.id >= 0 && !(share <= 0.0f) ? share * (log_share + (sum - z)) : 0.0f;
    if (!own.alone) all = team.sum(all);
    if (team.me == 0) {
        lse[first + t] = sum;
        // rounding can take a loss of nearly nothing below it
        loss[first + t] = !own.any ? 0.0f : all < 0.0f ? 0.0f : all;
    }
}

// ---- gradient --------------------------------------------------------------------------------

constexpr int kNoRow = INT32_MIN;
template <int T>
constexpr int kShift = T == UMAP_F16 ? 15 : 0;

// What the gradient's launches share of a row: its number in [1/2, 1), with kShift, and its exponent.
struct RowWeights {
    float *number;
    int *exponent;   // kNoRow: the row takes no part
    const int *largest;   // null, and the numbers 1, the exponents 0: all rows have the weight `all`
    float all;            // times it and 2^power, what the products give
    int power;
};
// x times 2^power, x in [1/2, 1) or 0.
struct Factor {
    float x;
    int power;
};
__device__ __forceinline__ int largest_of(const RowWeights &x) { return x.largest ? *x.largest : 0; }

// fp16's rows of different weights: where a row lies in D and in h's copy, what its entries are times, and where the bands
// begin (and the last ends), and the last one that has rows.  Null: each in its own place, times 1, one band.
struct RowPlaces {
    const int *slot;
    const float *shrink;
    const int *start;   // kBands + 2
};
constexpr int kBandBits = 6, kBands = 16;
// Of a row's exponent.  Rows beyond the last band, 2^-96 of the largest weight, are not seen by dW.
struct Band {
    int band, less;
    bool lost;
    __device__ __forceinline__ Band(int exponent, int largest)
    {
        const int off = exponent == kNoRow ? 0 : largest - exponent;
        lost = off >= kBandBits * kBands;
        band = lost ? kBands - 1 : off / kBandBits;
        less = lost ? 0 : off % kBandBits;
    }
};

__device__ __forceinline__ void split_weight(float g, float &number, int &exponent)
{
    exponent = 0;
    number = g;
    if (g != 0.0f && fabsf(g) < __builtin_inff()) {
        number = __builtin_amdgcn_frexp_mantf(g);
        exponent = __builtin_amdgcn_frexp_expf(g);
    }
}

// The largest and the smallest exponent of the rows that take part, found by one of WAVES waves' threads; 0 where there is none.
struct Exponents {
    int most, least;
};
template <int WAVES>
__device__ __forceinline__ Exponents exponents_of(const int *exponent, int64_t n)
{
    __shared__ Exponents part[WAVES];
    Exponents x{kNoRow, INT32_MAX};
    for (int64_t t = threadIdx.x; t < n; t += 64 * WAVES) {
        const int e = exponent[t];
        x.most = max(x.most, e);
        if (e != kNoRow) x.least = min(x.least, e);
    }
    for (int o = 1; o < 64; o <<= 1) {
        x.most = max(x.most, __shfl_xor(x.most, o));
        x.least = min(x.least, __shfl_xor(x.least, o));
    }
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WAVES; ++i) x = {max(x.most, part[i].most), min(x.least, part[i].least)};
    return x.most == kNoRow ? Exponents{0, 0} : x;
}
__global__ __launch_bounds__(1024) void k_head_largest(const int *exponent, int64_t n, Exponents *found)
{
    const Exponents x = exponents_of<16>(exponent, n);
    if (threadIdx.x == 0) *found = x;
}

// The rows' copies times 2^(e_t - E): `rows` of them, `parts` times one after the other.  With few rows every workgroup
// finds the largest exponent for itself, and the first leaves it to the launches that follow.
constexpr int64_t kFindRows = 8192;
template <int T>
__global__ __launch_bounds__(256) void k_head_scale(const Elem<T> *copy, int64_t rows, int parts, int pitch, const int *exponent,
                                                    Exponents *found, Elem<T> *scaled)
{
    const int64_t total = rows * (pitch / 8);
    int most;
    if (rows <= kFindRows) {
        const Exponents x = exponents_of<4>(exponent, rows);
        most = x.most;
        if (blockIdx.x == 0 && threadIdx.x == 0) *found = x;
    } else {
        most = found->most;
    }
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t t = i / (pitch / 8);
        const int by = exponent[t] == kNoRow ? 0 : exponent[t] - most;
        float v[8];
        floats_of<T, 8>(load_raw<T, 8>(copy + i * 8), v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = ldexpf(v[j], by);
        for (int p = 0; p < parts; ++p) store_raw<T, 8>(scaled + p * rows * pitch + i * 8, raw_of<T, 8>(v));
    }
}

// fp16's order of many rows: their places by band, in a band by number, unless there is one band only.  Each thread takes a
// stretch of the rows.
__global__ __launch_bounds__(1024) void k_head_order(const int *exponent, int64_t n, Exponents *found, int *slot, float *shrink, int *start)
{
    static_assert(kBands == 16, "a wave to a band");
    __shared__ int count[kBands][1024], base[kBands + 1];
    const Exponents x = exponents_of<16>(exponent, n);
    const int me = threadIdx.x, wave = me >> 6, lane = me & 63;
    const int64_t each = (n + 1023) / 1024, first = me * each, last = min(first + each, n);
    if (me == 0) *found = x;
    if (x.most - x.least < kBandBits) {
        if (me <= kBands + 1) start[me] = me == 0 || me > kBands ? 0 : (int)n;
        return;
    }
    for (int b = 0; b < kBands; ++b) count[b][me] = 0;
    for (int64_t t = first; t < last; ++t) ++count[Band(exponent[t], x.most).band][me];
    __syncthreads();
    int sum = 0;
    for (int i = 0; i < 16; ++i) sum += count[wave][lane * 16 + i];
    int before = sum;   // and those of the lanes below
    for (int o = 1; o < 64; o <<= 1) {
        const int other = __shfl_up(before, o);
        if (lane >= o) before += other;
    }
    if (lane == 63) base[wave + 1] = before;
    before -= sum;
    for (int i = 0; i < 16; ++i) {
        const int here = count[wave][lane * 16 + i];
        count[wave][lane * 16 + i] = before;
        before += here;
    }
    __syncthreads();
    if (me == 0) {
        int top = 0;
        base[0] = 0;
        for (int b = 1; b <= kBands; ++b) {
            if (base[b]) top = b - 1;
            base[b] += base[b - 1];
        }
        start[kBands + 1] = top;
    }
    __syncthreads();
    if (me <= kBands) start[me] = base[me];
    for (int64_t t = first; t < last; ++t) {
        const Band band(exponent[t], x.most);
        slot[t] = base[band.band] + count[band.band][me]++;
        shrink[t] = ldexpf(1.0f, -band.less);
    }
}

// fp16's copies of the rows, unscaled, in that order.  With few rows every workgroup finds the exponents and, where there is more
// than one band, counts its rows' places among all; the first leaves the bands to the launches that follow.
__global__ __launch_bounds__(256) void k_head_place(const Elem<UMAP_F16> *copy, int64_t rows, int parts, int pitch, const int *exponent,
                                                    Exponents *found, Elem<UMAP_F16> *placed, int *slot, float *shrink, int *start)
{
    constexpr int T = UMAP_F16;
    __shared__ int part[4], count[kBands];
    const bool finds = rows <= kFindRows;
    const int64_t per = pitch / 8, total = rows * per;
    const Exponents x = finds ? exponents_of<4>(exponent, rows) : *found;
    const bool many = x.most - x.least >= kBandBits, counts = finds && many;
    if (finds && blockIdx.x == 0) {
        if (threadIdx.x == 0) *found = x;
        if (many) {
            if (threadIdx.x < kBands) count[threadIdx.x] = 0;
            __syncthreads();
            for (int t = threadIdx.x; t < (int)rows; t += 256) atomicAdd(&count[Band(exponent[t], x.most).band], 1);
            __syncthreads();
            if (threadIdx.x == 0) {
                int before = 0, top = 0;
                for (int b = 0; b < kBands; ++b) {
                    start[b] = before;
                    before += count[b];
                    if (count[b]) top = b;
                }
                start[kBands] = before;
                start[kBands + 1] = top;
            }
        } else if (threadIdx.x <= kBands + 1) {
            start[threadIdx.x] = threadIdx.x == 0 || threadIdx.x > kBands ? 0 : (int)rows;
        }
    }
    for (int64_t i0 = (int64_t)blockIdx.x * 256; i0 < total; i0 += (int64_t)gridDim.x * 256) {
        const int64_t i = i0 + threadIdx.x, t = i / per;
        const int c = (int)(i - t * per);
        int64_t to = t;
        if (!finds && many && i < total) to = slot[t];
        if (counts) {
            for (int row = (int)(i0 / per), last = (int)((min(i0 + 256, total) - 1) / per); row <= last; ++row) {
                const int band = Band(exponent[row], x.most).band;
                int before = 0;
                for (int u = threadIdx.x; u < (int)rows; u += 256) {
                    const int other = Band(exponent[u], x.most).band;
                    before += other < band || (other == band && u < row);
                }
                for (int o = 1; o < 64; o <<= 1) before += __shfl_xor(before, o);
                __syncthreads();
                if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = before;
                __syncthreads();
                if (t == row) to = part[0] + part[1] + part[2] + part[3];
            }
        }
        if (i >= total) continue;
        const Band band(exponent[t], x.most);
        if ((finds || !many) && c == 0) {
            slot[t] = (int)to;
            shrink[t] = ldexpf(1.0f, -band.less);
        }
        Raw<T, 8> v = {};
        if (!band.lost) v = load_raw<T, 8>(copy + i * 8);
        for (int p = 0; p < parts; ++p) store_raw<T, 8>(placed + (p * rows + to) * pitch + c * 8, v);
    }
}

// What rounding takes from a row's largest entry at its own tokens, where D has one 16-bit part: dh's rows get it back in
// fp32 at the end, since it alone would be off as a whole (a row's token often has most of its gradient).
struct RowRests {
    int *token;    // null: none; -1: none for the row
    float *rest;
};

// A row's weight, its tokens with the entries of D, and its copy for the products, without gaps (`pitch` columns, zeros
// past the last), zeros in rows without part, and once for each part of D.
template <int T, int WAVES>
__global__ __launch_bounds__(RowTeam<WAVES>::kBlock) void k_head_rows(ProductSide w, ProductSide h, float scale, Taught taught, const float *lse,
                                                   const float *dloss, Factor factor, RowWeights weights, int *token,
                                                   float *value, RowRests rests, Elem<T> *copy, int pitch, int parts)
{
    __shared__ typename RowTeam<WAVES>::Lds lds;
    const RowTeam<WAVES> team(&lds);
    const int64_t t = (int64_t)blockIdx.x * RowTeam<WAVES>::kRows + threadIdx.x / RowTeam<WAVES>::kThreads;
    if (t >= h.rows) return;
    const Elem<T> *const row = static_cast<const Elem<T> *>(h.data) + t * h.stride;
    const OwnToken<WAVES> own(team, taught, t, w.rows);
    float number = 1.0f;
    int exponent = 0;
    if (dloss) {   // both factors in parts, since their product may be in fp32's range where one of them is not
        int more;
        split_weight(dloss[t], number, exponent);
        split_weight(number * factor.x, number, more);
        exponent += more + factor.power;
    }
    const bool part = own.any && number != 0.0f && factor.x != 0.0f;
    number = ldexpf(number, kShift<T>);
    const bool in_tile = T == UMAP_F32 || taught.k == 1;   // p is then taken from the tile, value from number p
    float p = 0.0f;
    if constexpr (T != UMAP_F32) {
        if (!in_tile) p = Logit<T>(scale).exp_less(own_dot<T, WAVES>(team, row, w, own, part ? taught.k : 0), Logit<T>::of_natural(lse[t]));
    }
    int id = part ? own.id : -1;
    const float share = all_shares(team, own, taught.k);
    if (share < 0.0f) id = -1;
    if (team.me >= taught.k) id = -1;
    float entry = 0.0f;
    if (id >= 0) entry = number * (in_tile ? share : p - share);
    if (team.me < taught.k) {
        token[t * taught.k + team.me] = id;
        value[t * taught.k + team.me] = entry;
    }
    if (rests.token && in_tile) {
        if (team.me == 0) rests.token[t] = id;   // the rest is the tile's too
    } else if (rests.token) {
        // of the largest entry (to 2^-15): its magnitude and its place as one number
        const uint32_t key = (__float_as_uint(fabsf(entry)) & ~255u) | (255u - team.me);
        const float most = team.max(id >= 0 ? __uint_as_float(key) : -1.0f);
        const int place = most < 0.0f ? kMostTokens : 255 - (int)(__float_as_uint(most) & 255u);
        if (team.me == place) rests.rest[t] = entry - elem_float<T>(float_elem<T>(entry));
        if (team.me == (place < kMostTokens ? place : 0)) rests.token[t] = place < kMostTokens ? id : -1;
    }
    if (team.me == 0) {
        weights.number[t] = part ? number : 0.0f;
        weights.exponent[t] = part ? exponent : kNoRow;
    }
    for (int c = team.me * 8; c < pitch; c += RowTeam<WAVES>::kThreads * 8) {
        float v[8] = {};
        if (part) fetch8<T>(row, c, (int)h.cols, v);
        for (int p = 0; p < parts; ++p) store_raw<T, 8>(copy + (p * h.rows + t) * pitch + c, raw_of<T, 8>(v));
    }
}

// Rounds to type T, and leaves in v what the rounding took away.
template <int T, int V>
__device__ __forceinline__ Raw<T, V> rounded(float (&v)[V])
{
    const Raw<T, V> r = raw_of<T, V>(v);
    float back[V];
    floats_of<T, V>(r, back);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] -= back[i];
    return r;
}

// Two fragments' rows of A, one above the other, as 8 next to each other.  A lane has 4 of each; the hardware swaps the
// odd groups of 16 lanes of the first with the even groups of the second, so that a lane has 8 of one of them and a store
// instruction 64 bytes of every row: rows first + pair_row() on.
template <int T>
__device__ __forceinline__ Raw<T, 8> pair_of(const Raw<T, 4> &a, const Raw<T, 4> &b)
{
    Raw<T, 8> r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const auto s = __builtin_amdgcn_permlane16_swap(a.w[i], b.w[i], false, false);
        r.w[i] = s[0];
        r.w[2 + i] = s[1];
    }
    return r;
}
__device__ __forceinline__ int pair_row()
{
    const int g = threadIdx.x >> 4 & 3;
    return (g & 1) * 16 + (g >> 1) * 8;
}

// D of a piece of the table: d[t][v], `pitch` columns, zeros past the piece's rows.  token and value: null, or each
// row's one token and what number p is less of there; rest: null, or receives what rounding takes from that entry.
template <int T, class P>
__global__ __launch_bounds__(P::kThreads) void k_head_d(ProductSide w, ProductSide h, float scale, Tiles tiles, const float *lse,
                                                        RowWeights weights, RowPlaces places, const int *token, const float *value,
                                                        float *rest, int64_t first, Elem<T> *d, int64_t pitch, int64_t below)
{
    __shared__ __align__(16) Piece lds[P::kLds / 16];
    constexpr int FM = P::kFM, FN = P::kFN;
    const TileAt at = tile_at(tiles, blockIdx.x);
    const int64_t m0 = (int64_t)at.m * P::M, n0 = (int64_t)at.n * P::N;
    Acc4 acc[FM][FN];
    P::run(w, h, m0, n0, 0, w.cols, lds, acc);
    const int live = (int)min((int64_t)P::M, w.rows - m0);
    const Logit<T> logit(scale);
    const int row = OwnPlaces<P>::row(-1), own = token && row >= 0 && n0 + row < h.rows ? token[n0 + row] : -1;
    const OwnPlaces<P> tokens(own >= 0 ? own - first - m0 : -1);
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const int64_t t = n0 + P::n_of(j);
        const int place = tokens.any(j) ? tokens.place(j) : -1;   // of all lanes
        if (t >= h.rows) continue;
        const float shrink = T == UMAP_F16 && places.slot ? places.shrink[t] : 1.0f;
        const float number = weights.number[t] * shrink, less = Logit<T>::of_natural(lse[t]);
        Elem<T> *const to = d + (T == UMAP_F16 && places.slot ? places.slot[t] : t) * pitch + m0;
        float v[FM][4];
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) v[i][r] = number * logit.exp_less(acc[i][j][r], less);
        if (tokens.any(j)) {
            const float taken = value[t] * shrink, entry = fmaf(number, logit.exp_less(OwnPlaces<P>::pick(place, acc, j), less), -taken);
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) v[i][r] = place == 16 * i + r ? entry : v[i][r];
            if (rest && OwnPlaces<P>::here(place)) rest[t] = (entry - elem_float<T>(float_elem<T>(entry))) * (1.0f / shrink);
        }
        if (live < P::M || number == 0.0f) {   // past the table, or a row without part
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) v[i][r] = number != 0.0f && P::m_of(i) + r < live ? v[i][r] : 0.0f;
        }
        auto store = [&](Elem<T> *at, auto round) {
            if constexpr (sizeof(Elem<T>) == 2 && FM % 2 == 0) {
#pragma unroll
                for (int i = 0; i < FM; i += 2) {
                    const Raw<T, 4> a = round(v[i]), b = round(v[i + 1]);
                    store_raw<T, 8>(at + P::m_first(i) + pair_row(), pair_of<T>(a, b));
                }
            } else {
#pragma unroll
                for (int i = 0; i < FM; ++i) store_raw<T, 4>(at + P::m_of(i), round(v[i]));
            }
        };
        if (!below) {
            store(to, [](float(&x)[4]) { return raw_of<T, 4>(x); });
        } else {
            store(to, [](float(&x)[4]) { return rounded<T, 4>(x); });
            store(to + below, [](float(&x)[4]) { return raw_of<T, 4>(x); });
        }
    }
}

// The entries of D at the rows' own tokens (fp32: value is taken from what is there).
template <int T>
__global__ __launch_bounds__(256) void k_head_own(const int *token, const float *value, int64_t count, int k, int64_t first,
                                                  int64_t rows, RowPlaces places, Elem<T> *d, int64_t pitch, int64_t below)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
        const int64_t v = token[i] - first;
        if (token[i] < 0 || v < 0 || v >= rows) continue;
        const int64_t t = i / k;
        Elem<T> *const at = d + (T == UMAP_F16 && places.slot ? places.slot[t] : t) * pitch + v;
        if constexpr (T == UMAP_F32) {   // each place has one token's value
            *at -= value[i];
            continue;
        }
        const float entry = T == UMAP_F16 && places.slot ? value[i] * places.shrink[t] : value[i];
        *at = float_elem<T>(entry);
        if (below) at[below] = float_elem<T>(entry - elem_float<T>(*at));
    }
}

// dh's sums over a part of the piece, [split][t][c], added to those of the pieces before.
struct RowSums {
    ProductSide w, d;
    Tiles tiles;
    int64_t depth;
    bool add;
    float *sums;
    int64_t pitch;
};
template <int T, class P>
__device__ __forceinline__ void rows_tile(const RowSums &x, int block, Piece *lds)
{
    constexpr int FM = P::kFM, FN = P::kFN;
    const auto &[w, d, tiles, depth, add, sums, pitch] = x;
    const int split = block / (tiles.m * tiles.n);
    const TileAt tile = tile_at(tiles, block % (tiles.m * tiles.n));
    const int64_t m0 = (int64_t)tile.m * P::M, n0 = (int64_t)tile.n * P::N, k0 = split * depth;
    Acc4 acc[FM][FN];
    P::run(w, d, m0, n0, k0, min(k0 + depth, w.rows), lds, acc);
    float *const to = sums + split * d.rows * pitch;
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const int64_t t = n0 + P::n_of(j);
        if (t >= d.rows) continue;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int64_t c = m0 + P::m_of(i);
            if (c >= pitch) continue;
            Acc4 *const at = reinterpret_cast<Acc4 *>(to + t * pitch + c);
            *at = add ? *at + acc[i][j] : acc[i][j];
        }
    }
}

// dh from the sums' parts: four columns per thread, or per 16 threads where there are many parts, each of which adds
// every 16th.
template <int T, int SLICES>
__global__ __launch_bounds__(256) void k_head_dh_join(const float *sums, int parts, int64_t pitch, RowWeights weights, RowPlaces places,
                                                      RowRests rests, ProductSide w, umap_rows dh)
{
    constexpr int kGroups = 256 / SLICES;
    __shared__ Acc4 part[SLICES > 1 ? SLICES : 1][kGroups];
    const int64_t groups = pitch / 4, total = dh.rows * groups;
    const int slice = threadIdx.x / kGroups, in = threadIdx.x % kGroups;
    for (int64_t i0 = (int64_t)blockIdx.x * kGroups; i0 < total; i0 += (int64_t)gridDim.x * kGroups) {
        const int64_t i = i0 + in, t = i / groups, c = i % groups * 4;
        Acc4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
        if (i < total) {
            const int64_t at = T == UMAP_F16 && places.slot ? places.slot[t] : t;
#pragma unroll 4
            for (int s = slice; s < parts; s += SLICES) sum += *reinterpret_cast<const Acc4 *>(sums + (s * dh.rows + at) * pitch + c);
        }
        if constexpr (SLICES > 1) {
            __syncthreads();
            part[slice][in] = sum;
            __syncthreads();
            if (slice) continue;
#pragma unroll
            for (int s = 1; s < SLICES; ++s) sum += part[s][in];
        }
        if (i >= total) continue;
        if (T == UMAP_F16 && places.slot) sum *= 1.0f / places.shrink[t];
        const int e = weights.exponent[t], own = rests.token ? rests.token[t] : -1;
        if (own >= 0) {
            const Elem<T> *const row = static_cast<const Elem<T> *>(w.data) + own * w.stride;
            const float rest = rests.rest[t];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j < dh.cols) sum[j] = fmaf(rest, elem_float<T>(row[c + j]), sum[j]);
        }
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = e == kNoRow ? 0.0f : ldexpf(sum[j] * weights.all, e - kShift<T> + weights.power);
        Elem<T> *const to = static_cast<Elem<T> *>(dh.data) + t * dh.stride + c;
        if (c + 4 <= dh.cols) {
            store_raw<T, 4>(to, raw_of<T, 4>(v));
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j < dh.cols) to[j] = float_elem<T>(v[j]);
        }
    }
}

// The table's gradient for a piece's rows.
struct TableRows {
    ProductSide h, d;
    Tiles tiles;
    RowWeights weights;
    RowPlaces places;
    int parts;   // of D, one after the other
    bool add;
    umap_rows dw;
};
template <int T, class P>
__device__ __forceinline__ void table_tile(const TableRows &x, int block, Piece *lds)
{
    constexpr int FM = P::kFM, FN = P::kFN;
    const ProductSide &h = x.h, &d = x.d;
    const RowWeights &weights = x.weights;
    const umap_rows &dw = x.dw;
    const bool add = x.add;
    const TileAt at = tile_at(x.tiles, block);
    const int64_t m0 = (int64_t)at.m * P::M, n0 = (int64_t)at.n * P::N;
    Acc4 acc[FM][FN];
    if constexpr (T != UMAP_F16) {
        P::run(h, d, m0, n0, 0, h.rows, lds, acc);
    } else {   // the bands, from the smallest weights on
        const int *const start = x.places.start;
        const int64_t each = start ? h.rows / x.parts : h.rows;
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = Acc4{0.0f, 0.0f, 0.0f, 0.0f};
        const int top = start ? __builtin_amdgcn_readfirstlane(start[kBands + 1]) : 0;
        for (int b = top; b >= 0; --b) {
            const int64_t k0 = start ? __builtin_amdgcn_readfirstlane(start[b]) : 0, k1 = start ? __builtin_amdgcn_readfirstlane(start[b + 1]) : each;
            if (b < top) {
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j) acc[i][j] *= 1.0f / (1 << kBandBits);
            }
            for (int64_t of = 0; k0 < k1 && of < h.rows; of += each) {   // a part of D
                const ProductSide some{h.data, h.stride, of + k1, h.cols}, entries{d.data, d.stride, of + k1, d.cols};
                P::template run<true>(some, entries, m0, n0, of + k0, of + k1, lds, acc);
            }
        }
    }
    const int e = h.rows > 0 ? largest_of(weights) - kShift<T> + weights.power : 0;
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const int64_t v = n0 + P::n_of(j);
        if (v >= dw.rows) continue;
        Elem<T> *const to = static_cast<Elem<T> *>(dw.data) + v * dw.stride + m0;
        auto four = [&](int i, int64_t c, float (&g)[4]) {   // columns c .. c + 3 of acc[i][j]
#pragma unroll
            for (int r = 0; r < 4; ++r) g[r] = ldexpf(acc[i][j][r] * weights.all, e);
            if (!add) return;
            float old[4] = {};
            if (c + 4 <= dw.cols) {
                floats_of<T, 4>(load_raw<T, 4>(to + (c - m0)), old);
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (c + r < dw.cols) old[r] = elem_float<T>(to[c - m0 + r]);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) g[r] += old[r];
        };
        if constexpr (sizeof(Elem<T>) == 2 && FM % 2 == 0) {
#pragma unroll
            for (int i = 0; i < FM; i += 2) {
                float a[4], b[4];
                const int64_t c = m0 + P::m_first(i) + pair_row();
                four(i, m0 + P::m_of(i), a);
                four(i + 1, m0 + P::m_of(i + 1), b);
                const Raw<T, 8> r = pair_of<T>(raw_of<T, 4>(a), raw_of<T, 4>(b));
                if (c + 8 <= dw.cols) {
                    store_raw<T, 8>(to + (c - m0), r);
                } else {
                    float g[8];
                    floats_of<T, 8>(r, g);
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        if (c + q < dw.cols) to[c - m0 + q] = float_elem<T>(g[q]);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                float g[4];
                const int64_t c = m0 + P::m_of(i);
                four(i, c, g);
                if (c + 4 <= dw.cols) {
                    store_raw<T, 4>(to + (c - m0), raw_of<T, 4>(g));
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (c + r < dw.cols) to[c - m0 + r] = float_elem<T>(g[r]);
                }
            }
        }
    }
}

template <int T, class P>
__global__ __launch_bounds__(P::kThreads) void k_head_dh(RowSums x)
{
    __shared__ __align__(16) Piece lds[P::kLds / 16];
    rows_tile<T, P>(x, blockIdx.x, lds);
}
template <int T, class P>
__global__ __launch_bounds__(P::kThreads) void k_head_dw(TableRows x)
{
    __shared__ __align__(16) Piece lds[P::kLds / 16];
    table_tile<T, P>(x, blockIdx.x, lds);
}
// Both in one launch, for products too small to fill the card: `rows` workgroups of the first.
template <int T, class P, class Q>
__global__ __launch_bounds__(P::kThreads) void k_head_dh_dw(RowSums x, int rows, TableRows y)
{
    static_assert(P::kThreads == Q::kThreads, "");
    __shared__ __align__(16) Piece lds[std::max(P::kLds, Q::kLds) / 16];
    if ((int)blockIdx.x < rows) rows_tile<T, P>(x, blockIdx.x, lds);
    else table_tile<T, Q>(y, blockIdx.x - rows, lds);
}

// ---- sizes -----------------------------------------------------------------------------------

constexpr int64_t up(int64_t a, int64_t b) { return over(a, b) * b; }

int elem_size(int32_t type) { return type == UMAP_F32 ? 4 : 2; }

// The products' tiles (TileShape), and for few rows of h tiles of 64 x 32 and 64 x 64, for dh of 128 columns.
template <int T, bool AA, bool AB>
using Large = Product<T, AA, AB, 2, 4, 8, 4, 2>;
template <int T, bool AA, bool AB>
using Small = Product<T, AA, AB, 2, 2, 4, 4, 2>;
template <int T, bool AA, bool AB, int DEPTH>
using Tiny = Product<T, AA, AB, 2, 2, 2, 2, DEPTH>;
template <int T, bool AA, int FN>
using Few = Product<T, AA, false, 4, 1, AA ? 2 : 1, FN, 4>;
constexpr int64_t kFewRows = 64;

// A table whose rows are not whole pieces at 16-byte places is copied first, a piece of 128 MB at most at a time.  (Taken by
// way of registers instead, with unaligned loads, 1,023 rows of fp16 against 32,003 x 1,001 took 118 us, of which the copy
// saved 16; 17 rows of bf16 against 15,824 x 3,999 took 60 us, with the copy 75, but their gradient 250, with it 200.)
constexpr int64_t kPackBytes = (int64_t)128 << 20;
int64_t pack_rows(int64_t pitch, int64_t elem) { return std::max<int64_t>(256, kPackBytes / (pitch * elem) / 256 * 256); }

// Forward: rows of h at a time, so that the partial sums stay within 128 MB (a quarter of that with the large tiles), but 256 rows
// at least, since each turn reads the whole table: from 4.2 million tokens on they take 32 bytes a token.
struct LossSizes {
    int64_t tiles, rows, pitch, piece;
    int64_t partial, own, copy, table, total;   // offsets into the workspace
    LossSizes(int64_t n, int64_t vocab, int32_t cols, int32_t type)
    {
        const int64_t elem = elem_size(type);
        tiles = over(vocab, 64);   // as many as the smallest have
        rows = std::max<int64_t>(256, ((int64_t)128 << 20) / (tiles * (int64_t)sizeof(MaxSum)) / 256 * 256);
        rows = std::min(rows, n);
        pitch = up(cols, 64);
        piece = std::min(pack_rows(pitch, elem), up(vocab, 256));
        partial = 0;
        own = up(rows * tiles * (int64_t)sizeof(MaxSum), 256);
        copy = own + up(rows * 4, 256);
        table = copy + up(rows * pitch * elem, 256);
        total = table + piece * pitch * elem;
    }
};

// Rows up to which a 16-bit D has two parts: few rows do not average the rounding out.  It is paid for in time: one part or two
// against 32,000 x 2,048 in bf16 take 81 and 81 us for 1 row, 84 and 86 for 16, 98 and 118 for 64, 128 and 170 for 128, 190
// and 235 for 256.  dtable's error, relative to its type's own, at worst of 60 cases each: one part 1.64 for 20 to 128 rows and
// 1.49 for 129 to 256, two parts 1.0006; one part for 257 to 700 rows 1.44.
constexpr int64_t kTwoPartRows = 256;

struct GradSizes {
    int64_t n, vocab, cols, k, elem;
    int64_t parts;     // of D
    TileShape dh_shape;
    bool dh_few;
    int64_t piece, d_pitch, h_pitch, sum_pitch, splits, depth;
    // offsets into the workspace
    int64_t largest, start, number, exponent, slot, shrink, token, value, rest_token, rest, copy, scaled, d, sums, packed, total;
    GradSizes(int64_t n_, int64_t vocab_, int32_t cols_, int64_t k_, int32_t type, bool pack)
        : n(n_), vocab(vocab_), cols(cols_), k(k_), elem(elem_size(type))
    {
        parts = elem == 2 && n <= kTwoPartRows ? 2 : 1;
        const int64_t budget = (int64_t)256 << 20;   // of D, but 256 tokens at least: 512 bytes a row of 16 bits
        int64_t most = std::max<int64_t>(256, budget / std::max<int64_t>(1, n * parts * elem) / 256 * 256);
        most = std::min(most, (int64_t)1 << 22);   // so that the launches' sizes fit
        h_pitch = up(cols, 64);
        if (pack) most = std::min(most, pack_rows(h_pitch, elem));
        const int64_t pieces = over(vocab, most);
        piece = up(over(vocab, pieces), 256);
        d_pitch = piece;
        sum_pitch = up(cols, 4);
        // the product for dh: parts of the piece at a time where its tiles alone do not fill the card
        const int64_t step = 128 / elem, steps = over(piece, step), most_splits = std::max<int64_t>(1, steps / (elem == 4 ? 2 : 4));
        dh_few = n * parts <= kFewRows && vocab * cols * elem >= ((int64_t)8 << 20);   // less, and one launch does both products
        dh_shape = tile_shape(cols, n * parts, most_splits, elem);
        const int64_t side = tile_side(dh_shape);
        if (dh_few) splits = parts_for(over(cols, 128), 512, most_splits);
        else splits = parts_for(over(cols, side) * over(std::max<int64_t>(n * parts, 1), side), side == 256 ? 256 : side == 128 ? 512 : 1024, most_splits);
        depth = over(steps, splits) * step;
        splits = over(piece, depth);
        int64_t at = 0;
        auto take = [&](int64_t bytes) {
            const int64_t was = at;
            at += up(bytes, 256);
            return was;
        };
        largest = take(sizeof(Exponents));
        start = take((kBands + 2) * 4);
        number = take(n * 4);
        exponent = take(n * 4);
        slot = take(n * 4);
        shrink = take(n * 4);
        token = take(n * k * 4);
        value = take(n * k * 4);
        rest_token = take(n * 4);
        rest = take(n * 4);
        copy = take(n * parts * h_pitch * elem);
        scaled = take(n * parts * h_pitch * elem);
        d = take(n * parts * d_pitch * elem);
        sums = take(splits * n * parts * sum_pitch * 4);
        packed = take(pack ? piece * h_pitch * elem : 0);
        total = at;
    }
};

// Calls f with a product's tiles.
template <int T, bool AA, bool AB, typename F>
hipError_t by_shape(TileShape shape, F f)
{
    switch (shape) {
    case TileShape::large:
        if constexpr (!Small<T, AA, AB>::kBlocks) return f(Large<T, AA, AB>{});
        [[fallthrough]];   // logits_shape() does not ask for it
    case TileShape::small: return f(Small<T, AA, AB>{});
    case TileShape::tiny: return f(Tiny<T, AA, AB, 2>{});
    default: return f(Tiny<T, AA, AB, 4>{});
    }
}
template <int T, bool AA, typename F>
hipError_t by_few(int64_t n, F f)
{
    return n <= 32 ? f(Few<T, AA, 2>{}) : f(Few<T, AA, 4>{});
}
// `rows` of a table against n rows of h.
template <int T, typename F>
hipError_t by_logits(int64_t rows, int64_t n, F f)
{
    return n <= kFewRows ? by_few<T, false>(n, f) : by_shape<T, false, false>(logits_shape(rows, n, sizeof(Elem<T>)), f);
}

// Calls f with the waves of a row: one; four where rows are few or have many tokens, and 16 where both holds.
template <typename F>
hipError_t by_team(int64_t rows, int64_t k, F f)
{
    if (rows <= 256 && k >= 8) return f(std::integral_constant<int, 16>{});
    if (rows < 2048 || k >= 8) return f(std::integral_constant<int, 4>{});
    return f(std::integral_constant<int, 1>{});
}

template <class P>
Tiles tiles_of(int64_t m, int64_t n)
{
    return {(int)over(m, P::M), (int)over(n, P::N)};
}

template <int T>
ProductSide side_of(const umap_rows &m, int64_t first, int64_t rows)
{
    return {static_cast<const Elem<T> *>(m.data) + first * m.stride, m.stride, rows, m.cols};
}

#define UL_LAUNCHED(expr)                      \
    do {                                       \
        const hipError_t ul_e_ = (expr);       \
        if (ul_e_ != hipSuccess) return ul_e_; \
    } while (0)

template <int T>
hipError_t pack(const ProductSide &from, Elem<T> *to, int64_t pitch, hipStream_t s)
{
    hipLaunchKernelGGL((k_head_pack<T>), dim3((unsigned)std::min<int64_t>(8192, over(from.rows * pitch / 8, 256))), dim3(256), 0, s, from,
                       to, (int)pitch);
    return hipGetLastError();
}

template <int T>
hipError_t loss(const umap_rows &h, const umap_rows &table, const Taught &taught, float scale, float *out, float *lse,
                void *workspace, hipStream_t s)
{
    const LossSizes z(h.rows, table.rows, h.cols, h.type);
    char *const base = static_cast<char *>(workspace);
    auto *const partial = reinterpret_cast<MaxSum *>(base + z.partial);
    float *const own = taught.k == 1 ? reinterpret_cast<float *>(base + z.own) : nullptr;
    const ProductSide all = side_of<T>(table, 0, table.rows);
    const bool packing = !direct_side<T>(all);
    const int64_t piece = packing ? z.piece : table.rows;
    for (int64_t first = 0; first < h.rows; first += z.rows) {
        const ProductSide given = side_of<T>(h, first, std::min(z.rows, h.rows - first));
        ProductSide rows = given;
        if (!direct_side<T>(given)) {
            UL_LAUNCHED(pack<T>(given, reinterpret_cast<Elem<T> *>(base + z.copy), z.pitch, s));
            rows = {base + z.copy, z.pitch, given.rows, z.pitch};
        }
        int64_t tiles = 0;   // of all pieces, whose tiles are of one size: that of the whole table
        (void)by_logits<T>(table.rows, rows.rows, [&](auto shape) {
            tiles = over(table.rows, decltype(shape)::M);
            return hipSuccess;
        });
        for (int64_t v = 0; v < table.rows; v += piece) {
            ProductSide w = side_of<T>(table, v, std::min(piece, table.rows - v));
            if (packing) {
                UL_LAUNCHED(pack<T>(w, reinterpret_cast<Elem<T> *>(base + z.table), z.pitch, s));
                w = {base + z.table, z.pitch, w.rows, z.pitch};
            }
            UL_LAUNCHED(by_logits<T>(table.rows, rows.rows, [&](auto shape) {
                using P = decltype(shape);
                const Tiles g = tiles_of<P>(w.rows, rows.rows);
                hipLaunchKernelGGL((k_head_lse<T, P>), dim3((unsigned)((int64_t)g.m * g.n)), dim3(P::kThreads), 0, s, w, rows, scale, g,
                                   v / P::M, tiles, partial, OwnLogits{taught.ids, first, table.rows, v, own});
                return hipGetLastError();
            }));
        }
        UL_LAUNCHED(by_team(rows.rows, taught.k, [&](auto waves) {
            constexpr int W = decltype(waves)::value;
            hipLaunchKernelGGL((k_head_loss<T, W>), dim3((unsigned)over(rows.rows, RowTeam<W>::kRows)), dim3(RowTeam<W>::kBlock), 0, s, all, given, scale,
                               taught, first, tiles, partial, own, out, lse);
            return hipGetLastError();
        }));
    }
    return hipSuccess;
}

template <int T>
hipError_t grad(const umap_rows &h, const umap_rows &table, const Taught &taught, float scale, const float *lse,
                const float *dloss, float dscale, const umap_rows *dh, const umap_rows *dtable, bool add, void *workspace,
                hipStream_t s)
{
    const ProductSide all = side_of<T>(table, 0, table.rows);
    const bool packing = !direct_side<T>(all);
    const GradSizes z(h.rows, table.rows, table.cols, taught.k, h.type, packing);
    char *const base = static_cast<char *>(workspace);
    auto *const token = reinterpret_cast<int *>(base + z.token);
    auto *const value = reinterpret_cast<float *>(base + z.value), *const sums = reinterpret_cast<float *>(base + z.sums);
    auto *const copy = reinterpret_cast<Elem<T> *>(base + z.copy), *const d = reinterpret_cast<Elem<T> *>(base + z.d);
    auto *const scaled = dloss ? reinterpret_cast<Elem<T> *>(base + z.scaled) : nullptr;
    // a product that fp32 may not hold; of two fp32 numbers, so a double does
    Factor factor;
    factor.x = (float)frexp((double)dscale * scale, &factor.power);
    auto *const found = reinterpret_cast<Exponents *>(base + z.largest);
    const RowWeights weights{reinterpret_cast<float *>(base + z.number), reinterpret_cast<int *>(base + z.exponent), dloss ? &found->most : nullptr, dloss ? 1.0f : factor.x,
                             dloss ? 0 : factor.power};
    const bool fixing = dh && z.parts == 1 && sizeof(Elem<T>) == 2;
    const RowRests rests{fixing ? reinterpret_cast<int *>(base + z.rest_token) : nullptr, reinterpret_cast<float *>(base + z.rest)};
    RowPlaces places{};
    if (z.n > 0) {
        UL_LAUNCHED(by_team(z.n, z.k, [&](auto waves) {
            constexpr int W = decltype(waves)::value;
            hipLaunchKernelGGL((k_head_rows<T, W>), dim3((unsigned)over(z.n, RowTeam<W>::kRows)), dim3(RowTeam<W>::kBlock), 0, s,
                               all, side_of<T>(h, 0, h.rows), scale, taught, lse, dloss, factor, weights,
                               token, value, rests, copy, (int)z.h_pitch, (int)z.parts);
            return hipGetLastError();
        }));
        if (dloss && dtable) {
            auto *const slot = reinterpret_cast<int *>(base + z.slot), *const start = reinterpret_cast<int *>(base + z.start);
            auto *const shrink = reinterpret_cast<float *>(base + z.shrink);
            if (z.n > kFindRows) {
                if constexpr (T == UMAP_F16)
                    hipLaunchKernelGGL(k_head_order, dim3(1), dim3(1024), 0, s, weights.exponent, z.n, found, slot, shrink, start);
                else
                    hipLaunchKernelGGL(k_head_largest, dim3(1), dim3(1024), 0, s, weights.exponent, z.n, found);
                UL_LAUNCHED(hipGetLastError());
            }
            const dim3 blocks((unsigned)std::min<int64_t>(8192, over(z.n * z.h_pitch / 8, 256)));
            if constexpr (T == UMAP_F16) {
                places = {slot, shrink, start};
                hipLaunchKernelGGL(k_head_place, blocks, dim3(256), 0, s, copy, z.n, (int)z.parts, (int)z.h_pitch, weights.exponent, found,
                                   scaled, slot, shrink, start);
            } else {
                hipLaunchKernelGGL((k_head_scale<T>), blocks, dim3(256), 0, s, copy, z.n, (int)z.parts, (int)z.h_pitch, weights.exponent,
                                   found, scaled);
            }
            UL_LAUNCHED(hipGetLastError());
        }
    }
    // the copies' and D's columns past the last are zeros, and so are pieces of them
    const int64_t d_rows = z.n * z.parts, below = z.parts > 1 ? z.n * z.d_pitch : 0;
    const ProductSide rows{copy, z.h_pitch, z.n, z.h_pitch}, weighted{scaled ? scaled : copy, z.h_pitch, d_rows, z.h_pitch};
    for (int64_t first = 0; first < z.vocab; first += z.piece) {
        const int64_t here = std::min(z.piece, z.vocab - first);
        ProductSide w = side_of<T>(table, first, here);
        if (packing) {
            UL_LAUNCHED(pack<T>(w, reinterpret_cast<Elem<T> *>(base + z.packed), z.h_pitch, s));
            w = {base + z.packed, z.h_pitch, here, z.h_pitch};
        }
        const ProductSide d_side{d, z.d_pitch, d_rows, z.d_pitch};
        if (z.n > 0) {
            const bool one = z.k == 1;
            UL_LAUNCHED((by_logits<T>(here, z.n, [&](auto shape) {
                using P = decltype(shape);
                const Tiles g = tiles_of<P>(z.d_pitch, z.n);
                hipLaunchKernelGGL((k_head_d<T, P>), dim3((unsigned)((int64_t)g.m * g.n)), dim3(P::kThreads), 0, s, w, rows, scale, g,
                                   lse, weights, places, one ? token : nullptr, one ? value : nullptr, one && fixing ? rests.rest : nullptr, first, d, z.d_pitch, below);
                return hipGetLastError();
            })));
            if (!one) {
                hipLaunchKernelGGL((k_head_own<T>), dim3((unsigned)std::min<int64_t>(1024, over(z.n * z.k, 256))), dim3(256), 0, s,
                                   token, value, z.n * z.k, (int)z.k, first, here, places, d, z.d_pitch, below);
                UL_LAUNCHED(hipGetLastError());
            }
        }
        umap_rows part = {};
        TileShape dw_shape = TileShape::tiny_deep;
        if (dtable) {
            part = *dtable;
            part.data = static_cast<Elem<T> *>(dtable->data) + first * dtable->stride;
            part.rows = here;
            dw_shape = tile_shape(z.cols, here, 1, z.elem);
        }
        const bool sums_due = dh && z.n > 0;
        auto row_sums = [&](Tiles g) { return RowSums{w, d_side, g, z.depth, first > 0, sums, z.sum_pitch}; };
        auto table_rows = [&](Tiles g) { return TableRows{weighted, d_side, g, weights, places, (int)z.parts, add, part}; };
        if (sums_due && dtable && !z.dh_few && z.dh_shape == TileShape::tiny_deep && dw_shape == TileShape::tiny_deep) {
            using P = Tiny<T, true, false, 4>;
            using Q = Tiny<T, true, true, 4>;
            const Tiles g = tiles_of<P>(z.cols, d_rows), o = tiles_of<Q>(z.cols, here);
            const int64_t rows_count = (int64_t)g.m * g.n * z.splits;
            hipLaunchKernelGGL((k_head_dh_dw<T, P, Q>), dim3((unsigned)(rows_count + (int64_t)o.m * o.n)), dim3(P::kThreads), 0, s,
                               row_sums(g), (int)rows_count, table_rows(o));
            UL_LAUNCHED(hipGetLastError());
            continue;
        }
        if (sums_due) {
            auto launch = [&](auto shape) {
                using P = decltype(shape);
                const Tiles g = tiles_of<P>(z.cols, d_rows);
                hipLaunchKernelGGL((k_head_dh<T, P>), dim3((unsigned)((int64_t)g.m * g.n * z.splits)), dim3(P::kThreads), 0, s,
                                   row_sums(g));
                return hipGetLastError();
            };
            UL_LAUNCHED(z.dh_few ? (by_few<T, true>(d_rows, launch)) : (by_shape<T, true, false>(z.dh_shape, launch)));
        }
        if (dtable) {
            UL_LAUNCHED((by_shape<T, true, true>(dw_shape, [&](auto shape) {
                using P = decltype(shape);
                const Tiles g = tiles_of<P>(z.cols, here);
                hipLaunchKernelGGL((k_head_dw<T, P>), dim3((unsigned)((int64_t)g.m * g.n)), dim3(P::kThreads), 0, s, table_rows(g));
                return hipGetLastError();
            })));
        }
    }
    if (dh && z.n > 0) {
        const int64_t total = z.n * z.sum_pitch / 4;
        const int parts = (int)(z.splits * z.parts);
        if (parts >= 8)
            hipLaunchKernelGGL((k_head_dh_join<T, 16>), dim3((unsigned)std::min<int64_t>(4096, over(total, 16))), dim3(256), 0, s, sums,
                               parts, z.sum_pitch, weights, places, rests, all, *dh);
        else
            hipLaunchKernelGGL((k_head_dh_join<T, 1>), dim3((unsigned)std::min<int64_t>(4096, over(total, 256))), dim3(256), 0, s, sums,
                               parts, z.sum_pitch, weights, places, rests, all, *dh);
        UL_LAUNCHED(hipGetLastError());
    }
    return hipSuccess;
}

Taught taught_of(RowIds ids, const umap_rows *teacher, float teacher_scale)
{
    if (!teacher) return {ids, 1, nullptr, 0, 0, 1.0f};
    return {ids, teacher->cols, teacher->data, teacher->stride, teacher->type, teacher_scale};
}

}  // namespace

int64_t rows_head_bytes(int64_t n, int64_t vocab, int32_t cols, int32_t type) { return LossSizes(n, vocab, cols, type).total; }

hipError_t launch_rows_head(const umap_rows &h, const umap_rows &table, RowIds ids, const umap_rows *teacher, float scale,
                            float teacher_scale, float *loss_out, float *lse, void *workspace, hipStream_t s)
{
    const Taught taught = taught_of(ids, teacher, teacher_scale);
    switch (h.type) {
    case UMAP_F32: return loss<UMAP_F32>(h, table, taught, scale, loss_out, lse, workspace, s);
    case UMAP_F16: return loss<UMAP_F16>(h, table, taught, scale, loss_out, lse, workspace, s);
    default: return loss<UMAP_BF16>(h, table, taught, scale, loss_out, lse, workspace, s);
    }
}

int64_t rows_head_grad_bytes(int64_t n, int64_t vocab, int32_t cols, int32_t k, int32_t type)
{
    const int64_t plain = GradSizes(n, vocab, cols, k, type, false).total;   // how the table lies is not known here
    return std::max(plain, GradSizes(n, vocab, cols, k, type, true).total);
}

hipError_t launch_rows_head_grad(const umap_rows &h, const umap_rows &table, RowIds ids, const umap_rows *teacher, float scale,
                                 float teacher_scale, const float *lse, const float *dloss, float dscale, const umap_rows *dh,
                                 const umap_rows *dtable, bool accumulate, void *workspace, hipStream_t s)
{
    const Taught taught = taught_of(ids, teacher, teacher_scale);
    switch (h.type) {
    case UMAP_F32: return grad<UMAP_F32>(h, table, taught, scale, lse, dloss, dscale, dh, dtable, accumulate, workspace, s);
    case UMAP_F16: return grad<UMAP_F16>(h, table, taught, scale, lse, dloss, dscale, dh, dtable, accumulate, workspace, s);
    default: return grad<UMAP_BF16>(h, table, taught, scale, lse, dloss, dscale, dh, dtable, accumulate, workspace, s);
    }
}

}  // namespace ul
