// rows_product.hpp -- matrix products on the matrix cores, in tiles, for the kernels of the
// token rows' head: acc(m, n) = sum_k A(m, k) B(n, k), fp32 sums of 16-bit or fp32 elements.
//
// A side lies in memory either along k (element (i, k) at [i][k]: rows of the table against
// rows of h) or across it (at [k][i]).  A step takes 128 bytes of k of every row of the tile:
// 64 16-bit elements, or 32 fp32.  Both sides' steps lie in LDS in 16-byte pieces, the place
// of a piece in its row turned by the row's number so that the lanes that read together meet
// different banks; a side across k is turned on the way out (ds_read_b64_tr_b16).
//
// A fragment is a lane's 16 bytes: row lane % 16 of 16, and of the step's elements of k those
// from (lane / 16) * 16 bytes on.  How the matrix instruction numbers k does not matter as long as
// both sides agree.
//
// The large tile, 256 x 256 by eight waves of 128 x 64, takes 128 KB of LDS, two steps.  The matrix cores are busy 61 to 65 %
// of the cycles in the gradient's three products at 2.0 GHz, 73 % in the loss's single long launch, whose clock their power
// holds at 1.5 while counted: 1,400 TFLOP/s of bf16 with random values, 1,750 with a table of zeros (the library's product 1,490
// and 2,000).  Four waves of 128 x 128 (one to a SIMD, 512 registers) took 9.0 ms where these
// took 7.1; loads not spread between the products cost 2 to 3 %.  No read meets another's bank (counted).
#pragma once

#include "rows_device.hpp"

namespace ul {

typedef float Acc4 __attribute__((ext_vector_type(4)));

struct ProductSide {
    const void *data;
    int64_t stride;   // elements
    int64_t rows;     // of the memory; what lies outside counts as zeros
    int64_t cols;
};

struct __attribute__((aligned(16))) Piece {
    uint32_t w[4];
};

template <int T>
__device__ __forceinline__ Acc4 multiply(const Piece &a, const Piece &b, Acc4 c)
{
    typedef __bf16 B8 __attribute__((ext_vector_type(8)));
    typedef _Float16 H8 __attribute__((ext_vector_type(8)));
    if constexpr (T == UMAP_BF16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(B8, a), __builtin_bit_cast(B8, b), c, 0, 0, 0);
    } else if constexpr (T == UMAP_F16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(H8, a), __builtin_bit_cast(H8, b), c, 0, 0, 0);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w[j]), __uint_as_float(b.w[j]), c, 0, 0, 0);
        return c;
    }
}

// One side's step of a tile of I rows.
template <int T, bool kAcross, int I>
struct Step {
    static constexpr int kElem = sizeof(Elem<T>), kPer = 16 / kElem, kDepth = 128 / kElem;
    static constexpr int kRow = kAcross ? I / kPer : 8;   // pieces of a row in LDS
    static constexpr int kPieces = I * 8;
    static constexpr int kReads = !kAcross ? 1 : kElem == 2 ? 2 : 4;   // LDS reads of a fragment
    // How the pieces of row r are turned: along k, the 8 lanes that read 16 bytes at once are of 8
    // rows; across, 32 lanes read 32 bytes of 8 rows (fp32: 64 bytes of 2 rows).
    __device__ static __forceinline__ int turn(int r)
    {
        if constexpr (!kAcross) return r & 7;
        else if constexpr (kElem == 2) return (((r & 3) | (r >> 1 & 4)) << 1) & (kRow - 1);
        else return r & 4;
    }
    // Row and column of LDS piece p, in memory, from the tile's origin.
    __device__ static __forceinline__ void place(int p, int &r, int &c)
    {
        r = p / kRow;
        c = ((p % kRow) ^ turn(r)) * kPer;
    }
    // Fragment of rows i .. i + 15, from the step's first or second half.
    __device__ static __forceinline__ Piece fragment(const Piece *lds, int i, int half, int lane)
    {
        const int j = lane & 15, g = lane >> 4;
        if constexpr (!kAcross) {
            const int r = i + j;
            return lds[r * 8 + ((half * 4 + g) ^ turn(r))];
        } else if constexpr (kElem == 2) {
            // 16 lanes fetch 4 rows of k, 16 elements each, and get a column each
            typedef short S4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) S4 *Lds;
            Piece p;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int r = half * 32 + g * 8 + q * 4 + (j >> 2), c = i / kPer + (j >> 1 & 1);
                const auto *at = reinterpret_cast<const uint64_t *>(lds + r * kRow + (c ^ turn(r))) + (j & 1);
                const S4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(at));
                __builtin_memcpy(&p.w[2 * q], &v, 8);
            }
            return p;
        } else {
            Piece p;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int r = half * 16 + g * 4 + q, c = i + j;
                p.w[q] = lds[r * kRow + ((c >> 2) ^ turn(r))].w[c & 3];
            }
            return p;
        }
    }
};

// Whether a side is made of whole pieces at 16-byte places, its rows apart, but close enough for 32-bit offsets.
template <int T>
bool direct_side(const ProductSide &s)
{
    constexpr int kElem = sizeof(Elem<T>), kPer = 16 / kElem;
    return (uintptr_t)s.data % 16 == 0 && s.stride % kPer == 0 && s.cols % kPer == 0 && s.stride >= s.cols &&
           s.stride < ((int64_t)1 << 30) / 256 / kElem;
}

// All of this wave's loads into LDS but the newest `left` have landed, then all waves'.
template <int LEFT>
__device__ __forceinline__ void landed()
{
    __builtin_amdgcn_s_waitcnt(0xc07f);   // LDS reads alone; the compiler, which counts them, is to know
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

// How a side's steps get into LDS: straight, 64 lanes, 64 pieces next to each other; piece p of a step is thread
// p % THREADS's.  Lanes whose piece lies outside the matrix are given an offset beyond the buffer, which loads zeros.
template <int T, bool kAcross, int I, int THREADS>
struct DirectSide {
    using S = Step<T, kAcross, I>;
    typedef uint32_t Words __attribute__((ext_vector_type(4)));
    static constexpr int kElem = S::kElem, kCount = S::kPieces / THREADS, kRows = THREADS / S::kRow;
    const ProductSide &side;
    const int64_t i0;
    int row, col;
    uint32_t offset;
    static_assert(kRows % (kAcross && kElem == 2 ? 16 : 8) == 0, "a piece's row is turned alike kRows rows on");
    __device__ __forceinline__ DirectSide(const ProductSide &of, int64_t first) : side(of), i0(first)
    {
        S::place(threadIdx.x, row, col);
        offset = (uint32_t)((row * side.stride + col) * kElem);
        if (kAcross && i0 + col >= side.cols) offset = 0x80000000u;
    }
    struct Loads {   // of one step
        Words buffer;
        uint32_t at, lds, step;
    };
    __device__ __forceinline__ Loads loads(int64_t k, bool there, Piece *to) const
    {
        const int64_t r0 = kAcross ? k : i0, c0 = kAcross ? i0 : k;
        const char *const base = static_cast<const char *>(side.data) + (r0 * side.stride + c0) * kElem;
        const int64_t rows = min((int64_t)(kAcross ? S::kDepth : I), side.rows - r0);
        const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        return {Words{(uint32_t)(uintptr_t)base, (uint32_t)((uintptr_t)base >> 32) & 0xffffu,
                      there && rows > 0 ? (uint32_t)(rows * side.stride * kElem) : 0u, 0x00027000u},
                !kAcross && k + col >= side.cols ? 0x80000000u : offset,
                (uint32_t)(uintptr_t)(__attribute__((address_space(3))) Piece *)to + wave * 1024, (uint32_t)(kRows * side.stride * kElem)};
    }
    // The q-th of the step's loads.
    __device__ __forceinline__ void one(const Loads &x, int q) const
    {
        // the whole offset in the lane's register: it is what the hardware compares with the buffer's length.  The others are
        // alike in all lanes, which a build without optimization has to be told.
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"((uint32_t)__builtin_amdgcn_readfirstlane(x.lds + q * THREADS * 16)),
                     "v"(x.at + q * x.step), "s"(Words{(uint32_t)__builtin_amdgcn_readfirstlane(x.buffer.x), (uint32_t)__builtin_amdgcn_readfirstlane(x.buffer.y), (uint32_t)__builtin_amdgcn_readfirstlane(x.buffer.z), (uint32_t)__builtin_amdgcn_readfirstlane(x.buffer.w)})
                     : "m0", "memory");
    }
};

// Tiles of a grid of m x n of them, one per workgroup.  Workgroups go round the 8 XCDs in turn; each XCD takes a
// stretch of the tiles, which goes over 8 rows of tiles at a time, so that the 32 tiles it works on at once
// share their sides' panels in its L2.
struct Tiles {
    int m, n;
};
struct TileAt {
    int m, n;
};
__device__ __forceinline__ TileAt tile_at(const Tiles &tiles, int block)
{
    constexpr int kXcds = 8, kRows = 8;
    const int total = tiles.m * tiles.n, each = total / kXcds, more = total % kXcds, xcd = block % kXcds;
    const int id = xcd * each + min(xcd, more) + block / kXcds;
    const int band = id / (kRows * tiles.n), first = band * kRows, rows = min(kRows, tiles.m - first), in = id - first * tiles.n;
    return {first + in % rows, in / rows};
}

// A tile of WM x WN waves of FM x FN fragments each, of sides in whole pieces (direct_side); DEPTH steps in LDS, all but
// one of them on their way.
//
// A step is two halves.  The fragments of a half are fetched while the half before is multiplied, and a step's loads
// are issued, when its place has become free, between the products too: evenly, since eight waves that issue
// theirs at once wait for each other.
template <int T, bool kAcrossA, bool kAcrossB, int WM, int WN, int FM, int FN, int DEPTH>
struct Product {
    static constexpr int kWM = WM, kWN = WN, kFM = FM, kFN = FN;
    static constexpr int kThreads = 64 * WM * WN, M = 16 * WM * FM, N = 16 * WN * FN;
    using A = Step<T, kAcrossA, M>;
    using B = Step<T, kAcrossB, N>;
    using SideA = DirectSide<T, kAcrossA, M, kThreads>;
    using SideB = DirectSide<T, kAcrossB, N, kThreads>;
    static constexpr int kDepth = A::kDepth, kStage = A::kPieces + B::kPieces;
    static constexpr int kLds = kStage * 16 * DEPTH;
    // fp32 logits, which are not rounded any further, are summed in blocks of 256 columns, and so not by large tiles, whose
    // registers are short for it.  lse of 174 rows against 589 x 3,008 was off by 2.2e-5 with one long sum, by 2.4e-6 so, dh by
    // 1.4e-6 and 4.6e-7 of its norm; 4,096 rows against 32,000 x 1,024 take 2.03 ms instead of 1.93, the gradient 5.97 for 5.86.
    static constexpr bool kBlocks = T == UMAP_F32 && !kAcrossA && !kAcrossB;
    static constexpr int kBlockSteps = 8;

    // acc of rows m0 .. of A and n0 .. of B, over k0 <= k < k1: along k a multiple of kDepth to the sides' columns or another one,
    // across it any to the sides' rows or a multiple of kDepth further.  kMore: added to what acc holds.
    template <bool kMore = false>
    static __device__ __forceinline__ void run(const ProductSide &a, const ProductSide &b, int64_t m0, int64_t n0,
                                               int64_t k0, int64_t k1, Piece *lds, Acc4 acc[FM][FN])
    {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = kMore ? acc[i][j] : Acc4{0.0f, 0.0f, 0.0f, 0.0f};
        if (k0 >= k1) return;
        const SideA da(a, m0);
        const SideB db(b, n0);
        const int steps = (int)((k1 - k0 + kDepth - 1) / kDepth);
        constexpr int kA = SideA::kCount, kLoads = kA + SideB::kCount;
        Piece fa[FM], fb[2][FN];
        // A half step's products with fb[set], row by row, and between the rows the fetches of the next half's fragments
        // (step s, half `half`; a row's of A once its own are multiplied) and, if `loading`, the loads of step l.
        auto half_step = [&](auto products, int set, int s, int half, auto loading, int l) {
            constexpr bool kProducts = decltype(products)::value, kLoading = decltype(loading)::value;
            const Piece *const from = lds + s % DEPTH * kStage;
            Piece *const to = lds + l % DEPTH * kStage;
            const auto la = da.loads(k0 + (int64_t)l * kDepth, l < steps, to);
            const auto lb = db.loads(k0 + (int64_t)l * kDepth, l < steps, to + A::kPieces);
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                if constexpr (kLoading) {
#pragma unroll
                    for (int q = i * kLoads / FM; q < (i + 1) * kLoads / FM; ++q) {
                        if (q < kA) da.one(la, q);
                        else db.one(lb, q - kA);
                    }
                }
#pragma unroll
                for (int j = i * FN / FM; j < (i + 1) * FN / FM; ++j)
                    fb[set ^ 1][j] = B::fragment(from + A::kPieces, (wn * FN + j) * 16, half, lane);
                if constexpr (kProducts) {
#pragma unroll
                    for (int j = 0; j < FN; ++j) acc[i][j] = multiply<T>(fa[i], fb[set][j], acc[i][j]);
                    __builtin_amdgcn_sched_barrier(0);
                }
                fa[i] = A::fragment(from, (wm * FM + i) * 16, half, lane);
            }
        };
        [[maybe_unused]] Acc4 whole[FM][FN] = {};
        [[maybe_unused]] auto add_block = [&] {
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    whole[i][j] += acc[i][j];
                    acc[i][j] = Acc4{0.0f, 0.0f, 0.0f, 0.0f};
                }
        };
        constexpr auto yes = std::true_type{};
        constexpr auto no = std::false_type{};
        for (int s = 0; s < DEPTH; ++s) {
            Piece *const to = lds + s * kStage;
            const auto la = da.loads(k0 + (int64_t)s * kDepth, s < steps, to);
            const auto lb = db.loads(k0 + (int64_t)s * kDepth, s < steps, to + A::kPieces);
#pragma unroll
            for (int q = 0; q < kA; ++q) da.one(la, q);
#pragma unroll
            for (int q = 0; q < SideB::kCount; ++q) db.one(lb, q);
        }
        landed<(DEPTH - 1) * kLoads>();
        half_step(no, 1, 0, 0, no, 0);
        for (int s = 0; s < steps; ++s) {
            half_step(yes, 0, s, 1, no, 0);
            landed<(DEPTH - 2) * kLoads>();   // step s + 1 is there, and everybody has fetched all of step s
            half_step(yes, 1, s + 1, 0, yes, s + DEPTH);   // behind the last step: nobody takes them
            if constexpr (kBlocks) {
                if (s % kBlockSteps == kBlockSteps - 1) add_block();
            }
        }
        landed<0>();
        if constexpr (kBlocks) {
            add_block();
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = whole[i][j];
        }
    }

    // Where a lane's values lie: acc[i][j][r] is row m_of(i) + r of A, one of 16 from m_first(i) on, and row n_of(j) of B.
    static __device__ __forceinline__ int m_first(int i) { return ((int)(threadIdx.x >> 6) / WN * FM + i) * 16; }
    static __device__ __forceinline__ int m_of(int i) { return m_first(i) + (threadIdx.x >> 4 & 3) * 4; }
    static __device__ __forceinline__ int n_of(int j)
    {
        const int wave = threadIdx.x >> 6;
        return ((wave % WN) * FN + j) * 16 + (threadIdx.x & 15);
    }
};

}  // namespace ul
