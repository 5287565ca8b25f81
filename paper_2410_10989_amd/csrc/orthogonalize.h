// Orthogonalising matrices by Newton-Schulz products.  For a matrix G of min(rows, cols) = m and max(rows, cols) = n
// (transposed where it has more rows than columns)
//
//     X = G / (|G|_F + eps),      then per step    A = X X^T,   B = a I + b A + c A A,   X <- B X        out = s X
//
// drives every singular value of X towards 1 and keeps its singular vectors.  Per step 2 m^2 n + 2 m^3 + 2 m^2 n
// operations; A and B are symmetric, so only the tiles on and below the diagonal are computed, the others mirrored.
// Two steps at a time, where n is twice m or more: A' = (B A) B stands for the Gram product of the X between them, which is
// never formed, and X <- (B' B) X: three symmetric m^3 products instead of m^2 n + 2 m^2 n, and X is read and
// written once less (24 matrices of 4096 x 1024, bf16: 1988 us step by step, 1606 so).  A's rounding errors grow by a^2 in A' and
// those of B' B reach X without an A between, so never two such pairs in a row, and only where the first step
// multiplies by little (OR_PAIR_GROWTH).  With (2, 1, 2) of five usual steps a matrix of noise is as far off as step by step
// (320 x 704 bf16: 2.15e-3 and 2.09e-3), one of rank 2, 300 times as large as noise, 1.3 times (3.2e-3 and 2.5e-3); with (2, 2, 1)
// noise is up to 1.5 times, and with all five at once 0.2.
//
// Numbers.  The iteration multiplies the smallest singular values by a^steps (485 for five of the usual steps), and any
// error in their directions with them.  The operands of the products are fp16, scaled by powers of two that keep them
// in range: 11 bits where bf16 has 8, at the same rate (relative error of the result 1.2e-3 instead of 1e-2 for a
// matrix of noise).  X can be held as the sum of two fp16 planes, hi and lo, 22 bits.
//   bf16 matrices: the first X is G times a power of two, exact in one plane (the rest of the norm goes into the first
//   step's factors).  The products take the hi planes; while what follows may multiply an error by more than
//   OR_CARRY, X is stored in both planes and X <- B hi + a lo, so that what is carried over is not rounded to 11
//   bits (a matrix of low rank and a little noise: 4e-4; with every X in one plane 3e-3, in bf16 0.14).  Up to
//   m = OR_SMALL, where A and B cost little, they have two planes, too (64 x 512: 1.75e-3 instead of 2.4e-3 with the
//   1.66e-3 of rounding the result to bf16).
//   fp32 matrices: two planes everywhere, every product is hi lo + lo hi + hi hi.
//   Where |G| is far below eps, X stays small for many steps (it grows by a in each).  Held times powers of two that
//   leave room for singular values near 1 it would lose its bits below fp16's range, so each matrix has powers of
//   two of its own beside those of all (or_load_kernel; |G| = 1e-15 and eps = 1e-7, 300 x 400 fp32: off by 2.2e-2 without
//   them, 1.6e-7 so).  A has none: where that would matter, B = a I to the last bit.
// Sums are fp32 in the matrix cores, the norm's fp64.  The cores cut a sum off where it leaves fp32: each 16 terms added
// to a sum of S take up to 2^-23 S from it, always towards zero, so the small products come first (16 x 4099 fp32:
// 7.2e-6 with hi hi first).
#pragma once
#include "mfma_tiles.h"
#include "rowvec.h"

namespace flce {

typedef _Float16 f16_t;
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int OR_MATRICES = 120;   // a launch's arguments stay below 4 KB
constexpr int OR_PAD = 64;         // rows and columns are padded with zeros to whole K steps
constexpr int OR_NORM_BLOCKS = 64; // workgroups that add up a matrix's squares
constexpr int OR_MAX_STEPS = 32;

constexpr int OR_SMALL = 256;      // bf16: A and B in two planes up to this many (padded) rows
constexpr float OR_CARRY = 16.0f;

// A = X X^T, B = a I + b A + c A A, A B (of symmetric matrices that commute: symmetric), X <- B X, out = s B X
enum { OR_GRAM = 0, OR_POLY = 1, OR_MULTIPLY = 2, OR_APPLY = 3, OR_LAST = 4 };
// A launch does whole products, or K ranges of them whose sums it leaves, or adds those up and writes the results.
enum { OR_WHOLE = 0, OR_RANGES = 1, OR_JOIN = 2 };

struct OrArgs {
    const f16_t *X, *A, *B;      // planes, of the first matrix; X: rows of [hi np | lo np], A and B of [hi mp (| lo mp)]
    int ldx, lda;                // from row to row
    f16_t* to;                   // the product's, unless OR_LAST
    int64_t stride_x, stride_a;  // elements from one matrix to the next
    int mp, np;                  // m and n, padded
    int count;
    int tiles_m, tiles_n, tiles;   // of a matrix
    // to = alpha * (the accumulated product) + beta * A (OR_POLY), beta * X's lo plane (add_lo), diagonal (OR_POLY)
    float alpha, beta, diagonal;
    int add_lo, put_lo;          // OR_APPLY, OR_LAST: X's lo plane is added; the result has one
    const double* size;          // of each matrix, OR_MAX_STEPS: X_k is what is held times size[k]
    int step, next;              // of the X that is read, of the one that is written (not OR_LAST)
    int ranges;                  // of K
    float* part;                 // the ranges' sums
    int rows, cols;              // OR_LAST: of out
    void* out[OR_MATRICES];
};
struct OrLoadArgs {
    const void* in[OR_MATRICES];
    double* partial;             // OR_NORM_BLOCKS per matrix
    double* size;                // of each matrix, OR_MAX_STEPS: see OrArgs
    int steps;
    int16_t growth[OR_MAX_STEPS]; // X_k is at most 2^(growth[k] - bits) of what its exponent allows where X_0 is at most 2^-bits
    f16_t* X;
    int64_t stride_x;
    int rows, cols, mp, np, ldx;
    int planes;                  // of X that are read
    int exponent;                // the largest element of the first X may be 2 to this
    double eps;
};

__device__ __forceinline__ f32x16 or_mfma(bf16x8 b, bf16x8 a, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, b), __builtin_bit_cast(f16x8, a), c, 0, 0, 0);
}
// Adds the product of the operands' blocks i and j; TURN: to its transpose.
template <bool TURN, int W>
__device__ __forceinline__ void or_multiply(f32x16 (&acc)[W][W], int i, int j, bf16x8 a, bf16x8 b) {
    if constexpr (TURN) acc[j][i] = or_mfma(a, b, acc[j][i]);
    else acc[i][j] = or_mfma(b, a, acc[i][j]);
}

// N values as two planes: their hi plane, and what it leaves of them.  (Each value is made to be an fp32 number first, and each
// pair of the hi plane to be in a register: a product that the compiler rounds to fp16 at once for the one plane and by way of
// fp32 for the other gives two his now and then.  Pairs take half the conversions, and what is left is one mixed multiply-add:
// 4 x 64 x 512 fp32 123 us before, 119 so; large matrices, which the power limit holds back, no difference.)
template <int N>
__device__ __forceinline__ void or_hi(float (&v)[N], uint32_t (&hi)[N / 2]) {
#pragma unroll
    for (int p = 0; p < N / 2; ++p) {
        asm("" : "+v"(v[2 * p]));
        asm("" : "+v"(v[2 * p + 1]));
        hi[p] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{v[2 * p], v[2 * p + 1]}), f16x2));
        asm("" : "+v"(hi[p]));
    }
}
template <int N>
__device__ __forceinline__ void or_lo(const float (&v)[N], const uint32_t (&hi)[N / 2], uint32_t (&lo)[N / 2]) {
#pragma unroll
    for (int p = 0; p < N / 2; ++p) {
        const f16x2 h = __builtin_bit_cast(f16x2, hi[p]);
        const float l0 = fmaf((float)h[0], -1.0f, v[2 * p]), l1 = fmaf((float)h[1], -1.0f, v[2 * p + 1]);
        lo[p] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{l0, l1}), f16x2));
    }
}

// Squares of a matrix; workgroup (p, matrix) adds up its share.  Those of a vector in fp32, these sums in fp64; a vector
// whose sum leaves the middle of fp32's range (or is zero, infinite or NaN) is taken in fp64 as a whole, where no
// square of an fp32 value overflows or vanishes.
template <typename T>
__global__ __launch_bounds__(256) void or_norm_kernel(OrLoadArgs a) {
    constexpr int N = RowVec<T>::N, AHEAD = 8;
    __shared__ double red[4];
    const T* in = static_cast<const T*>(a.in[blockIdx.y]);
    const int64_t all = (int64_t)a.rows * a.cols;
    const int nfull = (int)(all / N), rem = (int)(all % N);
    double s = 0.0;
    for (int v = (int)blockIdx.x * (AHEAD * 256) + (int)threadIdx.x; v < nfull; v += OR_NORM_BLOCKS * AHEAD * 256) {
        u32x4 raw[AHEAD];   // (all loads before the first sum; past the end the last vector again, which counts as zeros)
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) raw[k] = *reinterpret_cast<const u32x4_any*>(in + (int64_t)min(v + k * 256, nfull - 1) * N);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            float f[N], q = 0.f;
            RowVec<T>::unpack(v + k * 256 < nfull ? raw[k] : u32x4{0, 0, 0, 0}, f);
#pragma unroll
            for (int e = 0; e < N; ++e) q = fmaf(f[e], f[e], q);
            double d = (double)q;
            if (!(q > 0x1p-60f && q < 0x1p120f)) {
                d = 0.0;
#pragma unroll
                for (int e = 0; e < N; ++e) d = fma((double)f[e], (double)f[e], d);
            }
            s += d;
        }
    }
    if (blockIdx.x == OR_NORM_BLOCKS - 1 && (int)threadIdx.x < rem) {
        const double x = (double)to_f32(in[(int64_t)nfull * N + threadIdx.x]);
        s = fma(x, x, s);
    }
    s = wave_sum(s);
    if (threadIdx.x % WAVE == 0) red[threadIdx.x / WAVE] = s;
    __syncthreads();
    if (threadIdx.x == 0) a.partial[(int64_t)blockIdx.y * OR_NORM_BLOCKS + blockIdx.x] = red[0] + red[1] + red[2] + red[3];
}

// The first X: a workgroup writes 64 x 64 elements of G times the power of two that brings its norm to 2^exponent, zeros
// where the matrix ends.  TALL: it is turned around in LDS.  The factor that is left, norm / (norm + eps) up to a power
// of two, is X_0's size (see OrArgs), and the powers of two that norm / (norm + eps) lets the others be held larger by.
template <typename T, bool TALL>
__global__ __launch_bounds__(256) void or_load_kernel(OrLoadArgs a) {
    constexpr int N = RowVec<T>::N, LANES = 64 / N;   // lanes per row of the tile
    __shared__ float tile[64][65];
    const int tn = a.np / 64, m0 = (int)blockIdx.x / tn * 64, n0 = (int)blockIdx.x % tn * 64, matrix = blockIdx.y;
    const T* in = static_cast<const T*>(a.in[matrix]);
    double ss = 0.0;
    for (int p = 0; p < OR_NORM_BLOCKS; ++p) ss += a.partial[(int64_t)matrix * OR_NORM_BLOCKS + p];
    const double norm = sqrt(ss);
    const bool usual = norm > 0.0 && norm - norm == 0.0;
    const int e = usual ? ilogb(norm) + 1 : 0;   // norm <= 2^e
    const double scale = ldexp(1.0, a.exponent - e);
    if (blockIdx.x == 0 && (int)threadIdx.x < a.steps) {   // (zeros stay zeros; infinities and NaN make all of the result NaN)
        const int k = threadIdx.x, bits = usual ? -1 - ilogb(norm / (norm + a.eps)) : 0;   // norm / (norm + eps) <= 2^-bits
        const double first = usual ? ldexp(1.0, e) / (norm + a.eps) : norm == 0.0 ? 1.0 : __builtin_nan("");
        a.size[matrix * OR_MAX_STEPS + k] = k == 0 ? first : bits > 0 ? ldexp(1.0, -max(0, bits - a.growth[k])) : 1.0;
    }
    const int r0 = TALL ? n0 : m0, c0 = TALL ? m0 : n0;   // the tile's origin in the matrix
    for (int i = threadIdx.x; i < 64 * LANES; i += 256) {
        const int r = i / LANES, c = i % LANES * N;
        float f[N];
#pragma unroll
        for (int k = 0; k < N; ++k) f[k] = 0.f;
        if (r0 + r < a.rows) {
            const int left = a.cols - c0 - c;
            RowVec<T>::unpack(row_load(in + (int64_t)(r0 + r) * a.cols + c0 + c, 0, left >= N ? 1 : 0, left > 0 ? left : 0), f);
        }
#pragma unroll
        for (int k = 0; k < N; ++k) tile[r][c + k] = (float)((double)f[k] * scale);
    }
    __syncthreads();
    f16_t* X = a.X + matrix * a.stride_x;
    for (int i = threadIdx.x; i < 64 * 8; i += 256) {
        const int r = i / 8, c = i % 8 * 8;
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = TALL ? tile[c + k][r] : tile[r][c + k];
        uint32_t hi[4], lo[4];
        or_hi(v, hi);
        f16_t* to = X + (int64_t)(m0 + r) * a.ldx + n0 + c;
        *reinterpret_cast<u32x4*>(to) = u32x4{hi[0], hi[1], hi[2], hi[3]};
        if (a.planes == 2) {
            or_lo(v, hi, lo);
            *reinterpret_cast<u32x4*>(to + a.np) = u32x4{lo[0], lo[1], lo[2], lo[3]};
        }
    }
}

// A workgroup's K loop over nk K steps, from the first loads on, up to the last step's last sub-step, whose fragments are
// left in raw_a[1], raw_b[1] (or_last_quarter multiplies them; loads past the end are still under way: or_drain).  TURN: of
// the product's transpose, whose rows are the operand b's (the matrix instruction takes its operands the other way round).  The
// loop of fg_product (gemm_bf16_nt.h), which stays as it is there: as a function that both call it compiled to other
// code for those products.  acc: zeros.  smem: fg_lds_bytes(TILE) of LDS.
template <bool TURN, bool A_KM, bool B_KM, int TILE, int ORDER, int W>
__device__ __forceinline__ void or_k_loop(FgOperand<A_KM, TILE, ORDER>& opa, FgOperand<B_KM, TILE, ORDER>& opb, int nk,
                                          unsigned char* smem, int uwave, f32x16 (&acc)[W][W], FgRaw<A_KM> (&raw_a)[2][W],
                                          FgRaw<B_KM> (&raw_b)[2][W]) {
    static_assert(W == TILE / 64, "32 x 32 MFMA tiles per wavefront and direction");
    constexpr int SLOT = fg_slot_bytes(TILE);
    const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem;

    // Workgroup barrier of the pipeline.  Loads complete in order and every
    // wavefront issues NL = TILE / 32 per slot, so "at most NL outstanding" means everything
    // but the youngest slot (the A tile two steps ahead) has landed.  All LDS
    // reads of the step are complete as well, so its two slots can be refilled.
    auto pipeline_barrier = [&]() {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(TILE / 32) : "memory");
    };

    // One quarter of a K step: the 16 MFMAs of one K=16 sub-step on the fragments in
    // register buffer MB (TILE 256; 4 for TILE 128), interleaved with the 8 (4) fragment reads of sub-step KK of the
    // tile in slots (SA, SB) into buffer 1-MB (one fragment per MFMA, in the order
    // a0 b0 b1 b2 b3 a1 a2 a3 in which the next quarter consumes them), and with 4 of
    // the 16 loads of the step, one behind every fourth MFMA (DMA = 1: loads R0..R0+3
    // of the B tile of step kt into slot SD, DMA = 2: of the A tile).  Loads issued in
    // bursts fill the memory pipe's queue and stall the wavefront, and with it the
    // matrix pipe: measured 500 extra cycles for 8 back-to-back loads.
    auto quarter = [&](auto mb_, auto kk_, auto sa_, auto sb_, auto dma_, auto sd_, auto r0_, int kt) {
        constexpr int MB = decltype(mb_)::value, RB = 1 - MB, KK = decltype(kk_)::value;
        constexpr int SA = decltype(sa_)::value, SB = decltype(sb_)::value;
        constexpr int DMA = decltype(dma_)::value, SD = decltype(sd_)::value, R0 = decltype(r0_)::value;
        if constexpr (DMA == 1 && R0 == 0) opb.before_step(kt);
        if constexpr (DMA == 2 && R0 == 0) opa.before_step(kt);
        fg_wait(raw_a[MB], raw_b[MB]);
        bf16x8 fa[W], fb[W];
#pragma unroll
        for (int i = 0; i < W; ++i) {
            fa[i] = fg_value(raw_a[MB][i]);
            fb[i] = fg_value(raw_b[MB][i]);
        }
        const unsigned sa_addr = lds0 + SA * SLOT, sb_addr = lds0 + SB * SLOT;
        __builtin_amdgcn_sched_barrier(0);
#define FG_MFMA(q) or_multiply<TURN>(acc, (q) / W, (q) % W, fa[(q) / W], fb[(q) % W])
#define FG_DMA(n)                                                          \
        if constexpr (DMA == 1) opb.load_one(smem, SD, kt, uwave, R0 + (n));   \
        if constexpr (DMA == 2) opa.load_one(smem, SD, kt, uwave, R0 + (n))
#define FG_END __builtin_amdgcn_sched_barrier(0)
        if constexpr (W == 2) {
            FG_MFMA(0); fg_issue<KK, 0>(raw_a[RB][0], opa, sa_addr); fg_issue<KK, 0>(raw_b[RB][0], opb, sb_addr); FG_END;
            FG_MFMA(1); fg_issue<KK, 1>(raw_b[RB][1], opb, sb_addr); FG_DMA(0); FG_END;
            FG_MFMA(2); fg_issue<KK, 1>(raw_a[RB][1], opa, sa_addr); FG_END;
            FG_MFMA(3); FG_DMA(1); FG_END;
        } else {
        FG_MFMA(0);  fg_issue<KK, 0>(raw_a[RB][0], opa, sa_addr); FG_END;
        FG_MFMA(1);  fg_issue<KK, 0>(raw_b[RB][0], opb, sb_addr); FG_END;
        FG_MFMA(2);  fg_issue<KK, 1>(raw_b[RB][1], opb, sb_addr); FG_DMA(0); FG_END;
        FG_MFMA(3);  fg_issue<KK, 2>(raw_b[RB][2], opb, sb_addr); FG_END;
        FG_MFMA(4);  fg_issue<KK, 3>(raw_b[RB][3], opb, sb_addr); FG_END;
        FG_MFMA(5);  fg_issue<KK, 1>(raw_a[RB][1], opa, sa_addr); FG_END;
        FG_MFMA(6);  fg_issue<KK, 2>(raw_a[RB][2], opa, sa_addr); FG_DMA(1); FG_END;
        FG_MFMA(7);  fg_issue<KK, 3>(raw_a[RB][3], opa, sa_addr); FG_END;
        FG_MFMA(8);  FG_END;
        FG_MFMA(9);  FG_END;
        FG_MFMA(10); FG_DMA(2); FG_END;
        FG_MFMA(11); FG_END;
        FG_MFMA(12); FG_END;
        FG_MFMA(13); FG_END;
        FG_MFMA(14); FG_DMA(3); FG_END;
        FG_MFMA(15); FG_END;
        }
#undef FG_MFMA
#undef FG_DMA
#undef FG_END
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    using I2 = std::integral_constant<int, 2>;
    using I3 = std::integral_constant<int, 3>;

    // One K step.  PH = t % 5 fixes the slots: A(t) in (2 PH) % 5, B(t) in
    // (2 PH + 1) % 5; B(t+1) refills the slot A(t-1) left, A(t+2) the slot B(t-1)
    // left.  The fourth K=16 sub-step of a tile is multiplied in the first quarter
    // of the next step, behind the barrier, while the new fragments arrive.  Tiles
    // past the end are loaded but never consumed (the descriptor returns zeros
    // past its range), which keeps the steady state free of branches.
    auto step = [&](auto phase, int t) {
        constexpr int PH = decltype(phase)::value;
        using SA = std::integral_constant<int, (2 * PH) % 5>;
        using SB = std::integral_constant<int, (2 * PH + 1) % 5>;
        using SB1 = std::integral_constant<int, (2 * PH + 3) % 5>;
        using SA2 = std::integral_constant<int, (2 * PH + 4) % 5>;
        using I4 = std::integral_constant<int, TILE / 64>;   // half of a tile's loads
        quarter(I1{}, I0{}, SA{}, SB{}, I1{}, SB1{}, I0{}, t + 1);   // MFMA: sub-step 3 of tile t-1
        quarter(I0{}, I1{}, SA{}, SB{}, I1{}, SB1{}, I4{}, t + 1);   // MFMA: sub-step 0
        quarter(I1{}, I2{}, SA{}, SB{}, I2{}, SA2{}, I0{}, t + 2);   // MFMA: sub-step 1
        quarter(I0{}, I3{}, SA{}, SB{}, I2{}, SA2{}, I4{}, t + 2);   // MFMA: sub-step 2
        pipeline_barrier();
    };

    opa.load(smem, 0, 0, uwave);
    opb.load(smem, 1, 0, uwave);
    opa.load(smem, 2, 1, uwave);
#pragma unroll
    for (int i = 0; i < W; ++i) {        // the first step has no previous sub-step: add zero
        fg_zero(raw_a[1][i]);
        fg_zero(raw_b[1][i]);
    }
    pipeline_barrier();
    int t = 0;
    for (; t + 5 <= nk; t += 5) {
        step(std::integral_constant<int, 0>{}, t);
        step(std::integral_constant<int, 1>{}, t + 1);
        step(std::integral_constant<int, 2>{}, t + 2);
        step(std::integral_constant<int, 3>{}, t + 3);
        step(std::integral_constant<int, 4>{}, t + 4);
    }
    if (t < nk) step(std::integral_constant<int, 0>{}, t++);
    if (t < nk) step(std::integral_constant<int, 1>{}, t++);
    if (t < nk) step(std::integral_constant<int, 2>{}, t++);
    if (t < nk) step(std::integral_constant<int, 3>{}, t++);
}

// Sub-step 3 of the last K step.
template <bool TURN, bool A_KM, bool B_KM, int W>
__device__ __forceinline__ void or_last_quarter(f32x16 (&acc)[W][W], FgRaw<A_KM> (&raw_a)[2][W], FgRaw<B_KM> (&raw_b)[2][W]) {
    fg_wait(raw_a[1], raw_b[1]);
#pragma unroll
    for (int i = 0; i < W; ++i)
#pragma unroll
        for (int j = 0; j < W; ++j) or_multiply<TURN>(acc, i, j, fg_value(raw_a[1][i]), fg_value(raw_b[1][j]));
}

// The same for operands in two planes and tiles of 128: a K step has both planes of both operands, and takes the three
// products of them, 48 MFMAs per wavefront between two barriers instead of three times 16 (2 x 1000 x 2047 fp32:
// 457 us with the three one after the other, 381 so).  The small products have sums of their own.
// A slot of the ring holds [hi | lo] of an operand's tile, 32 KB, so one workgroup has the LDS of a CU; fragments
// raw[.][0 .. 1] are of the hi plane, [2 .. 3] of the lo plane.  lo_a, lo_b: bytes from a plane to the other.
template <bool TURN>
__device__ __forceinline__ void or_planes_multiply(f32x16 (&acc)[2][2], f32x16 (&small)[2][2], const bf16x8 (&fa)[4], const bf16x8 (&fb)[4], int q) {
    const int i = q / 2 % 2, j = q % 2;
    if (q < 4) or_multiply<TURN>(small, i, j, fa[i], fb[2 + j]);
    else if (q < 8) or_multiply<TURN>(acc, i, j, fa[i], fb[j]);
    else or_multiply<TURN>(small, i, j, fa[2 + i], fb[j]);
}
template <bool TURN, bool B_KM>
__device__ __forceinline__ void or_planes_loop(const FgOperand<false, 128>& opa, const FgOperand<B_KM, 128>& opb, int lo_a, int lo_b, int nk,
                                               unsigned char* smem, int uwave, f32x16 (&acc)[2][2], f32x16 (&small)[2][2]) {
    constexpr int PLANE = fg_slot_bytes(128), SLOT = 2 * PLANE;
    const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem;
    FgRaw<false> raw_a[2][4];
    FgRaw<B_KM> raw_b[2][4];
    auto pipeline_barrier = [&]() { asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)\n\ts_barrier" ::: "memory"); };   // (all but the youngest slot)
    // one of the 8 loads of a wavefront for K step kt into a slot
    auto load_one = [&](const auto& op, int lo, int slot, int kt, int r) {
        fg_load_lds(op.rsrc, smem + slot * SLOT + r / 4 * PLANE + uwave * 1024 + r % 4 * 4096, op.off[r % 4], kt * op.kstep + r / 4 * lo);
    };
    auto values = [&](auto mb_, bf16x8 (&fa)[4], bf16x8 (&fb)[4]) {
        constexpr int MB = decltype(mb_)::value;
        fg_wait(raw_a[MB], raw_b[MB]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            fa[i] = fg_value(raw_a[MB][i]);
            fb[i] = fg_value(raw_b[MB][i]);
        }
    };
    // One sub-step of K = 16: see or_k_loop.
    auto quarter = [&](auto mb_, auto kk_, auto sa_, auto sb_, auto dma_, auto sd_, auto r0_, int kt) {
        constexpr int RB = 1 - decltype(mb_)::value, KK = decltype(kk_)::value, DMA = decltype(dma_)::value, SD = decltype(sd_)::value;
        constexpr int R0 = decltype(r0_)::value;
        bf16x8 fa[4], fb[4];
        values(mb_, fa, fb);
        const unsigned a_hi = lds0 + decltype(sa_)::value * SLOT, b_hi = lds0 + decltype(sb_)::value * SLOT, a_lo = a_hi + PLANE, b_lo = b_hi + PLANE;
        __builtin_amdgcn_sched_barrier(0);
#define OR_MFMA(q) or_planes_multiply<TURN>(acc, small, fa, fb, q)
#define OR_DMA(n) \
        if constexpr (DMA == 1) load_one(opb, lo_b, SD, kt, R0 + (n)); \
        else load_one(opa, lo_a, SD, kt, R0 + (n))
#define OR_END __builtin_amdgcn_sched_barrier(0)
        OR_MFMA(0);  fg_issue<KK, 0>(raw_a[RB][0], opa, a_hi); OR_END;
        OR_MFMA(1);  fg_issue<KK, 0>(raw_b[RB][2], opb, b_lo); OR_END;
        OR_MFMA(2);  fg_issue<KK, 1>(raw_b[RB][3], opb, b_lo); OR_DMA(0); OR_END;
        OR_MFMA(3);  fg_issue<KK, 1>(raw_a[RB][1], opa, a_hi); OR_END;
        OR_MFMA(4);  fg_issue<KK, 0>(raw_b[RB][0], opb, b_hi); OR_END;
        OR_MFMA(5);  fg_issue<KK, 1>(raw_b[RB][1], opb, b_hi); OR_DMA(1); OR_END;
        OR_MFMA(6);  fg_issue<KK, 0>(raw_a[RB][2], opa, a_lo); OR_END;
        OR_MFMA(7);  fg_issue<KK, 1>(raw_a[RB][3], opa, a_lo); OR_END;
        OR_MFMA(8);  OR_DMA(2); OR_END;
        OR_MFMA(9);  OR_END;
        OR_MFMA(10); OR_DMA(3); OR_END;
        OR_MFMA(11); OR_END;
#undef OR_MFMA
#undef OR_DMA
#undef OR_END
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    using I2 = std::integral_constant<int, 2>;
    using I3 = std::integral_constant<int, 3>;
    using I4 = std::integral_constant<int, 4>;
    auto step = [&](auto phase, int t) {
        constexpr int PH = decltype(phase)::value;
        using SA = std::integral_constant<int, (2 * PH) % 5>;
        using SB = std::integral_constant<int, (2 * PH + 1) % 5>;
        using SB1 = std::integral_constant<int, (2 * PH + 3) % 5>;
        using SA2 = std::integral_constant<int, (2 * PH + 4) % 5>;
        quarter(I1{}, I0{}, SA{}, SB{}, I1{}, SB1{}, I0{}, t + 1);
        quarter(I0{}, I1{}, SA{}, SB{}, I1{}, SB1{}, I4{}, t + 1);
        quarter(I1{}, I2{}, SA{}, SB{}, I2{}, SA2{}, I0{}, t + 2);
        quarter(I0{}, I3{}, SA{}, SB{}, I2{}, SA2{}, I4{}, t + 2);
        pipeline_barrier();
    };
#pragma unroll
    for (int r = 0; r < 8; ++r) load_one(opa, lo_a, 0, 0, r);
#pragma unroll
    for (int r = 0; r < 8; ++r) load_one(opb, lo_b, 1, 0, r);
#pragma unroll
    for (int r = 0; r < 8; ++r) load_one(opa, lo_a, 2, 1, r);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        fg_zero(raw_a[1][i]);
        fg_zero(raw_b[1][i]);
    }
    pipeline_barrier();
    int t = 0;
    for (; t + 5 <= nk; t += 5) {
        step(I0{}, t);
        step(I1{}, t + 1);
        step(I2{}, t + 2);
        step(I3{}, t + 3);
        step(I4{}, t + 4);
    }
    if (t < nk) step(I0{}, t++);
    if (t < nk) step(I1{}, t++);
    if (t < nk) step(I2{}, t++);
    if (t < nk) step(I3{}, t++);
    bf16x8 fa[4], fb[4];
    values(I1{}, fa, fb);
#pragma unroll
    for (int q = 0; q < 12; ++q) or_planes_multiply<TURN>(acc, small, fa, fb, q);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int g = 0; g < 16; ++g) acc[i][j][g] += small[i][j][g];
}

// The loads of the tiles past the end still target LDS: let them land, for every
// wavefront of the workgroup, before LDS is reused (and before the workgroup can
// retire and its LDS be handed to another one).
__device__ __forceinline__ void or_drain() { asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory"); }

// OrArgs' alpha and beta, with the sizes of a matrix's X, and (OR_LAST) a power of two apart: the result times a small
// size may be an ordinary number while alpha alone is below fp32's normal range.
struct OrFactors {
    float alpha, beta;
    int exponent;
};
template <int PRODUCT>
__device__ __forceinline__ OrFactors or_factors(const OrArgs& a, int matrix) {
    auto uniform = [](float f) { return __uint_as_float((uint32_t)__builtin_amdgcn_readfirstlane((int)__float_as_uint(f))); };
    if constexpr (PRODUCT == OR_POLY || PRODUCT == OR_MULTIPLY) return {a.alpha, a.beta, 0};
    const double* size = a.size + matrix * OR_MAX_STEPS;
    const double from = size[a.step];
    if constexpr (PRODUCT == OR_GRAM) return {uniform((float)(a.alpha * from * from)), 0.0f, 0};
    if constexpr (PRODUCT == OR_APPLY) {
        const double f = from / size[a.next];
        return {uniform((float)(a.alpha * f)), uniform((float)(a.beta * f)), 0};
    }
    const double alpha = a.alpha * from;
    const int e = alpha != 0.0 && alpha - alpha == 0.0 ? ilogb(alpha) : 0;
    return {uniform((float)ldexp(alpha, -e)), uniform((float)ldexp(a.beta * from, -e)), __builtin_amdgcn_readfirstlane(e)};
}

// Writes a wavefront's part of a tile out, 32 rows at a time through LDS (see FgOut in gemm_bf16_nt.h for the layout of
// the accumulators), as planes of 8 values per lane, the mirrored tile too; or (OR_LAST) rounded to out.  Where the matrix
// is tall, the accumulators hold the transpose (24 matrices of 4096 x 1024, bf16: turning the finished tile around
// took 25 us more).  PL: planes that are multiplied, OUT: of A.
template <int PRODUCT, int PL, int OUT, int TILE, typename OutT, bool TALL>
struct OrOut {
    static constexpr int WN = TILE / 2, W = TILE / 64;
    static constexpr int LANES = WN / 8, ROWS = 64 / LANES, NACC = 32 / ROWS;   // lanes per row, rows and accesses per pass
    static constexpr int PITCH = WN + 4;
    static constexpr bool LAST = PRODUCT == OR_LAST, TURN = LAST && TALL, MIRROR = PRODUCT <= OR_MULTIPLY;
    static constexpr int IN = PRODUCT == OR_POLY ? PL : PRODUCT >= OR_APPLY && PL == 1 ? 1 : 0;   // planes of the addend: A, X's lo
    static constexpr int AHEAD = TURN ? 0 : IN;   // of these, loaded ahead
    static constexpr bool LO_ONLY = PRODUCT >= OR_APPLY;

    __amdgpu_buffer_rsrc_t rsrc_in, rsrc_out;
    int ld, pitch;   // columns of a plane and from row to row, of the addend and of the output
    int rows_all;    // their rows
    int row0, col0;  // of the wavefront's part
    int lane;
    float* stage;
    u32x4 addend[AHEAD ? 2 : 1][NACC][AHEAD ? AHEAD : 1];
    static_assert(64 * PITCH * 4 <= fg_lds_bytes(TILE) / 4, "two passes fit a wavefront's share of LDS");

    __device__ __forceinline__ void init(const f16_t* in, f16_t* to, int ld_, int pitch_, int rows_, bool add, int r0, int c0, unsigned char* smem,
                                         int lane_, int uwave) {
        ld = ld_;
        pitch = pitch_;
        rows_all = rows_;
        row0 = r0;
        col0 = c0;
        lane = lane_;
        stage = reinterpret_cast<float*>(smem + uwave * (fg_lds_bytes(TILE) / 4));
        // (a range of zero bytes makes every load return zero without touching memory)
        if constexpr (IN > 0) rsrc_in = fg_make_rsrc(in, add ? (uint32_t)rows_all * (uint32_t)pitch * 2u : 0u);
        if constexpr (!LAST) rsrc_out = fg_make_rsrc(to, (uint32_t)rows_all * (uint32_t)pitch * 2u);
    }
    // byte offset of 8 values in the first plane, or one past the end
    __device__ __forceinline__ int at(int row, int col) const { return row < rows_all && col < ld ? (row * pitch + col) * 2 : 0x7fffffff; }
    __device__ __forceinline__ int lane_row(int k) const { return k * ROWS + lane / LANES; }
    __device__ __forceinline__ int lane_col() const { return lane % LANES * 8; }

    template <int BUF>
    __device__ __forceinline__ void load_addend(int pass) {
        if constexpr (AHEAD > 0) {
#pragma unroll
            for (int k = 0; k < NACC; ++k) {
                const int off = at(row0 + pass * 32 + lane_row(k), col0 + lane_col());
#pragma unroll
                for (int p = 0; p < IN; ++p)
                    addend[BUF][k][p] = __builtin_amdgcn_raw_buffer_load_b128(rsrc_in, off, (LO_ONLY ? 1 : p) * ld * 2, 0);
            }
        }
    }
    // (Both stores have their whole offset in a vector register.  With part of it in a scalar one the compiler takes the
    // data for read at once and may let the very next instruction overwrite it; on this chip the store then wrote some of
    // the new values: one lo plane in 10^5, more where the memory pipe was full.)
    __device__ __forceinline__ void put_planes(int row, int col, float (&v)[8], bool put_lo) {
        uint32_t hi[4], lo[4];
        or_hi(v, hi);
        const uint32_t off = (uint32_t)at(row, col);
        __builtin_amdgcn_raw_buffer_store_b128(u32x4{hi[0], hi[1], hi[2], hi[3]}, rsrc_out, (int)off, 0, 0);
        if (OUT == 2 && put_lo) {
            or_lo(v, hi, lo);
            __builtin_amdgcn_raw_buffer_store_b128(u32x4{lo[0], lo[1], lo[2], lo[3]}, rsrc_out, (int)(off + 2u * (uint32_t)ld), 0, 0);
        }
    }
    static __device__ __forceinline__ void put_out(OutT* out, int rows, int cols, int row, int col, const float (&v)[8]) {
        if (row >= rows || col >= cols) return;
        OutT* to = out + (int64_t)row * cols + col;
        constexpr int N = RowVec<OutT>::N;
        if (col + 8 <= cols) {
#pragma unroll
            for (int g = 0; g < 8 / N; ++g) {
                float w[N];
#pragma unroll
                for (int e = 0; e < N; ++e) w[e] = v[g * N + e];
                *reinterpret_cast<u32x4_any*>(to + g * N) = RowVec<OutT>::pack(w);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (col + e < cols) to[e] = from_f32<OutT>(v[e]);
        }
    }

    // 4 values of a row of the stage.  Groups of 8 rows have them in another order each: what turned() reads at a time, 8
    // columns of 8 rows that are 8 apart, lies in 64 banks.
    __device__ __forceinline__ f32x4* staged(int row, int group) const {
        return reinterpret_cast<f32x4*>(stage + row * PITCH + (group ^ ((row >> 3) & 7)) * 4);
    }
    // Rows 32 i .. of the wavefront's part, from its accumulators of them; their addend is in buffer BUF.  MIRROR:
    // they are left in half H of the stage, for turned().
    template <int BUF, int H>
    __device__ __forceinline__ void pass(f32x16 (&acc)[W], const OrArgs& a, const OrFactors& f, OutT* out, int i) {
        const int frow = lane & 31, fhalf = lane >> 5;
        const bool put_lo = PRODUCT != OR_APPLY || PL == 2 || a.put_lo;
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float v0 = acc[j][4 * g], v1 = acc[j][4 * g + 1], v2 = acc[j][4 * g + 2], v3 = acc[j][4 * g + 3];
                *staged(H * 32 + frow, 8 * j + 2 * g + fhalf) = f32x4{v0, v1, v2, v3};
            }
        // (the region is the wavefront's own, and LDS executes its accesses in order)
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int k = 0; k < NACC; ++k) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; e += 4) {
                const f32x4 q = *staged(H * 32 + lane_row(k), (lane_col() + e) / 4);
#pragma unroll
                for (int u = 0; u < 4; ++u) v[e + u] = f.alpha * q[u];
            }
            const int row = row0 + 32 * i + lane_row(k), col = col0 + lane_col();
            if constexpr (AHEAD > 0) {
#pragma unroll
                for (int p = IN - 1; p >= 0; --p) {
                    const f16x8 w = __builtin_bit_cast(f16x8, addend[BUF][k][p]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = fmaf(f.beta, (float)w[e], v[e]);
                }
            }
            if constexpr (TURN && IN > 0) {
                if (a.add_lo) {   // (a last step that multiplies an error by more than OR_CARRY: columns of X)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        v[e] = fmaf(f.beta, (float)__builtin_bit_cast(f16_t, __builtin_amdgcn_raw_buffer_load_b16(rsrc_in, at(col + e, row), ld * 2, 0)), v[e]);
                }
            }
            if constexpr (PRODUCT == OR_POLY) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += row == col + e ? a.diagonal : 0.f;
            }
            if constexpr (LAST) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = __builtin_amdgcn_ldexpf(v[e], f.exponent);
                put_out(out, a.rows, a.cols, row, col, v);
            } else {
                put_planes(row, col, v, put_lo);
            }
            if constexpr (MIRROR) {
#pragma unroll
                for (int e = 0; e < 8; e += 4)
                    *staged(H * 32 + lane_row(k), (lane_col() + e) / 4) = f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]};
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    // The 64 rows (PASSES = 2) or 32 in the stage, whose first is row 32 i, as columns: whole lines of 128 bytes of 16-bit
    // values.
    template <int PASSES>
    __device__ __forceinline__ void turned(const OrArgs& a, int i) {
        constexpr int LPC = 4 * PASSES;   // lanes per column
        const bool put_lo = PRODUCT != OR_APPLY || PL == 2 || a.put_lo;
#pragma unroll
        for (int k = 0; k < WN * LPC / 64; ++k) {
            const int c = lane / LPC + 64 / LPC * k, r = lane % LPC * 8;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = reinterpret_cast<const float*>(staged(r + e, c / 4))[c % 4];
            put_planes(col0 + c, row0 + 32 * i + r, v, put_lo);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    // All of it; load_addend<0>(0) has been issued before.
    __device__ __forceinline__ void write(f32x16 (&acc)[W][W], const OrArgs& a, const OrFactors& f, int matrix, bool mirror) {
        OutT* out = LAST ? static_cast<OutT*>(a.out[matrix]) : nullptr;
#pragma unroll
        for (int i = 0; i < W; i += 2) {
            load_addend<AHEAD ? 1 : 0>(i + 1);
            pass<0, 0>(acc[i], a, f, out, i);
            if (i + 2 < W) load_addend<0>(i + 2);
            pass<AHEAD ? 1 : 0, 1>(acc[i + 1], a, f, out, i + 1);
            if (MIRROR && mirror) turned<2>(a, i);
        }
    }
};

// Tile t of a matrix: of a symmetric product, row by row on and below the diagonal; else OR_GROUP rows at a time, column
// by column among them.
constexpr int OR_GROUP = 4;
template <bool SYMMETRIC>
__device__ __forceinline__ void or_tile(int t, int tiles_m, int tiles_n, int& tm, int& tn) {
    if constexpr (SYMMETRIC) {
        tm = (int)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
        while ((tm + 1) * (tm + 2) / 2 <= t) ++tm;   // (the root may be off by a rounding)
        while (tm * (tm + 1) / 2 > t) --tm;
        tn = t - tm * (tm + 1) / 2;
    } else {
        const int grp = t / (OR_GROUP * tiles_n), first = grp * OR_GROUP, g = min(OR_GROUP, tiles_m - first);
        const int rem = t - grp * OR_GROUP * tiles_n;
        tm = first + rem % g;
        tn = rem / g;
    }
}

// One workgroup per tile of a matrix (and K range of it), 256 x 256, or 128 x 128 and, unless it multiplies both planes, two
// workgroups per CU.
template <int PRODUCT, int PL, int OUT, int TILE, typename OutT, bool TALL, int PART>
__global__ __launch_bounds__(FG_THREADS, TILE == 256 || (PL == 2 && PART != OR_JOIN) ? 1 : 2) void or_product_kernel(OrArgs a) {
    constexpr bool SYMMETRIC = PRODUCT <= OR_MULTIPLY, B_KM = !SYMMETRIC;
    constexpr bool PLANES = PL == 2 && TILE == 128;   // both at a time
    constexpr int ORDER = PL == 2 && !PLANES ? FG_PLANES : FG_PLAIN, W = TILE / 64;
    __shared__ __attribute__((aligned(16))) unsigned char smem[fg_lds_bytes(PLANES && PART != OR_JOIN ? 256 : TILE)];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wm = wave >> 1, wn = wave & 1;
    // workgroups go round-robin to the XCDs: each gets a stretch of tiles, range by range
    const int all = a.tiles * a.count, total = all * (PART == OR_RANGES ? a.ranges : PART == OR_JOIN ? W : 1);
    const int per_xcd = (total + FG_XCDS - 1) / FG_XCDS;
    int seq = (int)blockIdx.x % FG_XCDS * per_xcd + (int)blockIdx.x / FG_XCDS;
    if ((int)blockIdx.x / FG_XCDS >= per_xcd || seq >= total) return;
    const int range = PART == OR_WHOLE ? 0 : seq / all;   // (OR_JOIN: a workgroup does one pass of its wavefronts)
    seq -= range * all;
    const int matrix = seq / a.tiles;
    int tm, tn;
    or_tile<SYMMETRIC>(seq - matrix * a.tiles, a.tiles_m, a.tiles_n, tm, tn);
    tm = __builtin_amdgcn_readfirstlane(tm);
    tn = __builtin_amdgcn_readfirstlane(tn);
    const int m0 = tm * TILE, n0 = tn * TILE;
    const int uwave = __builtin_amdgcn_readfirstlane(wave);

    const f16_t* X = a.X + matrix * a.stride_x;
    const int K = PRODUCT == OR_GRAM ? a.np : a.mp, N = SYMMETRIC ? a.mp : a.np;
    // The sums of a range: accumulators as they lie, 16 bytes per lane.
    auto part_at = [&](int r, int i, int j, int g) {
        return reinterpret_cast<f32x4*>(a.part + ((int64_t)r * all + seq) * (TILE * TILE) + (((i * W + j) * 4 + g) * FG_THREADS + tid) * 4);
    };
    constexpr bool TURN = PRODUCT == OR_LAST && TALL;
    OrOut<PRODUCT, PL, OUT, TILE, OutT, TALL> out;
    auto begin_out = [&]() {
        const int row0 = m0 + __builtin_amdgcn_readfirstlane(wm) * (TILE / 2), col0 = n0 + __builtin_amdgcn_readfirstlane(wn) * (TILE / 2);
        out.init(PRODUCT == OR_POLY ? a.A + matrix * a.stride_a : X, a.to + matrix * (SYMMETRIC ? a.stride_a : a.stride_x), N,
                 SYMMETRIC ? a.lda : a.ldx, a.mp,
                 PRODUCT == OR_POLY || a.add_lo, TURN ? col0 : row0, TURN ? row0 : col0, smem, lane, uwave);
    };
    if constexpr (PART == OR_JOIN) {
        constexpr int AHEAD = 4;   // ranges whose loads are under way
        begin_out();
        const OrFactors factors = or_factors<PRODUCT>(a, matrix);
        out.template load_addend<0>(range);
        f32x16 acc[W];
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int g = 0; g < 16; ++g) acc[j][g] = 0.f;
        for (int r0 = 0; r0 < a.ranges; r0 += AHEAD) {
            f32x4 v[AHEAD][W][4];
#pragma unroll
            for (int r = 0; r < AHEAD; ++r)
#pragma unroll
                for (int j = 0; j < W; ++j)
#pragma unroll
                    for (int g = 0; g < 4; ++g) v[r][j][g] = *part_at(min(r0 + r, a.ranges - 1), range, j, g);
#pragma unroll
            for (int r = 0; r < AHEAD; ++r)
#pragma unroll
                for (int j = 0; j < W; ++j)
#pragma unroll
                    for (int g = 0; g < 16; ++g) acc[j][g] += r0 + r < a.ranges ? v[r][j][g / 4][g % 4] : 0.f;
        }
        OutT* to = PRODUCT == OR_LAST ? static_cast<OutT*>(a.out[matrix]) : nullptr;
        out.template pass<0, 0>(acc, a, factors, to, range);
        if (out.MIRROR && tm != tn) out.template turned<1>(a, range);
    } else {
        // operands: X X^T, A A, A B (rows of symmetric matrices for columns), B X
        constexpr bool RIGHT_M = PRODUCT == OR_POLY || PRODUCT == OR_MULTIPLY;   // the right one is m x m
        const f16_t* left = PRODUCT == OR_GRAM ? X : (PRODUCT >= OR_APPLY ? a.B : a.A) + matrix * a.stride_a;
        const f16_t* right = PRODUCT == OR_POLY ? left : PRODUCT == OR_MULTIPLY ? a.B + matrix * a.stride_a : X;
        const int ldl = PRODUCT == OR_GRAM ? a.ldx : a.lda, ldr = RIGHT_M ? a.lda : a.ldx;
        FgOperand<false, TILE, ORDER> opa;
        FgOperand<B_KM, TILE, ORDER> opb;
        opa.init(reinterpret_cast<const bf16_t*>(left), ldl, m0, a.mp, K, tid, wm);
        opb.init(reinterpret_cast<const bf16_t*>(right), ldr, n0, N, K, tid, wn);
        const int steps = K / FG_BK;
        int k0 = 0, nk = steps;
        if constexpr (PART == OR_RANGES) {
            k0 = (int)((int64_t)steps * range / a.ranges);
            nk = (int)((int64_t)steps * (range + 1) / a.ranges) - k0;
        }
        opa.start_at(k0);
        opb.start_at(k0);
        const int lo_a = (PRODUCT == OR_GRAM ? a.np : a.mp) * 2, lo_b = (RIGHT_M ? a.mp : a.np) * 2;
        if constexpr (ORDER == FG_PLANES) {
            opa.plane_steps = opb.plane_steps = nk;
            opa.plane_bytes = lo_a;
            opb.plane_bytes = lo_b;
            opa.lo_part = 1;
            opb.lo_part = 0;
            nk *= 3;
        }
        OrFactors factors{};
        if constexpr (PART == OR_WHOLE) factors = or_factors<PRODUCT>(a, matrix);   // (its loads end long before the K loop)
        f32x16 acc[W][W];
#pragma unroll
        for (int i = 0; i < W; ++i)
#pragma unroll
            for (int j = 0; j < W; ++j)
#pragma unroll
                for (int g = 0; g < 16; ++g) acc[i][j][g] = 0.f;
        if constexpr (PLANES) {
            f32x16 small[W][W];
#pragma unroll
            for (int i = 0; i < W; ++i)
#pragma unroll
                for (int j = 0; j < W; ++j) small[i][j] = acc[i][j];
            or_planes_loop<TURN>(opa, opb, lo_a, lo_b, nk, smem, uwave, acc, small);
        } else {
            FgRaw<false> raw_a[2][W];
            FgRaw<B_KM> raw_b[2][W];
            or_k_loop<TURN>(opa, opb, nk, smem, uwave, acc, raw_a, raw_b);
            if constexpr (PART == OR_WHOLE) {
                begin_out();
                out.template load_addend<0>(0);
            }
            or_last_quarter<TURN>(acc, raw_a, raw_b);
        }
        if constexpr (PLANES && PART == OR_WHOLE) {
            begin_out();
            out.template load_addend<0>(0);
        }
        or_drain();
        if constexpr (PART == OR_WHOLE) {
            out.write(acc, a, factors, matrix, tm != tn);
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i)
#pragma unroll
                for (int j = 0; j < W; ++j)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const float v0 = acc[i][j][4 * g], v1 = acc[i][j][4 * g + 1], v2 = acc[i][j][4 * g + 2], v3 = acc[i][j][4 * g + 3];
                        *part_at(range, i, j, g) = f32x4{v0, v1, v2, v3};
                    }
        }
    }
}

// All steps of small bf16 matrices between the first Gram product and the last B X, in m x m matrices alone (all of them
// polynomials of A, hence symmetric, and they commute):
//
//     B_k = a I + b A_k + c A_k A_k,   A_{k+1} = B_k A_k B_k,   Q = B_{steps-1} ... B_0,   out = s Q X
//
// One workgroup per matrix, two planes throughout, in LDS.  A's rounding errors (2^-22 of its largest eigenvalue) grow by
// the square of the most that B multiplies by per step, as its smallest eigenvalues do: for bf16 matrices, up to
// OR_ITERATE_GROWTH, little but the result's rounding is left to see (60 x 100 of rank 1, whose other directions are its
// rounding to bf16: five of the usual steps, 19800, 1.8e-3; five that begin with 4.08 and 3.95, 30300, 1.4e-2, and one by
// one, as they are taken, 1.7e-3).  fp32 matrices do not come here (all steps at once cost them up to 2.5 times the error of
// fp32 arithmetic).
// The launches between are what small matrices cost: 4 x 64 x 512 bf16 101 us with three per step, 38 with this one (19 of
// them here, 17 products of 1 us).
constexpr int OR_ITERATE_MOST = 128, OR_ITERATE_STEPS = 8;   // (padded) rows, steps
struct OrIterateArgs {
    const f16_t* A;      // of the first matrix; and where Q goes
    f16_t* Q;
    f16_t* B;            // steps matrices for each
    int64_t stride_a;
    int lda;
    int steps;
    float square[OR_ITERATE_STEPS], linear[OR_ITERATE_STEPS], diagonal[OR_ITERATE_STEPS];   // of B
    float t[OR_ITERATE_STEPS], next[OR_ITERATE_STEPS], q[OR_ITERATE_STEPS];                 // powers of two of B A, (B A) B, B Q
};

template <int MP>
__global__ __launch_bounds__(256) void or_iterate_kernel(OrIterateArgs a) {
    constexpr int W = MP / 64, PITCH = MP + 8;   // (rows 16 bytes further by 4 banks each)
    __shared__ __attribute__((aligned(16))) f16_t lds[2][2][MP * PITCH];   // two matrices of two planes
    const int tid = threadIdx.x, lane = tid % WAVE, wave = tid / WAVE;
    const int row0 = wave / 2 * (MP / 2), col0 = wave % 2 * (MP / 2), frow = lane & 31, fhalf = lane >> 5;
    const int64_t matrix = blockIdx.x;

    f32x16 acc[W][W];
    // acc = left * right (symmetric, so its rows are its columns), the small products first
    auto product = [&](const f16_t (&left)[2][MP * PITCH], const f16_t (&right)[2][MP * PITCH]) {
#pragma unroll
        for (int i = 0; i < W; ++i)
#pragma unroll
            for (int j = 0; j < W; ++j)
#pragma unroll
                for (int g = 0; g < 16; ++g) acc[i][j][g] = 0.f;
        auto fragment = [&](const f16_t* m, int r0, int k) {
            return *reinterpret_cast<const bf16x8*>(m + (r0 + frow) * PITCH + k * 16 + fhalf * 8);
        };
        auto part = [&](int pl, int pr) {
#pragma unroll
            for (int k = 0; k < MP / 16; ++k) {
                bf16x8 fa[W], fb[W];
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    fa[i] = fragment(left[pl], row0 + 32 * i, k);
                    fb[i] = fragment(right[pr], col0 + 32 * i, k);
                }
#pragma unroll
                for (int i = 0; i < W; ++i)
#pragma unroll
                    for (int j = 0; j < W; ++j) acc[i][j] = or_mfma(fb[j], fa[i], acc[i][j]);
            }
        };
        part(0, 1);
        part(1, 0);
        part(0, 0);
    };
    // what to do with four consecutive values of a row of acc
    auto each = [&](auto what) {
#pragma unroll
        for (int i = 0; i < W; ++i)
#pragma unroll
            for (int j = 0; j < W; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = acc[i][j][4 * g + e];
                    what(row0 + 32 * i + frow, col0 + 32 * j + 8 * g + 4 * fhalf, v);
                }
    };
    typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
    auto put = [&](f16_t (&to)[2][MP * PITCH], float scale) {
        each([&](int row, int col, float (&v)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] *= scale;
            uint32_t hi[2], lo[2];
            or_hi(v, hi);
            or_lo(v, hi, lo);
            *reinterpret_cast<uint2*>(&to[0][row * PITCH + col]) = uint2{hi[0], hi[1]};
            *reinterpret_cast<uint2*>(&to[1][row * PITCH + col]) = uint2{lo[0], lo[1]};
        });
    };
    auto fetch = [&](f16_t (&to)[2][MP * PITCH], const f16_t* from) {   // planes in memory: rows of [hi MP | lo MP]
        for (int i = tid; i < MP * MP / 4; i += 256) {
            const int row = i / (MP / 4), at = i % (MP / 4) * 8, plane = at / MP, col = at % MP;
            *reinterpret_cast<u32x4*>(&to[plane][row * PITCH + col]) = *reinterpret_cast<const u32x4*>(from + (int64_t)row * a.lda + at);
        }
    };
    f16_t* Bs = a.B + matrix * a.steps * a.stride_a;
    fetch(lds[0], a.A + matrix * a.stride_a);
    __syncthreads();
    for (int k = 0; k < a.steps; ++k) {
        product(lds[0], lds[0]);
        each([&](int row, int col, float (&v)[4]) {
            const f16x4 hi = *reinterpret_cast<const f16x4*>(&lds[0][0][row * PITCH + col]);
            const f16x4 lo = *reinterpret_cast<const f16x4*>(&lds[0][1][row * PITCH + col]);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = a.square[k] * v[e] + a.linear[k] * ((float)hi[e] + (float)lo[e]) + (row == col + e ? a.diagonal[k] : 0.f);
            uint32_t h[2], l[2];
            or_hi(v, h);
            or_lo(v, h, l);
            *reinterpret_cast<uint2*>(&lds[1][0][row * PITCH + col]) = uint2{h[0], h[1]};
            *reinterpret_cast<uint2*>(&lds[1][1][row * PITCH + col]) = uint2{l[0], l[1]};
            f16_t* to = Bs + k * a.stride_a + (int64_t)row * a.lda + col;
            *reinterpret_cast<uint2*>(to) = uint2{h[0], h[1]};
            *reinterpret_cast<uint2*>(to + MP) = uint2{l[0], l[1]};
        });
        __syncthreads();
        if (k + 1 == a.steps) break;
        product(lds[1], lds[0]);
        __syncthreads();
        put(lds[0], a.t[k]);
        __syncthreads();
        product(lds[0], lds[1]);
        __syncthreads();
        put(lds[0], a.next[k]);
        __syncthreads();
    }
    // Q: the last B is in lds[1], the others (and it) in memory, where this workgroup wrote them
    for (int k = a.steps - 2; k >= 0; --k) {
        fetch(lds[0], Bs + k * a.stride_a);
        __syncthreads();
        product(lds[0], lds[1]);
        __syncthreads();
        put(lds[1], a.q[k]);
        __syncthreads();
    }
    f16_t* Q = a.Q + matrix * a.stride_a;
    for (int i = tid; i < MP * MP / 4; i += 256) {
        const int row = i / (MP / 4), at = i % (MP / 4) * 8, plane = at / MP, col = at % MP;
        *reinterpret_cast<u32x4*>(Q + (int64_t)row * a.lda + at) = *reinterpret_cast<const u32x4*>(&lds[1][plane][row * PITCH + col]);
    }
}

}  // namespace flce
