// Sums over a row within the threads that hold it, and of the partial sums over rows that workgroups leave.
#pragma once
#include "flce_device.h"

namespace flce {

template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
// Sum over the aligned group of 16 or 64 lanes, the same bits in every lane: neighbours within a quad, quads and
// halves of a row of 16 by mirroring, then rows and halves of the wavefront exchanged.
template <int LANES>
__device__ __forceinline__ float lane_sum(float v) {
    static_assert(LANES == 16 || LANES == 64, "");
    v = dpp_add<0xB1>(v);    // quad_perm 1 0 3 2
    v = dpp_add<0x4E>(v);    // quad_perm 2 3 0 1
    v = dpp_add<0x141>(v);   // row_half_mirror
    v = dpp_add<0x140>(v);   // row_mirror
    if constexpr (LANES == 64) {
        const uint32_t a = __float_as_uint(v);
        const auto p = __builtin_amdgcn_permlane16_swap(a, a, false, false);
        v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
        const uint32_t b = __float_as_uint(v);
        const auto q = __builtin_amdgcn_permlane32_swap(b, b, false, false);
        v = __uint_as_float(q[0]) + __uint_as_float(q[1]);
    }
    return v;
}

// K sums over the TPR threads of a row's group, the same values in every one of them.  slot: LDS of these sums
// alone ([K][TPR / 64]; a group of several wavefronts is a whole workgroup), read until the next barrier.
template <int TPR, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], float* slot) {
#pragma unroll
    for (int i = 0; i < K; ++i) v[i] = lane_sum<(TPR < WAVE ? TPR : WAVE)>(v[i]);
    if constexpr (TPR > WAVE) {
        constexpr int NW = TPR / WAVE;
        if ((threadIdx.x & (WAVE - 1)) == 0)
#pragma unroll
            for (int i = 0; i < K; ++i) slot[i * NW + threadIdx.x / WAVE] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < K; ++i) {
            v[i] = slot[i * NW];
#pragma unroll
            for (int w = 1; w < NW; ++w) v[i] += slot[i * NW + w];
        }
    }
}
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* slot) {
    float k[1] = {v};
    row_sums<TPR, 1>(k, slot);
    return k[0];
}
// Threads of a workgroup, rows of it, and a thread's row in it (the same in a whole wavefront, if it is).
template <int TPR> constexpr int row_block = TPR > WAVE ? TPR : 256;
template <int TPR> constexpr int row_groups = row_block<TPR> / TPR;
template <int TPR>
__device__ __forceinline__ int row_group() {
    if constexpr (TPR > WAVE) return 0;
    if constexpr (TPR == WAVE) return __builtin_amdgcn_readfirstlane((int)threadIdx.x / WAVE);
    return (int)threadIdx.x / TPR;
}

// out[g][j] = sum over p of rows [g * parts + p][j] of fp32 partial sums, for up to three sets of them: the two
// gammas (one output row each) and the gate.  As in rmsnorm_dgamma_kernel a workgroup owns some columns of an
// output row (32: lines of 128 bytes), thread (c, q) adds rows q, q + 32, ... of column c, then the 32 sums are added in
// order; in fp64, which costs nothing here and leaves the fp32 sums of a workgroup's own rows as the only ones.  Bound
// by the latency of a thread's loads: eight under way at a time, issued without a condition (3-5 us).
struct PartialSums {
    const float* part[3];
    void* out[3];
    int64_t ld[3];
    int parts[3];
    int first[4];   // the sets' output rows are rows first[i] .. first[i + 1] of the grid
};
constexpr int SUM_COLS = 32, SUM_PARTS = 32;
template <typename T>
static __global__ __launch_bounds__(SUM_COLS * SUM_PARTS) void sum_partials_kernel(PartialSums b, int n) {
    __shared__ double sums[SUM_PARTS][SUM_COLS];
    const int c = threadIdx.x % SUM_COLS, q = threadIdx.x / SUM_COLS;
    const int r = blockIdx.y, j = blockIdx.x * SUM_COLS + c;
    const int set = r >= b.first[2] ? 2 : r >= b.first[1] ? 1 : 0;
    const int g = r - b.first[set], parts = b.parts[set];
    const float* from = b.part[set] + (int64_t)g * parts * n + j;
    double s = 0.0;
    if (j < n)
        for (int p0 = q; p0 < parts; p0 += 8 * SUM_PARTS) {   // (eight loads under way, also where there are fewer)
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = from[(int64_t)min(p0 + k * SUM_PARTS, parts - 1) * n];
#pragma unroll
            for (int k = 0; k < 8; ++k) s += p0 + k * SUM_PARTS < parts ? (double)v[k] : 0.0;
        }
    sums[q][c] = s;
    __syncthreads();
    if (q == 0 && j < n) {
        for (int k = 1; k < SUM_PARTS; ++k) s += sums[k][c];
        (static_cast<T*>(b.out[set]) + (int64_t)g * b.ld[set])[j] = from_f32<T>((float)s);
    }
}

}  // namespace flce
