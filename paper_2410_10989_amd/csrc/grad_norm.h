// Norm over all elements of many tensors, and scaling by it (gradient clipping):
//
//     norm = sqrt(sum_t sum_j g_tj^2)   or   max_t max_j |g_tj|
//     c    = min(1, max_norm / (norm + 1e-6)),  1 where norm is not finite;      out_tj = g_tj c
//
// A launch takes up to GN_TENSORS tensors by value, cut into chunks of equal size that its workgroups deal
// among themselves; every workgroup leaves one partial result.  Squares are summed in fp64: the square of any
// fp32 or bf16 value is finite there, and a thread's two fp64 operations per element (at the rate of fp32
// ones per lane) stay far below what HBM delivers.  Whoever needs the norm adds the partial results up
// itself, in the same order everywhere, so that no launch stands between the two sweeps.
#pragma once
#include "flce_device.h"
#include "rowvec.h"

namespace flce {

constexpr int GN_TENSORS = 120;   // a launch's arguments stay below 4 KB
constexpr int GN_THREADS = 256;
constexpr int GN_UNROLL = 8;      // 16-byte loads a thread has in flight
constexpr float GN_EPS = 1e-6f;

struct GnArgs {
    const void* in[GN_TENSORS];
    void* out[GN_TENSORS];
    int64_t count[GN_TENSORS];        // elements; bf16 tensors: ~elements
    int first_chunk[GN_TENSORS + 1];  // tensor t has chunks first_chunk[t] .. first_chunk[t + 1] - 1
    int tensors;
    int chunk_bytes;
    double* partial;                  // sweep 1: this launch's; sweep 2: all `partials` of them, from the first launch's on
    int partials;
    const float* norm_in;             // sweep 2: the norm is given
    float* norm_out;                  // sweep 2: workgroup 0 stores the norm, or null
    float max_norm;
    int inf_norm;
};

struct GnMax {
    static __device__ __forceinline__ double join(double a, double b) { return (b > a || b != b) ? b : a; }   // NaN stays
    static __device__ __forceinline__ double push(double a, float v) { return join(a, (double)fabsf(v)); }
    static __device__ __forceinline__ double norm(double a) { return a; }
};
struct GnSumSq {
    static __device__ __forceinline__ double join(double a, double b) { return a + b; }
    static __device__ __forceinline__ double push(double a, float v) { return fma((double)v, (double)v, a); }
    static __device__ __forceinline__ double norm(double a) { return sqrt(a); }
};

// Joined over a workgroup of GN_THREADS, the same value in every thread.
template <typename Op>
__device__ __forceinline__ double gn_block_join(double v, double* red) {
#pragma unroll
    for (int o = WAVE / 2; o > 0; o >>= 1) v = Op::join(v, __shfl_xor(v, o, WAVE));
    __syncthreads();
    if ((threadIdx.x & (WAVE - 1)) == 0) red[threadIdx.x / WAVE] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int w = 1; w < GN_THREADS / WAVE; ++w) v = Op::join(v, red[w]);
    return v;
}

// The tensor a chunk belongs to.
__device__ __forceinline__ int gn_tensor_of(const GnArgs& a, int chunk) {
    int lo = 0, hi = a.tensors;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.first_chunk[mid] <= chunk) lo = mid; else hi = mid;
    }
    return lo;
}

template <typename T, typename Op>
__device__ __forceinline__ double gn_sweep(const T* p, int64_t n, double acc) {
    constexpr int N = RowVec<T>::N;
    const int64_t nvec = n / N;
    int64_t v = threadIdx.x;
    auto take = [&](const u32x4& raw) {
        float f[N];
        RowVec<T>::unpack(raw, f);
#pragma unroll
        for (int e = 0; e < N; ++e) acc = Op::push(acc, f[e]);
    };
    for (; v + (GN_UNROLL - 1) * GN_THREADS < nvec; v += GN_UNROLL * GN_THREADS) {
        u32x4 raw[GN_UNROLL];
#pragma unroll
        for (int k = 0; k < GN_UNROLL; ++k) __builtin_memcpy(&raw[k], p + (v + k * GN_THREADS) * N, 16);
#pragma unroll
        for (int k = 0; k < GN_UNROLL; ++k) take(raw[k]);
    }
    for (; v < nvec; v += GN_THREADS) {
        u32x4 raw;
        __builtin_memcpy(&raw, p + v * N, 16);
        take(raw);
    }
    const int64_t j = nvec * N + threadIdx.x;
    if (j < n) acc = Op::push(acc, to_f32(p[j]));
    return acc;
}

template <typename Op>
__global__ __launch_bounds__(GN_THREADS) void grad_norm_kernel(GnArgs a) {
    __shared__ double red[GN_THREADS / WAVE];
    double acc = 0.0;
    for (int c = blockIdx.x; c < a.first_chunk[a.tensors]; c += gridDim.x) {
        const int t = gn_tensor_of(a, c);
        const bool is_bf16 = a.count[t] < 0;
        const int64_t n = is_bf16 ? ~a.count[t] : a.count[t];
        const int64_t per = a.chunk_bytes / (is_bf16 ? 2 : 4), at = (int64_t)(c - a.first_chunk[t]) * per;
        const int64_t len = min(per, n - at);
        acc = is_bf16 ? gn_sweep<bf16_t, Op>(static_cast<const bf16_t*>(a.in[t]) + at, len, acc)
                      : gn_sweep<float, Op>(static_cast<const float*>(a.in[t]) + at, len, acc);
    }
    acc = gn_block_join<Op>(acc, red);
    if (threadIdx.x == 0) a.partial[blockIdx.x] = acc;
}

template <typename Op>
__device__ __forceinline__ float gn_total(const double* partial, int partials, double* red) {
    double v = 0.0;
    for (int i = threadIdx.x; i < partials; i += GN_THREADS) v = Op::join(v, partial[i]);
    return (float)Op::norm(gn_block_join<Op>(v, red));
}
template <typename Op>
__global__ __launch_bounds__(GN_THREADS) void grad_norm_final_kernel(const double* partial, int partials, float* norm) {
    __shared__ double red[GN_THREADS / WAVE];
    const float v = gn_total<Op>(partial, partials, red);
    if (threadIdx.x == 0) *norm = v;
}

__device__ __forceinline__ float gn_factor(float norm, float max_norm) {
    if (!(norm - norm == 0.f)) return 1.0f;   // infinite or NaN
    const double c = (double)max_norm / ((double)norm + (double)GN_EPS);
    return c < 1.0 ? (float)c : 1.0f;
}

template <typename T>
__device__ __forceinline__ void gn_scale(const T* in, T* out, int64_t n, float c) {
    constexpr int N = RowVec<T>::N;
    const int64_t nvec = n / N;
    int64_t v = threadIdx.x;
    auto scaled = [&](const u32x4& raw) {
        float f[N];
        RowVec<T>::unpack(raw, f);
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] *= c;
        return RowVec<T>::pack(f);
    };
    for (; v + (GN_UNROLL - 1) * GN_THREADS < nvec; v += GN_UNROLL * GN_THREADS) {
        u32x4 raw[GN_UNROLL];
#pragma unroll
        for (int k = 0; k < GN_UNROLL; ++k) __builtin_memcpy(&raw[k], in + (v + k * GN_THREADS) * N, 16);
#pragma unroll
        for (int k = 0; k < GN_UNROLL; ++k) {
            const u32x4 r = scaled(raw[k]);
            __builtin_memcpy(out + (v + k * GN_THREADS) * N, &r, 16);
        }
    }
    for (; v < nvec; v += GN_THREADS) {
        u32x4 raw;
        __builtin_memcpy(&raw, in + v * N, 16);
        raw = scaled(raw);
        __builtin_memcpy(out + v * N, &raw, 16);
    }
    const int64_t j = nvec * N + threadIdx.x;
    if (j < n) out[j] = from_f32<T>(to_f32(in[j]) * c);
}

// Sweep 2 goes backwards: what sweep 1 read last is still in the memory-side cache.
template <typename Op>
__global__ __launch_bounds__(GN_THREADS) void grad_scale_kernel(GnArgs a) {
    __shared__ double red[GN_THREADS / WAVE];
    const float norm = a.norm_in ? *a.norm_in : gn_total<Op>(a.partial, a.partials, red);
    if (a.norm_out && blockIdx.x == 0 && threadIdx.x == 0) *a.norm_out = norm;
    const float f = gn_factor(norm, a.max_norm);
    const int chunks = a.first_chunk[a.tensors];
    for (int k = blockIdx.x; k < chunks; k += gridDim.x) {
        const int c = chunks - 1 - k, t = gn_tensor_of(a, c);
        if (f == 1.0f && a.in[t] == a.out[t]) continue;   // (in place: nothing to do)
        const bool is_bf16 = a.count[t] < 0;
        const int64_t n = is_bf16 ? ~a.count[t] : a.count[t];
        const int64_t per = a.chunk_bytes / (is_bf16 ? 2 : 4), at = (int64_t)(c - a.first_chunk[t]) * per;
        const int64_t len = min(per, n - at);
        if (is_bf16) gn_scale<bf16_t>(static_cast<const bf16_t*>(a.in[t]) + at, static_cast<bf16_t*>(a.out[t]) + at, len, f);
        else gn_scale<float>(static_cast<const float*>(a.in[t]) + at, static_cast<float*>(a.out[t]) + at, len, f);
    }
}

}  // namespace flce
