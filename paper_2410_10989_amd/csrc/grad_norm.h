// Norm over all elements of many tensors, and scaling by it (gradient clipping):
//
//     norm = sqrt(sum_t sum_j g_tj^2)   or   max_t max_j |g_tj|
//     c    = min(1, max_norm / (norm + 1e-6)),  1 where norm is not finite;      out_tj = g_tj c
//
// A launch takes up to GN_TENSORS tensors by value, cut into chunks of equal size that its workgroups deal
// among themselves; every workgroup leaves one partial result, and they are added up in the same order everywhere.
// Squares are summed in fp64: the square of any fp32 or bf16 value is finite there, and two fp64 operations per
// element cost nothing beside HBM (a plain read of the same bytes takes as long).
// Bound by HBM.  1.05 GB of bf16: 157 us (6.7 TB/s) with nontemporal loads, 196 without (what is read then stays
// in the memory-side cache, where no later part of the sweep finds it); 338 fp32 gradients of 1.41 GB clipped into
// other buffers: 716 us for 4.2 GB moved (5.9 TB/s).  32 KB chunks: one round of eight loads per thread; 64 KB chunks
// 6 % slower.
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
    int streamed;                     // chunks 0 .. streamed - 1 go past the memory-side cache
    double* partial;                  // sweep 1: this launch's; sweep 2: all `partials` of them, from the first launch's on
    int partials;
    const float* norm_in;             // sweep 2: the norm is given
    float* norm_out;                  // sweep 2: workgroup 0 stores the norm, or null
    float max_norm;
    int in_place;                     // every out is its in
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

// Which tensor a chunk belongs to: every lane of a wavefront keeps the ends of two tensors, and as many of them lie
// at or below the chunk as tensors lie before it (one load per workgroup, where a search in the arguments is seven
// dependent ones per chunk: 300 short tensors 14.3 -> 13.2 us).
struct GnEnds {
    int lo, hi;
    __device__ __forceinline__ explicit GnEnds(const GnArgs& a) {
        const int lane = threadIdx.x & (WAVE - 1);
        lo = lane < a.tensors ? a.first_chunk[lane + 1] : INT32_MAX;
        hi = lane + WAVE < a.tensors ? a.first_chunk[lane + WAVE + 1] : INT32_MAX;
    }
    __device__ __forceinline__ int tensor(int chunk) const {
        return __popcll(__ballot(lo <= chunk)) + __popcll(__ballot(hi <= chunk));
    }
};
static_assert(GN_TENSORS <= 2 * WAVE, "");

typedef u32x4 __attribute__((aligned(2))) u32x4_any;   // at any element
template <bool NT>
__device__ __forceinline__ u32x4 gn_load(const void* p) {
    if constexpr (NT) return __builtin_nontemporal_load(static_cast<const u32x4_any*>(p));
    else return *static_cast<const u32x4_any*>(p);
}

template <typename T, typename Op, bool NT>
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
        for (int k = 0; k < GN_UNROLL; ++k) raw[k] = gn_load<NT>(p + (v + k * GN_THREADS) * N);
#pragma unroll
        for (int k = 0; k < GN_UNROLL; ++k) take(raw[k]);
    }
    for (; v < nvec; v += GN_THREADS) take(gn_load<NT>(p + v * N));
    const int64_t j = nvec * N + threadIdx.x;
    if (j < n) acc = Op::push(acc, to_f32(p[j]));
    return acc;
}

// Chunk c of a launch: its tensor's elements at .. at + len - 1.
struct GnChunk {
    int t;
    bool is_bf16;
    int64_t at, len;
};
__device__ __forceinline__ GnChunk gn_chunk(const GnArgs& a, const GnEnds& ends, int c) {
    const int t = ends.tensor(c);
    const bool is_bf16 = a.count[t] < 0;
    const int64_t n = is_bf16 ? ~a.count[t] : a.count[t];
    const int64_t per = a.chunk_bytes / (is_bf16 ? 2 : 4), at = (int64_t)(c - a.first_chunk[t]) * per;
    return {t, is_bf16, at, min(per, n - at)};
}
// A workgroup's share of a launch's elements, joined over its threads.
template <typename Op>
__device__ __forceinline__ double gn_share(const GnArgs& a, double* red) {
    const GnEnds ends(a);
    double acc = 0.0;
    for (int c = blockIdx.x; c < a.first_chunk[a.tensors]; c += gridDim.x) {
        const GnChunk k = gn_chunk(a, ends, c);
        const bool nt = c < a.streamed;
        if (k.is_bf16) {
            const bf16_t* p = static_cast<const bf16_t*>(a.in[k.t]) + k.at;
            acc = nt ? gn_sweep<bf16_t, Op, true>(p, k.len, acc) : gn_sweep<bf16_t, Op, false>(p, k.len, acc);
        } else {
            const float* p = static_cast<const float*>(a.in[k.t]) + k.at;
            acc = nt ? gn_sweep<float, Op, true>(p, k.len, acc) : gn_sweep<float, Op, false>(p, k.len, acc);
        }
    }
    return gn_block_join<Op>(acc, red);
}

template <typename Op>
__global__ __launch_bounds__(GN_THREADS) void grad_norm_kernel(GnArgs a) {
    __shared__ double red[GN_THREADS / WAVE];
    const double v = gn_share<Op>(a, red);
    if (threadIdx.x == 0) a.partial[blockIdx.x] = v;
}

template <typename Op>
__device__ __forceinline__ float gn_total(const double* partial, int partials, double* red) {
    double v = 0.0;
    for (int i0 = threadIdx.x; i0 < partials; i0 += 4 * GN_THREADS) {   // (four loads under way, not one)
        double p[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) p[k] = i0 + k * GN_THREADS < partials ? partial[i0 + k * GN_THREADS] : 0.0;
#pragma unroll
        for (int k = 0; k < 4; ++k) v = Op::join(v, p[k]);
    }
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

template <typename T, bool NT>
__device__ __forceinline__ void gn_scale(const T* in, T* out, int64_t n, float c) {
    constexpr int N = RowVec<T>::N;
    const int64_t nvec = n / N;
    int64_t v = threadIdx.x;
    auto store = [&](int64_t at, const u32x4& raw) {
        float f[N];
        RowVec<T>::unpack(raw, f);
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] *= c;
        u32x4_any* p = reinterpret_cast<u32x4_any*>(out + at * N);
        if constexpr (NT) __builtin_nontemporal_store(RowVec<T>::pack(f), p);
        else *p = RowVec<T>::pack(f);
    };
    for (; v + (GN_UNROLL - 1) * GN_THREADS < nvec; v += GN_UNROLL * GN_THREADS) {
        u32x4 raw[GN_UNROLL];
#pragma unroll
        for (int k = 0; k < GN_UNROLL; ++k) raw[k] = gn_load<NT>(in + (v + k * GN_THREADS) * N);
#pragma unroll
        for (int k = 0; k < GN_UNROLL; ++k) store(v + k * GN_THREADS, raw[k]);
    }
    for (; v < nvec; v += GN_THREADS) store(v, gn_load<NT>(in + v * N));
    const int64_t j = nvec * N + threadIdx.x;
    if (j < n) out[j] = from_f32<T>(to_f32(in[j]) * c);
}

// Sweep 2 goes backwards: what sweep 1 read last is still in the memory-side cache.
__device__ __forceinline__ void gn_scale_share(const GnArgs& a, float f) {
    if (f == 1.0f && a.in_place) return;
    const GnEnds ends(a);
    const int chunks = a.first_chunk[a.tensors];
    for (int i = blockIdx.x; i < chunks; i += gridDim.x) {
        const int c = chunks - 1 - i;
        const GnChunk k = gn_chunk(a, ends, c);
        if (f == 1.0f && a.in[k.t] == a.out[k.t]) continue;
        const bool nt = c < a.streamed;
        if (k.is_bf16) {
            const bf16_t* p = static_cast<const bf16_t*>(a.in[k.t]) + k.at;
            bf16_t* q = static_cast<bf16_t*>(a.out[k.t]) + k.at;
            if (nt) gn_scale<bf16_t, true>(p, q, k.len, f); else gn_scale<bf16_t, false>(p, q, k.len, f);
        } else {
            const float* p = static_cast<const float*>(a.in[k.t]) + k.at;
            float* q = static_cast<float*>(a.out[k.t]) + k.at;
            if (nt) gn_scale<float, true>(p, q, k.len, f); else gn_scale<float, false>(p, q, k.len, f);
        }
    }
}
template <typename Op>
__global__ __launch_bounds__(GN_THREADS) void grad_scale_kernel(GnArgs a) {
    __shared__ double red[GN_THREADS / WAVE];
    const float norm = a.norm_in ? *a.norm_in : gn_total<Op>(a.partial, a.partials, red);
    if (a.norm_out && blockIdx.x == 0 && threadIdx.x == 0) *a.norm_out = norm;
    gn_scale_share(a, gn_factor(norm, a.max_norm));
}

// Few elements: one workgroup for all of it.  scale: whether they are to be clipped too.
template <typename Op>
__global__ __launch_bounds__(GN_THREADS) void grad_small_kernel(GnArgs a, int scale) {
    __shared__ double red[GN_THREADS / WAVE];
    const float norm = (float)Op::norm(gn_share<Op>(a, red));
    if (threadIdx.x == 0) *a.norm_out = norm;
    if (scale) gn_scale_share(a, gn_factor(norm, a.max_norm));   // (behind the join's barrier: all has been read)
}

}  // namespace flce
