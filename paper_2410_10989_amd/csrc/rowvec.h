// A 16-byte vector of a row and its elements as fp32 values; loads and stores of a row's vectors.
#pragma once
#include "flce_device.h"

namespace flce {

template <typename T> struct RowVec;
template <> struct RowVec<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void unpack(const u32x4& raw, float (&f)[4]) {
#pragma unroll
        for (int w = 0; w < 4; ++w) f[w] = __uint_as_float(raw[w]);
    }
    static __device__ __forceinline__ u32x4 pack(const float (&f)[4]) {
        u32x4 r;
#pragma unroll
        for (int w = 0; w < 4; ++w) r[w] = __float_as_uint(f[w]);
        return r;
    }
};
template <> struct RowVec<bf16_t> {
    static constexpr int N = 8;
    // a bf16 is the upper half of the float with the same value
    static __device__ __forceinline__ void unpack(const u32x4& raw, float (&f)[8]) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            f[2 * w] = __uint_as_float(raw[w] << 16);
            f[2 * w + 1] = __uint_as_float(raw[w] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ u32x4 pack(const float (&f)[8]) {
        u32x4 r;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const bf16x2 p = {(bf16_t)f[2 * w], (bf16_t)f[2 * w + 1]};   // round to nearest even
            r[w] = __builtin_bit_cast(uint32_t, p);
        }
        return r;
    }
};

typedef u32x4 __attribute__((aligned(2))) u32x4_any;   // at any element
typedef f32x4 __attribute__((aligned(4))) f32x4_any;

// Vector v of a row: whole for v < nfull; vector nfull has rem elements.
template <typename T>
__device__ __forceinline__ u32x4 row_load(const T* row, int v, int nfull, int rem) {
    constexpr int N = RowVec<T>::N;
    u32x4 r = {0u, 0u, 0u, 0u};
    if (v < nfull) {
        r = *reinterpret_cast<const u32x4_any*>(row + (int64_t)v * N);
    } else if (v == nfull && rem) {
        const T* p = row + (int64_t)v * N;
        float f[N];
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = e < rem ? to_f32(p[e]) : 0.f;
        r = RowVec<T>::pack(f);
    }
    return r;
}
template <typename T, bool NT>
__device__ __forceinline__ void row_store(T* row, int v, int nfull, int rem, const float (&f)[RowVec<T>::N]) {
    constexpr int N = RowVec<T>::N;
    if (v < nfull) {
        u32x4_any* p = reinterpret_cast<u32x4_any*>(row + (int64_t)v * N);
        if constexpr (NT) __builtin_nontemporal_store(RowVec<T>::pack(f), p);
        else *p = RowVec<T>::pack(f);
    } else if (v == nfull && rem) {
        T* p = row + (int64_t)v * N;
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < rem) p[e] = from_f32<T>(f[e]);
    }
}

// The same for loads that are issued a row ahead (H of at least one vector): putting a partial vector together
// waits for every load before it, so its place is taken by the 16 bytes that end with the row, and row_shift_tail
// moves its elements to the front when the row's turn comes (rows of 4095 bf16: 158 -> 109 us, 8192 of them).
template <typename T>
__device__ __forceinline__ u32x4 row_load_ahead(const T* row, int v, int nvec, int H) {
    constexpr int N = RowVec<T>::N;
    u32x4 r = {0u, 0u, 0u, 0u};
    if (v < nvec) r = *reinterpret_cast<const u32x4_any*>(row + min(v * N, H - N));
    return r;
}
template <typename T>
__device__ __forceinline__ void row_shift_tail(u32x4& r, int rem) {
    const int drop = (RowVec<T>::N - rem) * (int)sizeof(T), words = drop / 4, bits = drop % 4 * 8;
    const u32x4 from = r;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        auto word = [&](int i) { return i == 0 ? from[0] : i == 1 ? from[1] : i == 2 ? from[2] : i == 3 ? from[3] : 0u; };
        const uint32_t lo = word(w + words), hi = word(w + words + 1);
        r[w] = bits ? lo >> bits | hi << (32 - bits) : lo;
    }
}

}  // namespace flce
