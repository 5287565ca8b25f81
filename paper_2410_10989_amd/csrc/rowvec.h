// A 16-byte vector of a row and its elements as fp32 values.
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

}  // namespace flce
