// Norms before and after a block, fused with the block's gate and the residual sum (paper section 3.2,
// RMSNorm paragraph, Eq. RMSNorm-forward / RMSNorm-backward, applied to the row that is being summed).
// Row i of the forward, in fp32 on values widened from the storage type:
//
//     z = y            or, with a norm after the block,   z = y q gamma_post,   q = 1 / sqrt(mean y^2 + eps)
//     h = x + s a(g) z                                    n = h r gamma_pre,    r = 1 / sqrt(mean h^2 + eps)
//
// and of the backward, from the stored h and y (r and q are computed again, in the sums that are taken
// anyway, so nothing but the rows themselves is kept between the two):
//
//     u = dn gamma_pre,   D = dh + r (u - h r mean(u h r))     dx = D         dgamma_pre  = sum_i dn h r
//     dz = s a(g) D       dg = sum over its rows s a'(g) z D
//     v = dz gamma_post   dy = q (v - y q mean(v y q))                        dgamma_post = sum_i dz y q
//
// A row belongs to a group of TPR threads that holds it in registers (NV vectors of 16 bytes per thread and
// stream), so every stream is read once and written once; sums over a row go through the lanes and, for
// groups of several wavefronts, through LDS.  Rows may start at any element: 16-byte accesses need no
// alignment, and the last, partial vector of a row goes element by element.  Rows that are too long for that
// (`*_long`) are swept several times by a workgroup of 1024 threads.
#pragma once
#include "flce_device.h"
#include "rowvec.h"

namespace flce {

enum { BN_ACT_LINEAR = 0, BN_ACT_SIGMOID = 1, BN_ACT_SILU = 2, BN_ACT_TANH = 3 };
enum { BN_GATE_NONE = 0, BN_GATE_SUM = 1, BN_GATE_ROW = 2 };   // ROW: every row has a gate row of its own

constexpr int BN_LONG_THREADS = 1024;

struct BnArgs {
    const void *x, *y, *gate, *gpost, *gpre;   // forward; the backward has no x
    const void *h, *dn, *dh;                   // backward
    void *out_h, *out_n;                       // forward
    void *dx, *dy, *dgate;                     // backward; the gradients of the gammas and shared gates:
    float *part_pre, *part_post, *part_gate;   // fp32 sums, a row per workgroup (gate: per segment), or null
    int64_t ldx, ldy, ldgate, ldh, ldn, lddh, lddn, lddx, lddy, lddgate;
    int rows, H;
    int per;         // rows per gate row
    int act;
    float scale, eps;
    // The backward walks segments: segment s is part s % parts of the `per` rows of gate row s / parts.
    int segments, parts;
    int by_row;        // every row has a gate row of its own (per counts all rows then)
    int gate_direct;   // a segment is all rows of its gate row: dgate is written at once
};

template <typename T>
__device__ __forceinline__ u32x4 bn_load(const T* row, int v, int nfull, int rem) {
    constexpr int N = RowVec<T>::N;
    u32x4 r = {0u, 0u, 0u, 0u};
    if (v < nfull) {
        __builtin_memcpy(&r, row + (int64_t)v * N, 16);
    } else if (v == nfull && rem) {
        const T* p = row + (int64_t)v * N;
        float f[N];
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = e < rem ? to_f32(p[e]) : 0.f;
        r = RowVec<T>::pack(f);
    }
    return r;
}
template <typename T>
__device__ __forceinline__ void bn_store(T* row, int v, int nfull, int rem, const float (&f)[RowVec<T>::N]) {
    constexpr int N = RowVec<T>::N;
    if (v < nfull) {
        const u32x4 r = RowVec<T>::pack(f);
        __builtin_memcpy(row + (int64_t)v * N, &r, 16);
    } else if (v == nfull && rem) {
        T* p = row + (int64_t)v * N;
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < rem) p[e] = from_f32<T>(f[e]);
    }
}
__device__ __forceinline__ void bn_store_f32(float* row, int64_t j, int n, const float* f, int count) {
#pragma unroll
    for (int e = 0; e < count; ++e)
        if (j + e < n) row[j + e] = f[e];
}

// a(g) and a'(g).  exp is taken of -|g| only, and 1 - sigmoid and the derivatives come as products of what
// does not cancel, so that they keep their relative accuracy where a gate saturates.
__device__ __forceinline__ float bn_act(int act, float g) {
    if (act == BN_ACT_LINEAR) return g;
    if (act == BN_ACT_TANH) return tanhf(g);
    const float e = expf(-fabsf(g)), d = 1.0f / (1.0f + e);
    const float sig = g >= 0.f ? d : e * d;
    return act == BN_ACT_SIGMOID ? sig : g * sig;
}
__device__ __forceinline__ float bn_act_grad(int act, float g) {
    if (act == BN_ACT_LINEAR) return 1.0f;
    if (act == BN_ACT_TANH) {
        const float e = expf(-2.0f * fabsf(g)), d = 1.0f / (1.0f + e);
        return 4.0f * e * d * d;
    }
    const float e = expf(-fabsf(g)), d = 1.0f / (1.0f + e);
    const float sig = g >= 0.f ? d : e * d, rest = g >= 0.f ? e * d : d;
    return act == BN_ACT_SIGMOID ? sig * rest : sig * (1.0f + g * rest);
}

// Sum over the TPR threads of a row's group, the same value in every one of them.  slot: LDS of this sum
// alone (a group of several wavefronts is a whole workgroup), read until the workgroup's next barrier.
template <int TPR>
__device__ __forceinline__ float bn_sum(float v, float* slot) {
#pragma unroll
    for (int o = (TPR < WAVE ? TPR : WAVE) / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, WAVE);
    if constexpr (TPR > WAVE) {
        if ((threadIdx.x & (WAVE - 1)) == 0) slot[threadIdx.x % TPR / WAVE] = v;
        __syncthreads();
        v = slot[0];
#pragma unroll
        for (int w = 1; w < TPR / WAVE; ++w) v += slot[w];
    }
    return v;
}

// Forward: a workgroup holds BLOCK / TPR rows.
template <typename T, int TPR, int NV, bool POST, bool GATE>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void block_norm_fwd_kernel(BnArgs a) {
    constexpr int N = RowVec<T>::N, GROUPS = TPR < 256 ? 256 / TPR : 1;
    __shared__ float red[2][GROUPS][TPR > WAVE ? TPR / WAVE : 1];
    const int grp = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * GROUPS + grp;
    const bool live = row < a.rows;   // (a group past the last row takes part in the barriers)
    const int nfull = live ? a.H / N : 0, rem = live ? a.H % N : 0;
    const int64_t at = live ? row : 0;
    u32x4 xv[NV], yv[NV], gv[NV], pv[NV], nv[NV];
    if (a.x) {
        const T* p = static_cast<const T*>(a.x) + at * a.ldx;
#pragma unroll
        for (int k = 0; k < NV; ++k) xv[k] = bn_load(p, t + k * TPR, nfull, rem);
    }
    if (a.y) {
        const T* p = static_cast<const T*>(a.y) + at * a.ldy;
#pragma unroll
        for (int k = 0; k < NV; ++k) yv[k] = bn_load(p, t + k * TPR, nfull, rem);
    }
    if constexpr (GATE) {
        const T* p = static_cast<const T*>(a.gate) + (int64_t)((uint32_t)at / (uint32_t)a.per) * a.ldgate;
#pragma unroll
        for (int k = 0; k < NV; ++k) gv[k] = bn_load(p, t + k * TPR, nfull, rem);
    }
    if constexpr (POST) {
#pragma unroll
        for (int k = 0; k < NV; ++k) pv[k] = bn_load(static_cast<const T*>(a.gpost), t + k * TPR, nfull, rem);
    }
    if (a.gpre) {
#pragma unroll
        for (int k = 0; k < NV; ++k) nv[k] = bn_load(static_cast<const T*>(a.gpre), t + k * TPR, nfull, rem);
    }
    float f[NV][N];
    if (a.y) {
        float q = 1.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k) RowVec<T>::unpack(yv[k], f[k]);
        if constexpr (POST) {
            float ss = 0.f;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < N; ++e) ss += f[k][e] * f[k][e];
            ss = bn_sum<TPR>(ss, red[0][grp]);
            q = 1.0f / sqrtf(ss / (float)a.H + a.eps);
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float w[N], xx[N];
            if constexpr (POST) {
                RowVec<T>::unpack(pv[k], w);
#pragma unroll
                for (int e = 0; e < N; ++e) f[k][e] *= q * w[e];
            }
            if constexpr (GATE) {
                RowVec<T>::unpack(gv[k], w);
#pragma unroll
                for (int e = 0; e < N; ++e) f[k][e] *= bn_act(a.act, w[e]);
            }
            if (a.x) RowVec<T>::unpack(xv[k], xx);
#pragma unroll
            for (int e = 0; e < N; ++e) f[k][e] = a.x ? xx[e] + a.scale * f[k][e] : a.scale * f[k][e];
        }
        if (a.out_h) {
            T* p = static_cast<T*>(a.out_h) + at * a.ldh;
#pragma unroll
            for (int k = 0; k < NV; ++k) bn_store<T>(p, t + k * TPR, nfull, rem, f[k]);
        }
    } else {
#pragma unroll
        for (int k = 0; k < NV; ++k) RowVec<T>::unpack(xv[k], f[k]);
    }
    if (a.gpre) {
        float ss = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < N; ++e) ss += f[k][e] * f[k][e];
        ss = bn_sum<TPR>(ss, red[1][grp]);
        const float r = 1.0f / sqrtf(ss / (float)a.H + a.eps);
        T* p = static_cast<T*>(a.out_n) + at * a.ldn;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float w[N];
            RowVec<T>::unpack(nv[k], w);
#pragma unroll
            for (int e = 0; e < N; ++e) w[e] *= f[k][e] * r;
            bn_store<T>(p, t + k * TPR, nfull, rem, w);
        }
    }
}

// Sum over a workgroup of BN_LONG_THREADS; the barrier in front frees the LDS of the sum before.
__device__ __forceinline__ float bn_long_sum(float v, float* red) {
    __syncthreads();
    return bn_sum<BN_LONG_THREADS>(v, red);
}

// scale a(g) z of one vector of a row (z before the gate comes back too, for the backward).
template <typename T>
__device__ __forceinline__ void bn_long_z(const BnArgs& a, const T* y, const T* gate, float q, int v, int nfull,
                                          int rem, float (&z)[RowVec<T>::N], float (&out)[RowVec<T>::N]) {
    constexpr int N = RowVec<T>::N;
    float w[N];
    RowVec<T>::unpack(bn_load(y, v, nfull, rem), z);
    if (a.gpost) {
        RowVec<T>::unpack(bn_load(static_cast<const T*>(a.gpost), v, nfull, rem), w);
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] *= q * w[e];
    }
    if (gate) RowVec<T>::unpack(bn_load(gate, v, nfull, rem), w);
#pragma unroll
    for (int e = 0; e < N; ++e) out[e] = a.scale * (gate ? z[e] * bn_act(a.act, w[e]) : z[e]);
}

template <typename T>
__device__ __forceinline__ float bn_long_rstd(const T* row, int nvec, int nfull, int rem, const BnArgs& a, float* red) {
    constexpr int N = RowVec<T>::N;
    float ss = 0.f;
    for (int v = threadIdx.x; v < nvec; v += BN_LONG_THREADS) {
        float f[N];
        RowVec<T>::unpack(bn_load(row, v, nfull, rem), f);
#pragma unroll
        for (int e = 0; e < N; ++e) ss += f[e] * f[e];
    }
    return 1.0f / sqrtf(bn_long_sum(ss, red) / (float)a.H + a.eps);
}

// Rows beyond the register forms: one workgroup per row, swept up to three times; the last sweep alone writes,
// and a thread writes only where it has read, so that h may lie on x.
template <typename T>
__global__ __launch_bounds__(BN_LONG_THREADS) void block_norm_fwd_long(BnArgs a) {
    constexpr int N = RowVec<T>::N;
    __shared__ float red[BN_LONG_THREADS / WAVE];
    const int64_t row = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (row >= a.rows) return;
    const int nfull = a.H / N, rem = a.H % N, nvec = nfull + (rem ? 1 : 0);
    const T* x = a.x ? static_cast<const T*>(a.x) + row * a.ldx : nullptr;
    const T* y = a.y ? static_cast<const T*>(a.y) + row * a.ldy : nullptr;
    const T* gate = a.gate ? static_cast<const T*>(a.gate) + (int64_t)((uint32_t)row / (uint32_t)a.per) * a.ldgate : nullptr;
    const float q = y && a.gpost ? bn_long_rstd(y, nvec, nfull, rem, a, red) : 1.0f;
    auto sum_at = [&](int v, float (&f)[N]) {
        float z[N];
        if (y) bn_long_z<T>(a, y, gate, q, v, nfull, rem, z, f);
        if (x) {
            RowVec<T>::unpack(bn_load(x, v, nfull, rem), z);
#pragma unroll
            for (int e = 0; e < N; ++e) f[e] = y ? z[e] + f[e] : z[e];
        }
    };
    float r = 0.f;
    if (a.gpre) {
        float ss = 0.f;
        for (int v = threadIdx.x; v < nvec; v += BN_LONG_THREADS) {
            float f[N];
            sum_at(v, f);
#pragma unroll
            for (int e = 0; e < N; ++e) ss += f[e] * f[e];
        }
        r = 1.0f / sqrtf(bn_long_sum(ss, red) / (float)a.H + a.eps);
    }
    for (int v = threadIdx.x; v < nvec; v += BN_LONG_THREADS) {
        float f[N];
        sum_at(v, f);
        if (a.out_h) bn_store<T>(static_cast<T*>(a.out_h) + row * a.ldh, v, nfull, rem, f);
        if (a.gpre) {
            float w[N];
            RowVec<T>::unpack(bn_load(static_cast<const T*>(a.gpre), v, nfull, rem), w);
#pragma unroll
            for (int e = 0; e < N; ++e) w[e] *= f[e] * r;
            bn_store<T>(static_cast<T*>(a.out_n) + row * a.ldn, v, nfull, rem, w);
        }
    }
}

// First and last row of a segment.
struct BnSegment {
    int g, row, end;
};
__device__ __forceinline__ BnSegment bn_segment(const BnArgs& a, int s) {
    const int g = s / a.parts, p = s - g * a.parts;
    const int64_t first = (int64_t)g * a.per;
    const int64_t len = min((int64_t)a.per, (int64_t)a.rows - first);
    return {g, (int)(first + len * p / a.parts), (int)(first + len * (p + 1) / a.parts)};
}

// Backward: workgroup b takes segments b, b + gridDim.x, ...; its GROUPS rows at a time.  The sums over rows
// stay in registers: the gammas' until the workgroup's last row, a shared gate's until its segment's; then the
// groups of a workgroup add theirs up in a fixed order.  Sums of several workgroups are left as rows of fp32
// partial sums for bn_sum_partials_kernel: no atomics, the order of additions depends on the shape alone.
template <typename T, int TPR, int NV, bool POST, int GATE>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void block_norm_bwd_kernel(BnArgs a) {
    constexpr int N = RowVec<T>::N, GROUPS = TPR < 256 ? 256 / TPR : 1, BLOCK = TPR * GROUPS;
    __shared__ float red[4][GROUPS][TPR > WAVE ? TPR / WAVE : 1];
    __shared__ float cols[GROUPS > 1 ? BLOCK * NV * N : 1];
    const int grp = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const int nfull_all = a.H / N, rem_all = a.H % N;
    u32x4 prev[NV], postv[NV], gv[NV];
    float acc_pre[NV][N], acc_post[NV][N], acc_gate[NV][N];
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < N; ++e) acc_pre[k][e] = acc_post[k][e] = acc_gate[k][e] = 0.f;
    if (a.gpre)
#pragma unroll
        for (int k = 0; k < NV; ++k) prev[k] = bn_load(static_cast<const T*>(a.gpre), t + k * TPR, nfull_all, rem_all);
    if constexpr (POST)
#pragma unroll
        for (int k = 0; k < NV; ++k) postv[k] = bn_load(static_cast<const T*>(a.gpost), t + k * TPR, nfull_all, rem_all);

    // The sum over the workgroup's groups of a row of sums, handed column by column to put(column, value).
    auto over_groups = [&](float (&acc)[NV][N], auto put) {
        if constexpr (GROUPS > 1) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < N; ++e) cols[grp * (TPR * NV * N) + (t + k * TPR) * N + e] = acc[k][e];
            __syncthreads();
            for (int j = threadIdx.x; j < TPR * NV * N && j < a.H; j += BLOCK) {
                float s = cols[j];
                for (int q = 1; q < GROUPS; ++q) s += cols[q * (TPR * NV * N) + j];
                put(j, s);
            }
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if ((t + k * TPR) * N + e < a.H) put((t + k * TPR) * N + e, acc[k][e]);
        }
    };

    for (int s = blockIdx.x; s < a.segments; s += gridDim.x) {
        const BnSegment seg = bn_segment(a, s);
        if constexpr (GATE == BN_GATE_SUM) {
            const T* p = static_cast<const T*>(a.gate) + (int64_t)seg.g * a.ldgate;
#pragma unroll
            for (int k = 0; k < NV; ++k) gv[k] = bn_load(p, t + k * TPR, nfull_all, rem_all);
        }
        for (int base = seg.row; base < seg.end; base += GROUPS) {
            const bool live = base + grp < seg.end;   // (a group past the last row takes part in the barriers)
            const int64_t row = live ? base + grp : base;
            const int nfull = live ? nfull_all : 0, rem = live ? rem_all : 0;
            u32x4 hv[NV], nv[NV], dv[NV], yv[NV];
            if (a.gpre) {
                const T *p = static_cast<const T*>(a.h) + row * a.ldh, *p2 = static_cast<const T*>(a.dn) + row * a.lddn;
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    hv[k] = bn_load(p, t + k * TPR, nfull, rem);
                    nv[k] = bn_load(p2, t + k * TPR, nfull, rem);
                }
            }
            if (a.dh) {
                const T* p = static_cast<const T*>(a.dh) + row * a.lddh;
#pragma unroll
                for (int k = 0; k < NV; ++k) dv[k] = bn_load(p, t + k * TPR, nfull, rem);
            }
            if (a.y) {
                const T* p = static_cast<const T*>(a.y) + row * a.ldy;
#pragma unroll
                for (int k = 0; k < NV; ++k) yv[k] = bn_load(p, t + k * TPR, nfull, rem);
            }
            if constexpr (GATE == BN_GATE_ROW) {
                const T* p = static_cast<const T*>(a.gate) + row * a.ldgate;
#pragma unroll
                for (int k = 0; k < NV; ++k) gv[k] = bn_load(p, t + k * TPR, nfull, rem);
            }
            // D, the gradient of h
            float D[NV][N];
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                if (a.dh) RowVec<T>::unpack(dv[k], D[k]);
                else
#pragma unroll
                    for (int e = 0; e < N; ++e) D[k][e] = 0.f;
            }
            if (a.gpre) {
                float hh = 0.f, uh = 0.f;
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    float h[N], u[N], w[N];
                    RowVec<T>::unpack(hv[k], h);
                    RowVec<T>::unpack(nv[k], u);
                    RowVec<T>::unpack(prev[k], w);
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        hh += h[e] * h[e];
                        uh += u[e] * w[e] * h[e];
                    }
                }
                hh = bn_sum<TPR>(hh, red[0][grp]);
                uh = bn_sum<TPR>(uh, red[1][grp]);
                const float r = 1.0f / sqrtf(hh / (float)a.H + a.eps), c = uh * r / (float)a.H;
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    float h[N], u[N], w[N];
                    RowVec<T>::unpack(hv[k], h);
                    RowVec<T>::unpack(nv[k], u);
                    RowVec<T>::unpack(prev[k], w);
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const float xh = h[e] * r;
                        D[k][e] += r * (u[e] * w[e] - xh * c);
                        acc_pre[k][e] += u[e] * xh;
                    }
                }
            }
            if (a.dx) {
                T* p = static_cast<T*>(a.dx) + row * a.lddx;
#pragma unroll
                for (int k = 0; k < NV; ++k) bn_store<T>(p, t + k * TPR, nfull, rem, D[k]);
            }
            if (a.y) {
                float q = 1.0f;
                if constexpr (POST) {
                    float yy = 0.f;
#pragma unroll
                    for (int k = 0; k < NV; ++k) {
                        float y[N];
                        RowVec<T>::unpack(yv[k], y);
#pragma unroll
                        for (int e = 0; e < N; ++e) yy += y[e] * y[e];
                    }
                    yy = bn_sum<TPR>(yy, red[2][grp]);
                    q = 1.0f / sqrtf(yy / (float)a.H + a.eps);
                }
                // D becomes dz, then (with a norm after the block) v = dz gamma_post
                float vy = 0.f, dg[NV][N];
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    float y[N], w[N], g[N];
                    RowVec<T>::unpack(yv[k], y);
                    if constexpr (POST) RowVec<T>::unpack(postv[k], w);
                    if constexpr (GATE != BN_GATE_NONE) RowVec<T>::unpack(gv[k], g);
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        D[k][e] *= a.scale;
                        const float yh = POST ? y[e] * q : y[e];
                        if constexpr (GATE != BN_GATE_NONE) {
                            const float z = POST ? yh * w[e] : yh;
                            dg[k][e] = D[k][e] * z * bn_act_grad(a.act, g[e]);
                            if constexpr (GATE == BN_GATE_SUM) acc_gate[k][e] += dg[k][e];
                            D[k][e] *= bn_act(a.act, g[e]);
                        }
                        if constexpr (POST) {
                            acc_post[k][e] += D[k][e] * yh;
                            D[k][e] *= w[e];
                            vy += D[k][e] * yh;
                        }
                    }
                }
                if constexpr (GATE == BN_GATE_ROW) {
                    if (a.dgate) {
                        T* p = static_cast<T*>(a.dgate) + row * a.lddgate;
#pragma unroll
                        for (int k = 0; k < NV; ++k) bn_store<T>(p, t + k * TPR, nfull, rem, dg[k]);
                    }
                }
                if constexpr (POST) {
                    const float c = bn_sum<TPR>(vy, red[3][grp]) / (float)a.H;
#pragma unroll
                    for (int k = 0; k < NV; ++k) {
                        float y[N];
                        RowVec<T>::unpack(yv[k], y);
#pragma unroll
                        for (int e = 0; e < N; ++e) D[k][e] = q * (D[k][e] - y[e] * q * c);
                    }
                }
                if (a.dy) {
                    T* p = static_cast<T*>(a.dy) + row * a.lddy;
#pragma unroll
                    for (int k = 0; k < NV; ++k) bn_store<T>(p, t + k * TPR, nfull, rem, D[k]);
                }
            }
            if constexpr (TPR > WAVE) __syncthreads();   // the next row's sums reuse the LDS
        }
        if constexpr (GATE == BN_GATE_SUM) {
            if (a.gate_direct) {
                T* p = static_cast<T*>(a.dgate) + (int64_t)seg.g * a.lddgate;
                if (a.dgate) over_groups(acc_gate, [&](int j, float v) { p[j] = from_f32<T>(v); });
            } else if (a.part_gate) {
                float* p = a.part_gate + (int64_t)s * a.H;
                over_groups(acc_gate, [&](int j, float v) { p[j] = v; });
            }
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < N; ++e) acc_gate[k][e] = 0.f;
        }
    }
    if (a.part_pre) {
        float* p = a.part_pre + (int64_t)blockIdx.x * a.H;
        over_groups(acc_pre, [&](int j, float v) { p[j] = v; });
    }
    if constexpr (POST) {
        if (a.part_post) {
            float* p = a.part_post + (int64_t)blockIdx.x * a.H;
            over_groups(acc_post, [&](int j, float v) { p[j] = v; });
        }
    }
}

// Rows beyond the register forms (see block_norm_fwd_long).  The sums over rows live in the partial sums'
// memory (a gate's: a row per workgroup, or per segment where several share a gate row); a column always
// belongs to the same thread.
template <typename T>
__global__ __launch_bounds__(BN_LONG_THREADS) void block_norm_bwd_long(BnArgs a) {
    constexpr int N = RowVec<T>::N;
    __shared__ float red[BN_LONG_THREADS / WAVE];
    const int nfull = a.H / N, rem = a.H % N, nvec = nfull + (rem ? 1 : 0);
    const T* gpre = static_cast<const T*>(a.gpre);
    const T* gpost = static_cast<const T*>(a.gpost);
    float* pre = a.part_pre ? a.part_pre + (int64_t)blockIdx.x * a.H : nullptr;
    float* post = a.part_post ? a.part_post + (int64_t)blockIdx.x * a.H : nullptr;
    auto each = [&](float* p, auto what) {   // the columns of this thread
        for (int v = threadIdx.x; v < nvec; v += BN_LONG_THREADS)
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (v * N + e < a.H) what(p, v * N + e);
    };
    if (pre) each(pre, [](float* p, int j) { p[j] = 0.f; });
    if (post) each(post, [](float* p, int j) { p[j] = 0.f; });
    for (int s = blockIdx.x; s < a.segments; s += gridDim.x) {
        const BnSegment seg = bn_segment(a, s);
        float* gsum = a.part_gate ? a.part_gate + (int64_t)(a.gate_direct ? blockIdx.x : s) * a.H : nullptr;
        if (gsum) each(gsum, [](float* p, int j) { p[j] = 0.f; });
        for (int64_t row = seg.row; row < seg.end; ++row) {
            const T* h = gpre ? static_cast<const T*>(a.h) + row * a.ldh : nullptr;
            const T* dn = gpre ? static_cast<const T*>(a.dn) + row * a.lddn : nullptr;
            const T* dh = a.dh ? static_cast<const T*>(a.dh) + row * a.lddh : nullptr;
            const T* y = a.y ? static_cast<const T*>(a.y) + row * a.ldy : nullptr;
            const T* gate = a.gate ? static_cast<const T*>(a.gate) + (a.by_row ? row : (int64_t)seg.g) * a.ldgate : nullptr;
            float r = 0.f, c = 0.f, q = 1.0f, cy = 0.f;
            if (h) {
                float hh = 0.f, uh = 0.f;
                for (int v = threadIdx.x; v < nvec; v += BN_LONG_THREADS) {
                    float hf[N], u[N], w[N];
                    RowVec<T>::unpack(bn_load(h, v, nfull, rem), hf);
                    RowVec<T>::unpack(bn_load(dn, v, nfull, rem), u);
                    RowVec<T>::unpack(bn_load(gpre, v, nfull, rem), w);
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        hh += hf[e] * hf[e];
                        uh += u[e] * w[e] * hf[e];
                    }
                }
                hh = bn_long_sum(hh, red);
                uh = bn_long_sum(uh, red);
                r = 1.0f / sqrtf(hh / (float)a.H + a.eps);
                c = uh * r / (float)a.H;
            }
            if (y && gpost) q = bn_long_rstd(y, nvec, nfull, rem, a, red);
            auto grad_h = [&](int v, float (&D)[N]) {
#pragma unroll
                for (int e = 0; e < N; ++e) D[e] = 0.f;
                if (dh) RowVec<T>::unpack(bn_load(dh, v, nfull, rem), D);
                if (h) {
                    float hf[N], u[N], w[N];
                    RowVec<T>::unpack(bn_load(h, v, nfull, rem), hf);
                    RowVec<T>::unpack(bn_load(dn, v, nfull, rem), u);
                    RowVec<T>::unpack(bn_load(gpre, v, nfull, rem), w);
#pragma unroll
                    for (int e = 0; e < N; ++e) D[e] += r * (u[e] * w[e] - hf[e] * r * c);
                }
            };
            auto grad_z = [&](int v, const float (&D)[N], float (&dz)[N]) {
                float g[N];
                if (gate) RowVec<T>::unpack(bn_load(gate, v, nfull, rem), g);
#pragma unroll
                for (int e = 0; e < N; ++e) dz[e] = a.scale * D[e] * (gate ? bn_act(a.act, g[e]) : 1.0f);
            };
            if (y && gpost) {
                float vy = 0.f;
                for (int v = threadIdx.x; v < nvec; v += BN_LONG_THREADS) {
                    float D[N], dz[N], yf[N], w[N];
                    grad_h(v, D);
                    grad_z(v, D, dz);
                    RowVec<T>::unpack(bn_load(y, v, nfull, rem), yf);
                    RowVec<T>::unpack(bn_load(gpost, v, nfull, rem), w);
#pragma unroll
                    for (int e = 0; e < N; ++e) vy += dz[e] * w[e] * yf[e] * q;
                }
                cy = bn_long_sum(vy, red) / (float)a.H;
            }
            for (int v = threadIdx.x; v < nvec; v += BN_LONG_THREADS) {
                float D[N];
                grad_h(v, D);
                if (pre) {
                    float hf[N], u[N];
                    RowVec<T>::unpack(bn_load(h, v, nfull, rem), hf);
                    RowVec<T>::unpack(bn_load(dn, v, nfull, rem), u);
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        if (v * N + e < a.H) pre[v * N + e] += u[e] * (hf[e] * r);
                }
                if (y) {
                    float dz[N], yf[N], w[N], g[N], dg[N];
                    grad_z(v, D, dz);
                    RowVec<T>::unpack(bn_load(y, v, nfull, rem), yf);
                    if (gpost) RowVec<T>::unpack(bn_load(gpost, v, nfull, rem), w);
                    if (gate) {
                        RowVec<T>::unpack(bn_load(gate, v, nfull, rem), g);
#pragma unroll
                        for (int e = 0; e < N; ++e) {
                            const float z = gpost ? yf[e] * q * w[e] : yf[e];
                            dg[e] = a.scale * D[e] * z * bn_act_grad(a.act, g[e]);
                            if (gsum && v * N + e < a.H) gsum[v * N + e] += dg[e];
                        }
                        if (a.by_row && a.dgate)
                            bn_store<T>(static_cast<T*>(a.dgate) + row * a.lddgate, v, nfull, rem, dg);
                    }
                    if (gpost) {
#pragma unroll
                        for (int e = 0; e < N; ++e) {
                            const float yh = yf[e] * q;
                            if (post && v * N + e < a.H) post[v * N + e] += dz[e] * yh;
                            dz[e] = q * (dz[e] * w[e] - yh * cy);
                        }
                    }
                    if (a.dy) bn_store<T>(static_cast<T*>(a.dy) + row * a.lddy, v, nfull, rem, dz);
                }
                if (a.dx) bn_store<T>(static_cast<T*>(a.dx) + row * a.lddx, v, nfull, rem, D);
            }
        }
        if (gsum && a.gate_direct) {
            T* out = static_cast<T*>(a.dgate) + (int64_t)seg.g * a.lddgate;
            each(gsum, [&](float* p, int j) { out[j] = from_f32<T>(p[j]); });
        }
    }
}

// out[g][j] = sum over p of rows [g * parts + p][j] of fp32 partial sums, for up to three sets of them: the two
// gammas (one output row each) and the gate.  As in rmsnorm_dgamma_kernel a workgroup owns 64 columns of an
// output row, thread (c, q) adds rows q, q + 16, ... of column c, then the 16 sums are added in order.
struct BnSums {
    const float* part[3];
    void* out[3];
    int64_t ld[3];
    int parts[3];
    int first[4];   // the sets' output rows are rows first[i] .. first[i + 1] of the grid
};
constexpr int BN_SUM_COLS = 64, BN_SUM_PARTS = 16;
template <typename T>
__global__ __launch_bounds__(BN_SUM_COLS * BN_SUM_PARTS) void bn_sum_partials_kernel(BnSums b, int n) {
    __shared__ float sums[BN_SUM_PARTS][BN_SUM_COLS];
    const int c = threadIdx.x % BN_SUM_COLS, q = threadIdx.x / BN_SUM_COLS;
    const int r = blockIdx.y, j = blockIdx.x * BN_SUM_COLS + c;
    const int set = r >= b.first[2] ? 2 : r >= b.first[1] ? 1 : 0;
    const int g = r - b.first[set], parts = b.parts[set];
    const float* from = b.part[set] + (int64_t)g * parts * n + j;
    float s = 0.f;
    if (j < n)
#pragma unroll 8
        for (int p = q; p < parts; p += BN_SUM_PARTS) s += from[(int64_t)p * n];
    sums[q][c] = s;
    __syncthreads();
    if (q == 0 && j < n) {
        for (int k = 1; k < BN_SUM_PARTS; ++k) s += sums[k][c];
        (static_cast<T*>(b.out[set]) + (int64_t)g * b.ld[set])[j] = from_f32<T>(s);
    }
}

}  // namespace flce
