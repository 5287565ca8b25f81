// Layer norm with the residual sum in front of it.  Row i, in fp32 on values widened from the storage type:
//
//     h = x + y  (or x)      m = mean h,  d = h - m,  r = 1 / sqrt(mean d^2 + eps)      n = d r gamma + beta
//
// and backward, from the stored h alone (m and r are computed again):
//
//     u = dn gamma      dx = dh + r (u - mean u - d r mean(u d r))      dgamma = sum_i dn d r      dbeta = sum_i dn
//
// The mean is taken first and the squares are those of h - mean: their sum does not cancel, however far a row lies from
// zero.  The mean's own rounding (up to 2^-19 of |h|, which r may multiply by eps^-1/2: fp32 rows of a thousand equal elements,
// 10 to 1000 large, had n off by up to 0.19 gamma) is the mean of h - mean, whose sum is taken with the squares':
//
//     p = fl(mean h),  q = mean (h - p),     d = (h - p) - q,  mean d^2 = mean (h - p)^2 - q^2
//
// with q far below |h|, so that what rounds it off is 2^-38 of |h|.  (The backward's rows of up to 16384 bf16 elements add up
// to their sum itself, as far as that matters beside their deviation: elements of 8 bits that are alike have sums of
// at most 22, and what is cut off of others is 2^-24 of a sum that their deviation is not far below.  There q is the
// quotient's remainder.)  A row lies in the registers of a group of TPR threads
// (see block_norm.h), so the second pass over it reads nothing; what it costs is a second exchange between the threads,
// in which the backward takes its other sums along.
//
// Bound by HBM.  Forward, 16384 x 3584 bf16 with a residual: 80 us, 5.9 TB/s.  Backward, 8192 x 4096 bf16 with a residual: 53
// to 55 us, 4.9 TB/s (a workgroup has one row on the way while it does another, whose two exchanges it waits for), and 5
// for the sums over rows.
#pragma once
#include "rowsums.h"
#include "rowvec.h"

namespace flce {

struct LnArgs {
    const void *x, *y, *gamma, *beta;      // forward
    void *out_h, *out_n;
    const void *h, *dn, *dh;               // backward
    void* dx;
    float *part_gamma, *part_beta;         // fp32 sums, a row per workgroup, or null
    void *dgamma, *dbeta;                  // one workgroup has all rows: written at once
    int64_t ldx, ldy, ldh, ldn, lddx, lddh, lddn;
    int rows, H;
    float eps;
};

constexpr int LN_LONG_THREADS = 1024;

// Elements of vector v that belong to the row.
template <typename T>
__device__ __forceinline__ int ln_live(int v, int nfull, int rem) {
    return v < nfull ? RowVec<T>::N : v == nfull ? rem : 0;
}

// The same value in a scalar register, where a row's threads are whole wavefronts.
template <int TPR>
__device__ __forceinline__ float ln_uniform(float v) {
    if constexpr (TPR < WAVE) return v;
    return __uint_as_float((uint32_t)__builtin_amdgcn_readfirstlane((int)__float_as_uint(v)));
}

// mean d^2 from the sums of (h - p)^2 and of h - p (rounding may leave less than nothing of it), and q.
__device__ __forceinline__ float ln_variance(float squares, float sum, float inv_H, float& q) {
    q = sum * inv_H;
    return fmaxf(fmaf(-q, q, squares * inv_H), 0.f);
}

// f - mean, 0 for what is behind the row's end.  (A vector at a time: a choice per element is two instructions more for
// each of about twenty.)
template <typename T>
__device__ __forceinline__ void ln_center(float (&f)[RowVec<T>::N], float mean, int v, int nfull, int rem) {
    constexpr int N = RowVec<T>::N;
    if (v < nfull) {
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] -= mean;
    } else {
        const int n = ln_live<T>(v, nfull, rem);
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = e < n ? f[e] - mean : 0.f;
    }
}

template <typename T, int TPR, int NV, bool NT>
__global__ __launch_bounds__(row_block<TPR>) void layer_norm_fwd_kernel(LnArgs a) {
    constexpr int N = RowVec<T>::N, GROUPS = row_groups<TPR>;
    __shared__ float red[2][2 * (TPR > WAVE ? TPR / WAVE : 1)];
    const int grp = row_group<TPR>(), t = threadIdx.x % TPR;
    const float inv_H = 1.0f / (float)a.H;
    const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * GROUPS + grp;
    const bool live = row < a.rows;   // (a group past the last row takes part in the barriers)
    const int nfull = live ? a.H / N : 0, rem = live ? a.H % N : 0;
    const int64_t at = live ? row : 0;
    u32x4 xv[NV], yv[NV], gv[NV], bv[NV];
    auto load = [&](u32x4 (&to)[NV], const void* m, int64_t offset) {
        const T* p = static_cast<const T*>(m) + offset;
#pragma unroll
        for (int k = 0; k < NV; ++k) to[k] = row_load(p, t + k * TPR, nfull, rem);
    };
    load(xv, a.x, at * a.ldx);
    if (a.y) load(yv, a.y, at * a.ldy);
    if (a.gamma) load(gv, a.gamma, 0);
    if (a.beta) load(bv, a.beta, 0);
    float f[NV][N];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        RowVec<T>::unpack(xv[k], f[k]);
        if (a.y) {
            float w[N];
            RowVec<T>::unpack(yv[k], w);
#pragma unroll
            for (int e = 0; e < N; ++e) f[k][e] += w[e];
        }
    }
    if (a.out_h) {
        T* p = static_cast<T*>(a.out_h) + at * a.ldh;
#pragma unroll
        for (int k = 0; k < NV; ++k) row_store<T, NT>(p, t + k * TPR, nfull, rem, f[k]);
    }
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < N; ++e) s += f[k][e];
    const float mean = ln_uniform<TPR>(row_sum<TPR>(s, red[0]) / (float)a.H);
    float sums[2] = {0.f, 0.f};   // of (h - p)^2, h - p
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        ln_center<T>(f[k], mean, t + k * TPR, nfull, rem);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            sums[0] = fmaf(f[k][e], f[k][e], sums[0]);
            sums[1] += f[k][e];
        }
    }
    row_sums<TPR, 2>(sums, red[1]);
    float q;
    const float r = ln_uniform<TPR>(rsqrtf(ln_variance(sums[0], sums[1], inv_H, q) + a.eps));
    const float shift = ln_uniform<TPR>(-q * r);   // (d r = (h - p) r - q r)
    T* p = static_cast<T*>(a.out_n) + at * a.ldn;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        float g[N], b[N];
        if (a.gamma) RowVec<T>::unpack(gv[k], g);
        if (a.beta) RowVec<T>::unpack(bv[k], b);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            f[k][e] = fmaf(f[k][e], r, shift);
            if (a.gamma) f[k][e] *= g[e];
            if (a.beta) f[k][e] += b[e];
        }
        row_store<T, NT>(p, t + k * TPR, nfull, rem, f[k]);
    }
}

// Sum over a workgroup of LN_LONG_THREADS; the barrier in front frees the LDS of the sum before.
template <int K>
__device__ __forceinline__ void ln_long_sums(float (&v)[K], float* red) {
    __syncthreads();
    row_sums<LN_LONG_THREADS, K>(v, red);
}

// Rows beyond the register forms: a workgroup per row, swept three times; the last sweep alone writes, and a thread
// writes only where it has read.
template <typename T, bool NT>
__global__ __launch_bounds__(LN_LONG_THREADS) void layer_norm_fwd_long(LnArgs a) {
    constexpr int N = RowVec<T>::N;
    __shared__ float red[2 * LN_LONG_THREADS / WAVE];
    const int64_t row = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (row >= a.rows) return;
    const int nfull = a.H / N, rem = a.H % N, nvec = nfull + (rem ? 1 : 0);
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* y = a.y ? static_cast<const T*>(a.y) + row * a.ldy : nullptr;
    auto sum_at = [&](int v, float (&f)[N]) {
        RowVec<T>::unpack(row_load(x, v, nfull, rem), f);
        if (y) {
            float w[N];
            RowVec<T>::unpack(row_load(y, v, nfull, rem), w);
#pragma unroll
            for (int e = 0; e < N; ++e) f[e] += w[e];
        }
    };
    float s[1] = {0.f};
    for (int v = threadIdx.x; v < nvec; v += LN_LONG_THREADS) {
        float f[N];
        sum_at(v, f);
#pragma unroll
        for (int e = 0; e < N; ++e) s[0] += f[e];
    }
    ln_long_sums(s, red);
    const float mean = s[0] / (float)a.H;
    float sums[2] = {0.f, 0.f};
    for (int v = threadIdx.x; v < nvec; v += LN_LONG_THREADS) {
        float f[N];
        sum_at(v, f);
        const int n = ln_live<T>(v, nfull, rem);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float d = e < n ? f[e] - mean : 0.f;
            sums[0] = fmaf(d, d, sums[0]);
            sums[1] += d;
        }
    }
    ln_long_sums(sums, red);
    float q;
    const float r = 1.0f / sqrtf(ln_variance(sums[0], sums[1], 1.0f / (float)a.H, q) + a.eps);
    for (int v = threadIdx.x; v < nvec; v += LN_LONG_THREADS) {
        float f[N], w[N];
        sum_at(v, f);
        if (a.out_h) row_store<T, NT>(static_cast<T*>(a.out_h) + row * a.ldh, v, nfull, rem, f);
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = ((f[e] - mean) - q) * r;
        if (a.gamma) {
            RowVec<T>::unpack(row_load(static_cast<const T*>(a.gamma), v, nfull, rem), w);
#pragma unroll
            for (int e = 0; e < N; ++e) f[e] *= w[e];
        }
        if (a.beta) {
            RowVec<T>::unpack(row_load(static_cast<const T*>(a.beta), v, nfull, rem), w);
#pragma unroll
            for (int e = 0; e < N; ++e) f[e] += w[e];
        }
        row_store<T, NT>(static_cast<T*>(a.out_n) + row * a.ldn, v, nfull, rem, f);
    }
}

// Backward: workgroup b takes rows b * GROUPS, (b + gridDim.x) * GROUPS, ...: all workgroups read neighbouring rows at
// a time.  The sums over rows stay in registers until the workgroup's last row and are left as one row of fp32
// partial sums (sum_partials_kernel adds them up in fp64): no atomics, the order depends on the shape and the number
// of workgroups alone.  AHEAD: the next row's loads are issued before a row is worked on.
template <typename T, int TPR, int NV, bool AHEAD, bool NT>
__global__ __launch_bounds__(row_block<TPR>) void layer_norm_bwd_kernel(LnArgs a) {
    constexpr int N = RowVec<T>::N, BLOCK = row_block<TPR>, GROUPS = row_groups<TPR>, NW = TPR > WAVE ? TPR / WAVE : 1;
    constexpr bool EXACT = sizeof(T) == 2;   // the sum of a row
    constexpr bool IN_LDS = TPR == 1024;     // the sums over rows: with them a thread's 128 registers do not do
    __shared__ float red[2][2][4 * NW];
    __shared__ __align__(16) float cols[IN_LDS ? 2 * BLOCK * NV * N : GROUPS > 1 ? BLOCK * NV * N : 4];
    const int grp = row_group<TPR>(), t = threadIdx.x % TPR;
    const int nfull = a.H / N, rem = a.H % N, nvec = nfull + (rem ? 1 : 0);
    const float inv_H = 1.0f / (float)a.H;
    u32x4 gv[NV];
    if (a.gamma)
#pragma unroll
        for (int k = 0; k < NV; ++k) gv[k] = row_load(static_cast<const T*>(a.gamma), t + k * TPR, nfull, rem);
    float acc_gamma[NV][N], acc_beta[NV][N];
    // IN_LDS: four of them, in set 0 (gamma's) or 1; a thread has its own
    auto sums_at = [&](int set, int k, int e) {
        return reinterpret_cast<f32x4*>(cols + ((set * NV + k) * N + e) * BLOCK + (int)threadIdx.x * 4);
    };
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < N; ++e) acc_gamma[k][e] = acc_beta[k][e] = 0.f;
    if constexpr (IN_LDS)
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < N; e += 4) *sums_at(0, k, e) = *sums_at(1, k, e) = f32x4{0.f, 0.f, 0.f, 0.f};

    struct Row {
        u32x4 h[NV], dn[NV], dh[NV];
    };
    auto load_row = [&](Row& r, int64_t base) {
        const bool live = base + grp < a.rows;   // (a group past the last row loads nothing)
        const int64_t row = live ? base + grp : base;
        auto load = [&](u32x4 (&to)[NV], const void* m, int64_t ld) {
            const T* p = static_cast<const T*>(m) + row * ld;
#pragma unroll
            for (int k = 0; k < NV; ++k) to[k] = row_load_ahead(p, t + k * TPR, live ? nvec : 0, a.H);
        };
        load(r.h, a.h, a.ldh);
        load(r.dn, a.dn, a.lddn);
        if (a.dh) load(r.dh, a.dh, a.lddh);
    };
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    int64_t base = (int64_t)blockIdx.x * GROUPS;
    Row next;
    if (AHEAD && base < a.rows) load_row(next, base);
    for (int turn = 0; base < a.rows; base += step, turn ^= 1) {
        if (GROUPS > 1 && base + grp >= a.rows) break;   // (at most a wavefront: no barrier in here is meant for it)
        Row in;
        if constexpr (AHEAD) {
            in = next;
            if (base + step < a.rows) load_row(next, base + step);
        } else {
            load_row(in, base);
        }
        if (rem) {
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (t + k * TPR == nfull) {
                    row_shift_tail<T>(in.h[k], rem);
                    row_shift_tail<T>(in.dn[k], rem);
                    if (a.dh) row_shift_tail<T>(in.dh[k], rem);
                }
        }
        float d[NV][N];   // h, then h - p
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            RowVec<T>::unpack(in.h[k], d[k]);
#pragma unroll
            for (int e = 0; e < N; ++e) s += d[k][e];
        }
        s = row_sum<TPR>(s, red[turn][0]);
        const float mean = ln_uniform<TPR>(s / (float)a.H);
        // the sums of (h - p)^2, u, u (h - p) and, unless it is known, h - p in one exchange
        constexpr int SUMS = EXACT ? 3 : 4;
        float sums[SUMS] = {};
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float u[N], g[N];
            ln_center<T>(d[k], mean, t + k * TPR, nfull, rem);
            RowVec<T>::unpack(in.dn[k], u);
            if (a.gamma) {
                RowVec<T>::unpack(gv[k], g);
#pragma unroll
                for (int e = 0; e < N; ++e) u[e] *= g[e];
            }
#pragma unroll
            for (int e = 0; e < N; ++e) {
                sums[0] = fmaf(d[k][e], d[k][e], sums[0]);
                sums[1] += u[e];
                sums[2] = fmaf(u[e], d[k][e], sums[2]);
                if constexpr (!EXACT) sums[SUMS - 1] += d[k][e];
            }
        }
        row_sums<TPR, SUMS>(sums, red[turn][1]);
        float q;
        const float var = ln_variance(sums[0], EXACT ? fmaf(-mean, (float)a.H, s) : sums[SUMS - 1], inv_H, q);
        q = ln_uniform<TPR>(q);
        const float ud = fmaf(-q, sums[1], sums[2]);   // sum u d
        // dx = dh + r u - r mean u - d r^3 mean(u d)
        const float r = ln_uniform<TPR>(rsqrtf(var + a.eps)), shift = ln_uniform<TPR>(-r * (sums[1] * inv_H));
        const float slope = ln_uniform<TPR>(-(r * (r * (r * (ud * inv_H)))));
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float dn[N], g[N], D[N];
            RowVec<T>::unpack(in.dn[k], dn);
            if (a.gamma) RowVec<T>::unpack(gv[k], g);
            if (a.dh) RowVec<T>::unpack(in.dh[k], D);
            if constexpr (IN_LDS) {
#pragma unroll
                for (int e = 0; e < N; e += 4) {
                    f32x4 b = *sums_at(1, k, e), c = *sums_at(0, k, e);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        b[i] += dn[e + i];
                        c[i] = fmaf(dn[e + i] * r, d[k][e + i] - q, c[i]);
                    }
                    *sums_at(1, k, e) = b;
                    *sums_at(0, k, e) = c;
                }
            }
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float dnr = dn[e] * r, dq = d[k][e] - q;
                if constexpr (!IN_LDS) {
                    acc_beta[k][e] += dn[e];
                    acc_gamma[k][e] = fmaf(dnr, dq, acc_gamma[k][e]);
                }
                const float v = fmaf(slope, dq, a.gamma ? fmaf(dnr, g[e], shift) : dnr + shift);
                D[e] = a.dh ? D[e] + v : v;
            }
            if (a.dx) row_store<T, NT>(static_cast<T*>(a.dx) + (base + grp) * a.lddx, t + k * TPR, nfull, rem, D);
        }
    }

    if constexpr (IN_LDS) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                acc_gamma[k][e] = (*sums_at(0, k, e / 4 * 4))[e % 4];
                acc_beta[k][e] = (*sums_at(1, k, e / 4 * 4))[e % 4];
            }
    }
    // The workgroup's row of sums (over its groups, in order), rounded to `out` or as it is to `part`.
    auto put_sums = [&](float (&acc)[NV][N], T* out, float* part) {
        if constexpr (GROUPS > 1) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < N; e += 4)
                    *reinterpret_cast<f32x4*>(&cols[grp * (TPR * NV * N) + (t + k * TPR) * N + e]) =
                        f32x4{acc[k][e], acc[k][e + 1], acc[k][e + 2], acc[k][e + 3]};
            __syncthreads();
            for (int j = threadIdx.x; j < TPR * NV * N && j < a.H; j += BLOCK) {
                float s = cols[j];
                for (int q = 1; q < GROUPS; ++q) s += cols[q * (TPR * NV * N) + j];
                if (out) out[j] = from_f32<T>(s); else part[j] = s;
            }
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int at = t + k * TPR;
                if (out) {
                    row_store<T, false>(out, at, nfull, rem, acc[k]);
                } else if (at < nfull) {
#pragma unroll
                    for (int e = 0; e < N; e += 4)
                        *reinterpret_cast<f32x4_any*>(part + at * N + e) = f32x4{acc[k][e], acc[k][e + 1], acc[k][e + 2], acc[k][e + 3]};
                } else if (at == nfull) {
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        if (e < rem) part[at * N + e] = acc[k][e];
                }
            }
        }
    };
    if (a.dgamma) put_sums(acc_gamma, static_cast<T*>(a.dgamma), nullptr);
    else if (a.part_gamma) put_sums(acc_gamma, nullptr, a.part_gamma + (int64_t)blockIdx.x * a.H);
    if (a.dbeta) put_sums(acc_beta, static_cast<T*>(a.dbeta), nullptr);
    else if (a.part_beta) put_sums(acc_beta, nullptr, a.part_beta + (int64_t)blockIdx.x * a.H);
}

// Rows beyond the register forms, and rows of less than a vector.  The sums over rows live in the partial sums'
// memory; a column always belongs to the same thread.
template <typename T, bool NT>
__global__ __launch_bounds__(LN_LONG_THREADS) void layer_norm_bwd_long(LnArgs a) {
    constexpr int N = RowVec<T>::N;
    __shared__ float red[4 * LN_LONG_THREADS / WAVE];
    const int nfull = a.H / N, rem = a.H % N, nvec = nfull + (rem ? 1 : 0);
    float* pg = a.part_gamma ? a.part_gamma + (int64_t)blockIdx.x * a.H : nullptr;
    float* pb = a.part_beta ? a.part_beta + (int64_t)blockIdx.x * a.H : nullptr;
    const T* gamma = static_cast<const T*>(a.gamma);
    bool first = true;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, first = false) {
        const T* h = static_cast<const T*>(a.h) + row * a.ldh;
        const T* dn = static_cast<const T*>(a.dn) + row * a.lddn;
        float s[1] = {0.f};
        for (int v = threadIdx.x; v < nvec; v += LN_LONG_THREADS) {
            float f[N];
            RowVec<T>::unpack(row_load(h, v, nfull, rem), f);
#pragma unroll
            for (int e = 0; e < N; ++e) s[0] += f[e];
        }
        ln_long_sums(s, red);
        const float mean = s[0] / (float)a.H;
        float sums[4] = {0.f, 0.f, 0.f, 0.f};
        auto centered = [&](int v, float (&d)[N], float (&u)[N], float (&g)[N]) {   // h - p, dn, gamma
            RowVec<T>::unpack(row_load(h, v, nfull, rem), d);
            RowVec<T>::unpack(row_load(dn, v, nfull, rem), u);
            if (gamma) RowVec<T>::unpack(row_load(gamma, v, nfull, rem), g);
            const int n = ln_live<T>(v, nfull, rem);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                d[e] = e < n ? d[e] - mean : 0.f;
                if (!gamma) g[e] = 1.0f;
            }
        };
        for (int v = threadIdx.x; v < nvec; v += LN_LONG_THREADS) {
            float d[N], u[N], g[N];
            centered(v, d, u, g);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                sums[0] = fmaf(d[e], d[e], sums[0]);
                sums[1] = fmaf(u[e], g[e], sums[1]);
                sums[2] = fmaf(u[e] * g[e], d[e], sums[2]);
                sums[3] += d[e];
            }
        }
        ln_long_sums(sums, red);
        float q;
        const float r = 1.0f / sqrtf(ln_variance(sums[0], sums[3], 1.0f / (float)a.H, q) + a.eps);
        const float mu = sums[1] / (float)a.H, mx = fmaf(-q, sums[1], sums[2]) * r / (float)a.H;
        for (int v = threadIdx.x; v < nvec; v += LN_LONG_THREADS) {
            float d[N], u[N], g[N], D[N];
            centered(v, d, u, g);
            if (a.dh) RowVec<T>::unpack(row_load(static_cast<const T*>(a.dh) + row * a.lddh, v, nfull, rem), D);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float xh = (d[e] - q) * r, w = r * (u[e] * g[e] - mu - xh * mx);
                D[e] = a.dh ? D[e] + w : w;
                if (v * N + e < a.H) {
                    if (pg) pg[v * N + e] = first ? u[e] * xh : fmaf(u[e], xh, pg[v * N + e]);
                    if (pb) pb[v * N + e] = first ? u[e] : u[e] + pb[v * N + e];
                }
            }
            if (a.dx) row_store<T, NT>(static_cast<T*>(a.dx) + row * a.lddx, v, nfull, rem, D);
        }
    }
}

}  // namespace flce
