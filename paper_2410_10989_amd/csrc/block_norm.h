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
// alignment (they cost where lines are straddled: backward of 8192 rows of 4096 / 4095 bf16 67 / 88 us).  Rows that
// are too long for that (`*_long`) are swept several times by a workgroup of 1024 threads (2048 x 20000 bf16 with both
// norms and a gate: forward 127 us, backward 619).
//
// Bound by HBM.  What streams of 117 MB each reach on this chip with nothing to compute, from one set of buffers (of
// which the memory-side cache keeps some from pass to pass) / from three in turn: two read and two written 7.2 / 6.3
// TB/s, four read and two written 6.9 / 6.1.
#pragma once
#include "flce_device.h"
#include "rowsums.h"
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
    void *dpre, *dpost;   // one workgroup has all rows: the gammas' gradients are written at once
};

// 1 / (1 + e), e in [0, 1]: the hardware's reciprocal (1 ulp) and one Newton step.
__device__ __forceinline__ float bn_one_over_1p(float e) {
    const float x = 1.0f + e, d = __builtin_amdgcn_rcpf(x);
    return fmaf(fmaf(-x, d, 1.0f), d, d);
}
// a(g) and a'(g).  exp is taken of -|g| only, and 1 - sigmoid and the derivatives come as products of what
// does not cancel, so that they keep their relative accuracy where a gate saturates.
__device__ __forceinline__ float bn_act(int act, float g) {
    if (act == BN_ACT_LINEAR) return g;
    if (act == BN_ACT_TANH) return tanhf(g);
    const float e = expf(-fabsf(g)), d = bn_one_over_1p(e);
    const float sig = g >= 0.f ? d : e * d;
    return act == BN_ACT_SIGMOID ? sig : g * sig;
}
__device__ __forceinline__ void bn_act_both(int act, float g, float& a, float& da) {
    if (act == BN_ACT_LINEAR) {
        a = g;
        da = 1.0f;
    } else if (act == BN_ACT_TANH) {
        const float e = expf(-2.0f * fabsf(g)), d = bn_one_over_1p(e);
        a = tanhf(g);
        da = 4.0f * e * d * d;
    } else {
        const float e = expf(-fabsf(g)), d = bn_one_over_1p(e);
        const float sig = g >= 0.f ? d : e * d, rest = g >= 0.f ? e * d : d;
        a = act == BN_ACT_SIGMOID ? sig : g * sig;
        da = act == BN_ACT_SIGMOID ? sig * rest : sig * (1.0f + g * rest);
    }
}

// Forward: a workgroup holds row_groups rows.  All loads of a row are issued before the first is used, the
// occupancy (37 to 106 registers with everything on) covers the rest.  us: 8192 x 4096 bf16 with the next block's norm
// 38 (7.0 TB/s), 16384 x 3584 with both norms and a gate 67 (7.0; 85 where nothing read is in the cache yet: 5.5),
// 2047 x 1000 fp32 with a sigmoid gate per token 10.5, one row of 4096 2.8.
template <typename T, int TPR, int NV, bool POST, bool GATE, bool NT>
__global__ __launch_bounds__(row_block<TPR>) void block_norm_fwd_kernel(BnArgs a) {
    constexpr int N = RowVec<T>::N, GROUPS = row_groups<TPR>;
    __shared__ float red[2][TPR > WAVE ? TPR / WAVE : 1];
    const int grp = row_group<TPR>(), t = threadIdx.x % TPR;
    const float inv_H = 1.0f / (float)a.H;
    const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * GROUPS + grp;
    const bool live = row < a.rows;   // (a group past the last row takes part in the barriers)
    const int nfull = live ? a.H / N : 0, rem = live ? a.H % N : 0;
    const int64_t at = live ? row : 0;
    u32x4 xv[NV], yv[NV], gv[NV], pv[NV], nv[NV];
    auto load = [&](u32x4 (&to)[NV], const void* m, int64_t offset) {
        const T* p = static_cast<const T*>(m) + offset;
#pragma unroll
        for (int k = 0; k < NV; ++k) to[k] = row_load(p, t + k * TPR, nfull, rem);
    };
    if (a.x) load(xv, a.x, at * a.ldx);
    if (a.y) load(yv, a.y, at * a.ldy);
    if constexpr (GATE) load(gv, a.gate, (int64_t)((uint32_t)at / (uint32_t)a.per) * a.ldgate);
    if constexpr (POST) load(pv, a.gpost, 0);
    if (a.gpre) load(nv, a.gpre, 0);
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
            q = rsqrtf(row_sum<TPR>(ss, red[0]) * inv_H + a.eps);
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
            for (int k = 0; k < NV; ++k) row_store<T, NT>(p, t + k * TPR, nfull, rem, f[k]);
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
        const float r = rsqrtf(row_sum<TPR>(ss, red[1]) * inv_H + a.eps);
        T* p = static_cast<T*>(a.out_n) + at * a.ldn;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float w[N];
            RowVec<T>::unpack(nv[k], w);
#pragma unroll
            for (int e = 0; e < N; ++e) w[e] *= f[k][e] * r;
            row_store<T, NT>(p, t + k * TPR, nfull, rem, w);
        }
    }
}

// Sum over a workgroup of BN_LONG_THREADS; the barrier in front frees the LDS of the sum before.
__device__ __forceinline__ float bn_long_sum(float v, float* red) {
    __syncthreads();
    return row_sum<BN_LONG_THREADS>(v, red);
}

// scale a(g) z of one vector of a row (z before the gate comes back too, for the backward).
template <typename T>
__device__ __forceinline__ void bn_long_z(const BnArgs& a, const T* y, const T* gate, float q, int v, int nfull,
                                          int rem, float (&z)[RowVec<T>::N], float (&out)[RowVec<T>::N]) {
    constexpr int N = RowVec<T>::N;
    float w[N];
    RowVec<T>::unpack(row_load(y, v, nfull, rem), z);
    if (a.gpost) {
        RowVec<T>::unpack(row_load(static_cast<const T*>(a.gpost), v, nfull, rem), w);
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] *= q * w[e];
    }
    if (gate) RowVec<T>::unpack(row_load(gate, v, nfull, rem), w);
#pragma unroll
    for (int e = 0; e < N; ++e) out[e] = a.scale * (gate ? z[e] * bn_act(a.act, w[e]) : z[e]);
}

template <typename T>
__device__ __forceinline__ float bn_long_rstd(const T* row, int nvec, int nfull, int rem, const BnArgs& a, float* red) {
    constexpr int N = RowVec<T>::N;
    float ss = 0.f;
    for (int v = threadIdx.x; v < nvec; v += BN_LONG_THREADS) {
        float f[N];
        RowVec<T>::unpack(row_load(row, v, nfull, rem), f);
#pragma unroll
        for (int e = 0; e < N; ++e) ss += f[e] * f[e];
    }
    return 1.0f / sqrtf(bn_long_sum(ss, red) / (float)a.H + a.eps);
}

// Rows beyond the register forms: one workgroup per row, swept up to three times; the last sweep alone writes,
// and a thread writes only where it has read, so that h may lie on x.
template <typename T, bool NT>
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
            RowVec<T>::unpack(row_load(x, v, nfull, rem), z);
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
        if (a.out_h) row_store<T, NT>(static_cast<T*>(a.out_h) + row * a.ldh, v, nfull, rem, f);
        if (a.gpre) {
            float w[N];
            RowVec<T>::unpack(row_load(static_cast<const T*>(a.gpre), v, nfull, rem), w);
#pragma unroll
            for (int e = 0; e < N; ++e) w[e] *= f[e] * r;
            row_store<T, NT>(static_cast<T*>(a.out_n) + row * a.ldn, v, nfull, rem, w);
        }
    }
}

// Segment s: the rows row, row + step, ... below end of gate row g, `groups` rows side by side each time.
struct BnSegment {
    int g, row, end, step;
};
__device__ __forceinline__ BnSegment bn_segment(const BnArgs& a, int s, int groups) {
    const int g = s / a.parts;
    const int first = g * a.per;
    return {g, first + (s - g * a.parts) * groups, first + min(a.per, a.rows - first), a.parts * groups};
}

// A thread's part of a row of every stream the backward reads.
template <int NV>
struct BnRow {
    u32x4 h[NV], dn[NV], y[NV], dh[NV], gate[NV];
};

// Backward: workgroup b takes segments b, b + gridDim.x, ...; its GROUPS rows at a time.  The sums over rows
// stay in registers: the gammas' until the workgroup's last row, a shared gate's until its segment's; then the
// groups of a workgroup add theirs up in a fixed order.  Sums of several workgroups are left as rows of fp32
// partial sums for sum_partials_kernel: no atomics, the order of additions depends on the shape and the number
// of workgroups alone.  The rows of a segment's parts are dealt side by side, so that all workgroups read
// neighbouring rows at a time (16384 x 3584: 149 -> 136 us against one stretch of rows each), and the sums are stored
// in 16-byte pieces (element by element, 32 x 4096 11.3 instead of 8.3 us).
// AHEAD: the next row's loads are issued before a row is worked on: registers instead of more workgroups, every one
// of which costs its partial sums (8192 x 4096 without sums of a second norm 74 -> 69 us).  WIDE: the sums over rows
// are kept in LDS, where registers do not hold them beside rows of 32 elements per thread; each column belongs to one
// thread.  us, there / in the long form: 2048 x 12000 bf16 with one set of sums 62 / 140, two 84 / 247, three 123 / 356;
// 2048 x 8200 fp32 72 / 140, 120 / 232, 197 / 307.  Registers spill to scratch memory in the WIDE forms of fp32 but for
// the one without a norm after the block and a gate (44 to 184 bytes per lane), in those of bf16 with a norm after the
// block (12 to 84), and in (512, 16) with three sets (fp32 64, bf16 44): 4096 x 8192 bf16 82 us, 56 with one set.
// us, with the partial sums' launch (4-5): 16384 x 3584 bf16, both norms, a gate per channel 134 (5.3 TB/s; traffic
// 470 MB read and 246 written, 705 it cannot do without; vector instructions 47 % of the cycles), 8192 x 4096 with
// the next block's norm 55, 2047 x 1000 fp32 with a silu gate per sequence 19.
constexpr int BN_WIDE_COLS = 16384, BN_WIDE_COLS_3 = 13312;   // of up to two and of three sets of sums: 160 KB
template <typename T, int TPR, int NV, bool POST, int GATE, bool AHEAD, bool WIDE, bool NT>
__global__ __launch_bounds__(row_block<TPR>) void block_norm_bwd_kernel(BnArgs a) {
    constexpr int N = RowVec<T>::N, BLOCK = row_block<TPR>, GROUPS = row_groups<TPR>, NW = TPR > WAVE ? TPR / WAVE : 1;
    __shared__ float red[3][3 * NW];
    __shared__ __align__(16) float cols[GROUPS > 1 ? BLOCK * NV * N : 4];
    constexpr int SETS = 1 + POST + (GATE == BN_GATE_SUM), COLS = SETS == 3 ? BN_WIDE_COLS_3 : BN_WIDE_COLS;
    constexpr int AT_PRE = 0, AT_POST = COLS, AT_GATE = (1 + POST) * COLS;
    __shared__ __align__(16) float wide[WIDE ? SETS * COLS : 4];
    const int grp = row_group<TPR>(), t = threadIdx.x % TPR;
    const int nfull_all = a.H / N, rem_all = a.H % N;
    const float inv_H = 1.0f / (float)a.H;
    u32x4 prev[NV], postv[NV];
    constexpr int NA = WIDE ? 1 : NV;
    float acc_pre[NA][N], acc_post[NA][N], acc_gate[NA][N];
    float ga[NA][N], gd[NA][N];   // scale a(g), scale a'(g); WIDE: of the vector at hand
#pragma unroll
    for (int k = 0; k < NA; ++k)
#pragma unroll
        for (int e = 0; e < N; ++e) acc_pre[k][e] = acc_post[k][e] = acc_gate[k][e] = 0.f;
    // the sums of a thread's vector k in LDS, and what is added to them
    auto wide_at = [&](int set, int k) { return wide + set + (t + k * TPR) * N; };
    auto wide_clear = [&](int set) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if ((t + k * TPR) * N < a.H)
#pragma unroll
                for (int e = 0; e < N; ++e) wide_at(set, k)[e] = 0.f;
    };
    auto wide_add = [&](int set, int k, const float (&v)[N]) {
        if ((t + k * TPR) * N < a.H) {
            f32x4* p = reinterpret_cast<f32x4*>(wide_at(set, k));
#pragma unroll
            for (int q = 0; q < N / 4; ++q) {
                f32x4 s = p[q];
#pragma unroll
                for (int e = 0; e < 4; ++e) s[e] += v[q * 4 + e];
                p[q] = s;
            }
        }
    };
    if constexpr (WIDE)
        for (int i = 0; i < SETS; ++i) wide_clear(i * COLS);
    auto load_shared = [&](const void* m, int64_t offset, int v) {   // of what many rows share
        // (WIDE reads it again for every row: kept over the rows it would take the registers of the rows)
        if constexpr (WIDE) asm volatile("" : "+s"(m));
        return row_load(static_cast<const T*>(m) + offset, v, nfull_all, rem_all);
    };
    if (a.gpre && !WIDE)
#pragma unroll
        for (int k = 0; k < NV; ++k) prev[k] = load_shared(a.gpre, 0, t + k * TPR);
    if constexpr (POST && !WIDE)
#pragma unroll
        for (int k = 0; k < NV; ++k) postv[k] = load_shared(a.gpost, 0, t + k * TPR);
    auto pre_vector = [&](int k) { return WIDE ? load_shared(a.gpre, 0, t + k * TPR) : prev[k]; };
    [[maybe_unused]] auto post_vector = [&](int k) { return WIDE ? load_shared(a.gpost, 0, t + k * TPR) : postv[k]; };

    // The workgroup's row of sums (over its groups, in order), rounded to `out` or as it is to `part`.
    auto put_sums = [&](float (&acc)[NA][N], [[maybe_unused]] int set, T* out, float* part) {
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
                float v[N];
                const int at = t + k * TPR;
                if (at * N >= a.H) continue;   // (the sets in LDS end there)
#pragma unroll
                for (int e = 0; e < N; ++e) v[e] = WIDE ? wide_at(set, k)[e] : acc[WIDE ? 0 : k][e];
                if (out) {
                    row_store<T, false>(out, at, nfull_all, rem_all, v);
                } else if (at < nfull_all) {
#pragma unroll
                    for (int e = 0; e < N; e += 4)
                        *reinterpret_cast<f32x4_any*>(part + at * N + e) = f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]};
                } else if (at == nfull_all) {
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        if (e < rem_all) part[at * N + e] = v[e];
                }
            }
        }
    };

    auto load_row = [&](BnRow<NV>& r, int base, int end) {
        const bool live = GROUPS == 1 || base + grp < end;   // (a group past the last row loads nothing)
        const int64_t row = live ? base + grp : base;
        const int nvec = live ? nfull_all + (rem_all ? 1 : 0) : 0;
        auto load = [&](u32x4 (&to)[NV], const void* m, int64_t ld) {
            const T* p = static_cast<const T*>(m) + row * ld;
#pragma unroll
            for (int k = 0; k < NV; ++k) to[k] = row_load_ahead(p, t + k * TPR, nvec, a.H);
        };
        if (a.gpre) {
            load(r.h, a.h, a.ldh);
            load(r.dn, a.dn, a.lddn);
        }
        if (a.y) load(r.y, a.y, a.ldy);
        if (a.dh) load(r.dh, a.dh, a.lddh);
        if constexpr (GATE == BN_GATE_ROW) load(r.gate, a.gate, a.ldgate);
    };

    int turn = 0;
    for (int s = blockIdx.x; s < a.segments; s += gridDim.x) {
        const BnSegment seg = bn_segment(a, s, GROUPS);
        auto gate_vector = [&](int k, float (&act)[N], float (&slope)[N]) {
            float g[N];
            RowVec<T>::unpack(load_shared(a.gate, (int64_t)seg.g * a.ldgate, t + k * TPR), g);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                bn_act_both(a.act, g[e], act[e], slope[e]);
                act[e] *= a.scale;
                slope[e] *= a.scale;
            }
        };
        if constexpr (GATE == BN_GATE_SUM && !WIDE) {
#pragma unroll
            for (int k = 0; k < NV; ++k) gate_vector(k, ga[k], gd[k]);
        }
        BnRow<NV> next;
        if (AHEAD && seg.row < seg.end) load_row(next, seg.row, seg.end);
        for (int base = seg.row; base < seg.end; base += seg.step, turn ^= 1) {
            // A group past the segment's last row (at most a wavefront: no barrier in here is meant for it) has none in
            // any later step either.  It must not go on with zeros: with eps = 0 their 1 / rms is infinite, and 0 times
            // that would be NaN in the sums over rows.
            if (GROUPS > 1 && base + grp >= seg.end) break;
            const int64_t row = base + grp;
            const int nfull = nfull_all, rem = rem_all;
            BnRow<NV> in;
            if constexpr (AHEAD) {
                in = next;
                if (base + seg.step < seg.end) load_row(next, base + seg.step, seg.end);
            } else {
                load_row(in, base, seg.end);
            }
            if (rem) {
#pragma unroll
                for (int k = 0; k < NV; ++k)
                    if (t + k * TPR == nfull) {
                        if (a.gpre) {
                            row_shift_tail<T>(in.h[k], rem);
                            row_shift_tail<T>(in.dn[k], rem);
                        }
                        if (a.y) row_shift_tail<T>(in.y[k], rem);
                        if (a.dh) row_shift_tail<T>(in.dh[k], rem);
                        if constexpr (GATE == BN_GATE_ROW) row_shift_tail<T>(in.gate[k], rem);
                    }
            }
            // sum h^2, sum u h and sum y^2 in one exchange
            float sums[3] = {0.f, 0.f, 0.f};
            if (a.gpre) {
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    float h[N], d[N], w[N];
                    RowVec<T>::unpack(in.h[k], h);
                    RowVec<T>::unpack(in.dn[k], d);
                    RowVec<T>::unpack(pre_vector(k), w);
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        sums[0] = fmaf(h[e], h[e], sums[0]);
                        sums[1] = fmaf(d[e] * w[e], h[e], sums[1]);
                    }
                }
            }
            if constexpr (POST) {
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    float y[N];
                    RowVec<T>::unpack(in.y[k], y);
#pragma unroll
                    for (int e = 0; e < N; ++e) sums[2] = fmaf(y[e], y[e], sums[2]);
                }
            }
            if constexpr (POST) {
                row_sums<TPR, 3>(sums, red[0]);   // (the barrier of the second exchange stands between two of these)
            } else if (a.gpre) {
                float two[2] = {sums[0], sums[1]};
                row_sums<TPR, 2>(two, red[turn]);
                sums[0] = two[0];
                sums[1] = two[1];
            }
            // D = dh + r u - r^2 mean(u h r) h, the gradient of h
            float D[NV][N];
            auto unpack_dh = [&](float (&to)[N], int k) {
                if (a.dh) RowVec<T>::unpack(in.dh[k], to);
                else
#pragma unroll
                    for (int e = 0; e < N; ++e) to[e] = 0.f;
            };
            if (a.gpre) {
                const float r = rsqrtf(sums[0] * inv_H + a.eps), hk = -(r * (r * (sums[1] * r * inv_H)));
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    float h[N], d[N], w[N];
                    RowVec<T>::unpack(in.h[k], h);
                    RowVec<T>::unpack(in.dn[k], d);
                    RowVec<T>::unpack(pre_vector(k), w);
                    unpack_dh(D[k], k);
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const float dr = d[e] * r;
                        D[k][e] = fmaf(dr, w[e], fmaf(hk, h[e], D[k][e]));
                        if constexpr (WIDE) d[e] = dr * h[e];
                        else acc_pre[k][e] = fmaf(dr, h[e], acc_pre[k][e]);
                    }
                    if constexpr (WIDE) wide_add(AT_PRE, k, d);
                }
            } else {
#pragma unroll
                for (int k = 0; k < NV; ++k) unpack_dh(D[k], k);
            }
            if (a.dx) {
                T* p = static_cast<T*>(a.dx) + row * a.lddx;
#pragma unroll
                for (int k = 0; k < NV; ++k) row_store<T, NT>(p, t + k * TPR, nfull, rem, D[k]);
            }
            if (!a.y) continue;
            const float q = POST ? rsqrtf(sums[2] * inv_H + a.eps) : 1.0f;
            // D becomes dz, then (with a norm after the block) v = dz gamma_post
            float vy[1] = {0.f};
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                float y[N], w[N], g[N];
                RowVec<T>::unpack(in.y[k], y);
                if constexpr (POST) RowVec<T>::unpack(post_vector(k), w);
                if constexpr (GATE == BN_GATE_ROW) RowVec<T>::unpack(in.gate[k], g);
                if constexpr (GATE == BN_GATE_SUM && WIDE) gate_vector(k, ga[0], gd[0]);
                [[maybe_unused]] float to_post[N], to_gate[N];
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if constexpr (POST) y[e] *= q;
                    if constexpr (GATE == BN_GATE_NONE) {
                        D[k][e] *= a.scale;
                    } else if constexpr (GATE == BN_GATE_SUM) {
                        const float z = POST ? y[e] * w[e] : y[e];
                        if constexpr (WIDE) to_gate[e] = D[k][e] * gd[0][e] * z;
                        else acc_gate[k][e] = fmaf(D[k][e] * gd[k][e], z, acc_gate[k][e]);
                        D[k][e] *= ga[WIDE ? 0 : k][e];
                    } else {
                        const float z = POST ? y[e] * w[e] : y[e];
                        float act, slope;
                        bn_act_both(a.act, g[e], act, slope);
                        D[k][e] *= a.scale;
                        g[e] = D[k][e] * z * slope;
                        D[k][e] *= act;
                    }
                    if constexpr (POST) {
                        if constexpr (WIDE) to_post[e] = D[k][e] * y[e];
                        else acc_post[k][e] = fmaf(D[k][e], y[e], acc_post[k][e]);
                        D[k][e] *= w[e];
                        vy[0] = fmaf(D[k][e], y[e], vy[0]);
                    }
                }
                if constexpr (WIDE && GATE == BN_GATE_SUM) wide_add(AT_GATE, k, to_gate);
                if constexpr (WIDE && POST) wide_add(AT_POST, k, to_post);
                if constexpr (GATE == BN_GATE_ROW) {
                    if (a.dgate) row_store<T, NT>(static_cast<T*>(a.dgate) + row * a.lddgate, t + k * TPR, nfull, rem, g);
                }
            }
            if constexpr (POST) {
                row_sums<TPR, 1>(vy, red[2]);
                const float yk = -(q * (q * (vy[0] * inv_H)));
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    float y[N];
                    RowVec<T>::unpack(in.y[k], y);
#pragma unroll
                    for (int e = 0; e < N; ++e) D[k][e] = fmaf(yk, y[e], q * D[k][e]);
                }
            }
            if (a.dy) {
                T* p = static_cast<T*>(a.dy) + row * a.lddy;
#pragma unroll
                for (int k = 0; k < NV; ++k) row_store<T, NT>(p, t + k * TPR, nfull, rem, D[k]);
            }
        }
        if constexpr (GATE == BN_GATE_SUM) {
            if (a.gate_direct) put_sums(acc_gate, AT_GATE, static_cast<T*>(a.dgate) + (int64_t)seg.g * a.lddgate, nullptr);
            else if (a.part_gate) put_sums(acc_gate, AT_GATE, nullptr, a.part_gate + (int64_t)s * a.H);
            if constexpr (WIDE) wide_clear(AT_GATE);
#pragma unroll
            for (int k = 0; k < NA; ++k)
#pragma unroll
                for (int e = 0; e < N; ++e) acc_gate[k][e] = 0.f;
        }
    }
    if (a.dpre) put_sums(acc_pre, AT_PRE, static_cast<T*>(a.dpre), nullptr);
    else if (a.part_pre) put_sums(acc_pre, AT_PRE, nullptr, a.part_pre + (int64_t)blockIdx.x * a.H);
    if constexpr (POST) {
        if (a.dpost) put_sums(acc_post, AT_POST, static_cast<T*>(a.dpost), nullptr);
        else if (a.part_post) put_sums(acc_post, AT_POST, nullptr, a.part_post + (int64_t)blockIdx.x * a.H);
    }
}

// Rows beyond the register forms (see block_norm_fwd_long).  The sums over rows live in the partial sums'
// memory (a gate's: a row per workgroup, or per segment where several share a gate row); a column always
// belongs to the same thread.
template <typename T, bool NT>
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
        const BnSegment seg = bn_segment(a, s, 1);
        float* gsum = a.part_gate ? a.part_gate + (int64_t)(a.gate_direct ? blockIdx.x : s) * a.H : nullptr;
        if (gsum) each(gsum, [](float* p, int j) { p[j] = 0.f; });
        for (int64_t row = seg.row; row < seg.end; row += seg.step) {
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
                    RowVec<T>::unpack(row_load(h, v, nfull, rem), hf);
                    RowVec<T>::unpack(row_load(dn, v, nfull, rem), u);
                    RowVec<T>::unpack(row_load(gpre, v, nfull, rem), w);
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
                if (dh) RowVec<T>::unpack(row_load(dh, v, nfull, rem), D);
                if (h) {
                    float hf[N], u[N], w[N];
                    RowVec<T>::unpack(row_load(h, v, nfull, rem), hf);
                    RowVec<T>::unpack(row_load(dn, v, nfull, rem), u);
                    RowVec<T>::unpack(row_load(gpre, v, nfull, rem), w);
#pragma unroll
                    for (int e = 0; e < N; ++e) D[e] += r * (u[e] * w[e] - hf[e] * r * c);
                }
            };
            auto grad_z = [&](int v, const float (&D)[N], float (&dz)[N]) {
                float g[N];
                if (gate) RowVec<T>::unpack(row_load(gate, v, nfull, rem), g);
#pragma unroll
                for (int e = 0; e < N; ++e) dz[e] = a.scale * D[e] * (gate ? bn_act(a.act, g[e]) : 1.0f);
            };
            if (y && gpost) {
                float vy = 0.f;
                for (int v = threadIdx.x; v < nvec; v += BN_LONG_THREADS) {
                    float D[N], dz[N], yf[N], w[N];
                    grad_h(v, D);
                    grad_z(v, D, dz);
                    RowVec<T>::unpack(row_load(y, v, nfull, rem), yf);
                    RowVec<T>::unpack(row_load(gpost, v, nfull, rem), w);
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
                    RowVec<T>::unpack(row_load(h, v, nfull, rem), hf);
                    RowVec<T>::unpack(row_load(dn, v, nfull, rem), u);
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        if (v * N + e < a.H) pre[v * N + e] += u[e] * (hf[e] * r);
                }
                if (y) {
                    float dz[N], yf[N], w[N], g[N], dg[N];
                    grad_z(v, D, dz);
                    RowVec<T>::unpack(row_load(y, v, nfull, rem), yf);
                    if (gpost) RowVec<T>::unpack(row_load(gpost, v, nfull, rem), w);
                    if (gate) {
                        RowVec<T>::unpack(row_load(gate, v, nfull, rem), g);
#pragma unroll
                        for (int e = 0; e < N; ++e) {
                            const float z = gpost ? yf[e] * q * w[e] : yf[e];
                            float act, slope;
                            bn_act_both(a.act, g[e], act, slope);
                            dg[e] = a.scale * D[e] * z * slope;
                            if (gsum && v * N + e < a.H) gsum[v * N + e] += dg[e];
                        }
                        if (a.by_row && a.dgate)
                            row_store<T, NT>(static_cast<T*>(a.dgate) + row * a.lddgate, v, nfull, rem, dg);
                    }
                    if (gpost) {
#pragma unroll
                        for (int e = 0; e < N; ++e) {
                            const float yh = yf[e] * q;
                            if (post && v * N + e < a.H) post[v * N + e] += dz[e] * yh;
                            dz[e] = q * (dz[e] * w[e] - yh * cy);
                        }
                    }
                    if (a.dy) row_store<T, NT>(static_cast<T*>(a.dy) + row * a.lddy, v, nfull, rem, dz);
                }
                if (a.dx) row_store<T, NT>(static_cast<T*>(a.dx) + row * a.lddx, v, nfull, rem, D);
            }
        }
        if (gsum && a.gate_direct) {
            T* out = static_cast<T*>(a.dgate) + (int64_t)seg.g * a.lddgate;
            each(gsum, [&](float* p, int j) { out[j] = from_f32<T>(p[j]); });
        }
    }
}

}  // namespace flce
