// Embedding lookup with scaling, and the gradient of the table.  With t_i the token of row i counted from the table's
// first one, live rows those whose t_i is a row of the table and not the ignored token,
//
//     out_i = s E[t_i]   (0 for rows that are not live)          dE_v = (dE_v +) s sum_{i live, t_i = v} dY_i
//
// The gradient's rows are added up in the order of i, whatever the machine does: no atomics on values.
//   1. embed_sort_kernel    the live rows' numbers ordered by token (a stable counting sort), in one launch: workgroup
//                           b owns EM tokens and looks at all rows, so it counts what lies before its tokens itself and
//                           waits for nobody.  Rows of the table that no token names are filled with zeros here.
//   2. embed_sum_kernel     pieces of EM_PIECE consecutive entries of that order, a wavefront per piece and
//                           64 vectors of the row: the same work for everybody, however often a token comes.  What
//                           begins and ends in a piece is written at once, the rest is left as fp32 sums.
//   3. embed_join_kernel    the sums of a token that several pieces share, in order, in fp64.
#pragma once
#include "rowvec.h"

namespace flce {

struct EmbedArgs {
    const int64_t* tokens;
    int64_t first, ignored;   // the table's first token; the token whose rows are left out
    int rows, V, H;
    float scale;
    const void* in;           // forward: the table; backward: dY
    void* out;                // forward: the rows; backward: the table's gradient
    int64_t ldin, ldout;
    // backward
    int add;                  // to what the gradient's buffer holds
    int range;                // tokens per workgroup of the sort, a power of two
    int *begin;               // V + 1: entries in front of a token's
    int *token, *row;         // of the entries in order
    float* part;              // piece p: row 2 p its first token's sum if that began before, 2 p + 1 its last one's
    int slices;               // of 64 vectors, per row
};

// The row of the table that token t names, or -1.
__device__ __forceinline__ int embed_row(const EmbedArgs& a, int64_t t) {
    const uint64_t v = (uint64_t)t - (uint64_t)a.first;
    return t != a.ignored && v < (uint64_t)a.V ? (int)v : -1;
}

// LPR lanes per row, K loads of a lane in flight.  One wavefront per row where a row has 64 vectors or more.
template <typename T, int LPR, int K, bool NT>
__global__ __launch_bounds__(256) void embed_fwd_kernel(EmbedArgs a) {
    constexpr int N = RowVec<T>::N, ROWS = 256 / LPR;
    const int lane = threadIdx.x % LPR;
    const int nfull = a.H / N, rem = a.H % N, nvec = nfull + (rem ? 1 : 0);
    int64_t i = (int64_t)blockIdx.x * ROWS + threadIdx.x / LPR;
    if constexpr (LPR == WAVE) i = (int64_t)blockIdx.x * ROWS + __builtin_amdgcn_readfirstlane((int)threadIdx.x / LPR);
    for (; i < a.rows; i += (int64_t)gridDim.x * ROWS) {
        const int v = embed_row(a, a.tokens[i]);
        const T* from = static_cast<const T*>(a.in) + (int64_t)max(v, 0) * a.ldin;
        T* to = static_cast<T*>(a.out) + i * a.ldout;
        for (int j0 = 0; j0 < nvec; j0 += LPR * K) {
            u32x4 raw[K];
#pragma unroll
            for (int k = 0; k < K; ++k) raw[k] = row_load(from, j0 + lane + k * LPR, v < 0 ? 0 : nfull, v < 0 ? 0 : rem);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float f[N];
                RowVec<T>::unpack(raw[k], f);
#pragma unroll
                for (int e = 0; e < N; ++e) f[e] = v < 0 ? 0.f : f[e] * a.scale;
                row_store<T, NT>(to, j0 + lane + k * LPR, nfull, rem, f);
            }
        }
    }
}

constexpr int EM_SORT_THREADS = 1024, EM_SORT_WAVES = EM_SORT_THREADS / WAVE;
constexpr int EM_RANGE = 512;      // most tokens of a workgroup of the sort
constexpr int EM_PIECE = 32;       // entries that a wavefront adds up: with one on either side less than its lanes
constexpr int EM_AHEAD = 8;        // loads in flight, per lane
constexpr int EM_JOIN_THREADS = 512, EM_JOIN_WAVES = EM_JOIN_THREADS / WAVE;

// Wavefront w of a workgroup looks at the w-th part of the rows: twice, to count and to place.
template <typename T, bool NT>
__global__ __launch_bounds__(EM_SORT_THREADS) void embed_sort_kernel(EmbedArgs a) {
    constexpr int AHEAD = 8;
    __shared__ int count[EM_SORT_WAVES][EM_RANGE];   // later: the next entry of a wavefront's rows of a token
    __shared__ int total[EM_RANGE];
    __shared__ int wave_sum_of[EM_SORT_WAVES], before_of[EM_SORT_WAVES];
    const int tid = threadIdx.x, lane = tid % WAVE, wave = __builtin_amdgcn_readfirstlane(tid / WAVE);
    const int lo = (int)blockIdx.x * a.range, n = min(a.range, a.V - lo);
    for (int j = tid; j < EM_SORT_WAVES * EM_RANGE; j += EM_SORT_THREADS) (&count[0][0])[j] = 0;
    __syncthreads();
    const int share = ((a.rows + EM_SORT_WAVES - 1) / EM_SORT_WAVES + WAVE - 1) / WAVE * WAVE;
    const int64_t i0 = (int64_t)wave * share, i1 = min((int64_t)a.rows, i0 + share);
    int before = 0;
    for (int64_t i = i0; i < i1; i += AHEAD * WAVE) {
        int64_t t[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) t[k] = a.tokens[min(i + k * WAVE + lane, (int64_t)a.rows - 1)];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int v = i + k * WAVE + lane < i1 ? embed_row(a, t[k]) : -1;
            before += v >= 0 && v < lo;
            if (v >= lo && v < lo + n) atomicAdd(&count[wave][v - lo], 1);
        }
    }
    before = wave_sum(before);
    if (lane == 0) before_of[wave] = before;
    __syncthreads();
    // per token: where each wavefront's rows begin among them; then where the tokens begin
    int mine = 0;
    if (tid < EM_RANGE) {
#pragma unroll
        for (int w = 0; w < EM_SORT_WAVES; ++w) {
            const int c = count[w][tid];
            count[w][tid] = mine;
            mine += c;
        }
        total[tid] = mine;
    }
    int up_to = mine;   // inclusive sum over the wavefront's tokens
#pragma unroll
    for (int o = 1; o < WAVE; o <<= 1) {
        const int other = __shfl_up(up_to, o, WAVE);
        if (lane >= o) up_to += other;
    }
    if (lane == WAVE - 1) wave_sum_of[wave] = up_to;
    __syncthreads();
    int at = up_to - mine;
    for (int w = 0; w < EM_SORT_WAVES; ++w) {
        if (w < wave) at += wave_sum_of[w];
        at += before_of[w];
    }
    if (tid < EM_RANGE) {
        if (tid < n) a.begin[lo + tid] = at;
        if (tid == n - 1 && lo + n == a.V) a.begin[a.V] = at + mine;
#pragma unroll
        for (int w = 0; w < EM_SORT_WAVES; ++w) count[w][tid] += at;
    }
    __syncthreads();
    for (int64_t i = i0; i < i1; i += AHEAD * WAVE) {
        int64_t t[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) t[k] = a.tokens[min(i + k * WAVE + lane, (int64_t)a.rows - 1)];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int v = i + k * WAVE + lane < i1 ? embed_row(a, t[k]) : -1;
            const bool here = v >= lo && v < lo + n;
            uint64_t peers = __ballot(here);
            if (!peers) continue;
            // the lanes with the same token, bit by bit
#pragma unroll
            for (int b = 1; b < EM_RANGE; b <<= 1) {
                const bool set = (v - lo) & b;
                const uint64_t with = __ballot(set);
                peers &= set ? with : ~with;
            }
            const int rank = __popcll(peers & ((1ull << lane) - 1)), leader = __ffsll((unsigned long long)peers) - 1;
            int base = 0;
            if (here && rank == 0) base = atomicAdd(&count[wave][v - lo], __popcll(peers));
            base = __shfl(base, max(leader, 0), WAVE);
            if (here) {
                a.token[base + rank] = v;
                a.row[base + rank] = (int)(i + k * WAVE + lane);
            }
        }
    }
    if (a.add) return;
    constexpr int N = RowVec<T>::N;
    const int nfull = a.H / N, rem = a.H % N, nvec = nfull + (rem ? 1 : 0);
    const float zero[N] = {};
    for (int j = wave; j < n; j += EM_SORT_WAVES) {
        if (total[j]) continue;
        T* to = static_cast<T*>(a.out) + (int64_t)(lo + j) * a.ldout;
        for (int v = lane; v < nvec; v += WAVE) row_store<T, NT>(to, v, nfull, rem, zero);
    }
}

// Writes (or adds) the finished sum of vector v of a row of the table.
template <typename T, bool NT>
__device__ __forceinline__ void embed_put(const EmbedArgs& a, int token, int v, int nfull, int rem, const float (&sum)[RowVec<T>::N]) {
    constexpr int N = RowVec<T>::N;
    T* to = static_cast<T*>(a.out) + (int64_t)token * a.ldout;
    float f[N];
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = 0.f;
    if (a.add) RowVec<T>::unpack(row_load(to, v, nfull, rem), f);
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = a.add ? f[e] + a.scale * sum[e] : a.scale * sum[e];
    row_store<T, NT>(to, v, nfull, rem, f);
}

template <typename T, bool NT>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedArgs a) {
    constexpr int N = RowVec<T>::N;
    static_assert(EM_PIECE + 2 <= WAVE, "a lane per entry and one on either side");
    const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / WAVE);
    const int nfull = a.H / N, rem = a.H % N, nvec = nfull + (rem ? 1 : 0);
    const int entries = a.begin[a.V];
    const int64_t units = (int64_t)((entries + EM_PIECE - 1) / EM_PIECE) * a.slices;
    for (int64_t u = (int64_t)blockIdx.x * 4 + wave; u < units; u += (int64_t)gridDim.x * 4) {
        const int piece = (int)(u / a.slices), v = (int)(u % a.slices) * WAVE + lane;
        const int e0 = piece * EM_PIECE, count = min(EM_PIECE, entries - e0);
        // lane 1 + i holds entry i of the piece
        const int at = e0 - 1 + lane;
        const bool there = lane <= EM_PIECE + 1 && at >= 0 && at < entries;
        const int tokens = there ? a.token[at] : -1, rows = there ? a.row[at] : 0;
        float sum[N];
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] = 0.f;
        int token = __builtin_amdgcn_readlane(tokens, 1);
        bool began = __builtin_amdgcn_readlane(tokens, 0) != token;   // the token at hand began in this piece
        auto leave = [&](int which) {
            if (v >= nvec) return;
            float* to = a.part + ((int64_t)piece * 2 + which) * a.slices * (WAVE * N) + (int64_t)v * N;
#pragma unroll
            for (int e = 0; e < N; e += 4) *reinterpret_cast<f32x4*>(to + e) = f32x4{sum[e], sum[e + 1], sum[e + 2], sum[e + 3]};
        };
        for (int g = 0; g < count; g += EM_AHEAD) {
            u32x4 raw[EM_AHEAD];
#pragma unroll
            for (int k = 0; k < EM_AHEAD; ++k) {
                const int row = __builtin_amdgcn_readlane(rows, 1 + min(g + k, count - 1));
                const T* from = static_cast<const T*>(a.in) + (int64_t)row * a.ldin;
                raw[k] = a.H < N ? row_load(from, v, nfull, rem) : row_load_ahead(from, v, nvec, a.H);
            }
            if (rem && a.H >= N && v == nfull) {
#pragma unroll
                for (int k = 0; k < EM_AHEAD; ++k) row_shift_tail<T>(raw[k], rem);
            }
#pragma unroll
            for (int k = 0; k < EM_AHEAD; ++k) {
                if (g + k >= count) break;
                const int t = __builtin_amdgcn_readlane(tokens, 1 + g + k);
                if (t != token) {
                    if (began) embed_put<T, NT>(a, token, v, nfull, rem, sum);
                    else leave(0);
#pragma unroll
                    for (int e = 0; e < N; ++e) sum[e] = 0.f;
                    token = t;
                    began = true;
                }
                float f[N];
                RowVec<T>::unpack(raw[k], f);
#pragma unroll
                for (int e = 0; e < N; ++e) sum[e] += f[e];
            }
        }
        const bool ends = __builtin_amdgcn_readlane(tokens, 1 + count) != token;
        if (began && ends) embed_put<T, NT>(a, token, v, nfull, rem, sum);
        else leave(began ? 1 : 0);
    }
}

// A workgroup per piece and slice: adds up the sums of the token that begins in the piece and goes on behind it.
template <typename T, bool NT>
__global__ __launch_bounds__(EM_JOIN_THREADS) void embed_join_kernel(EmbedArgs a) {
    constexpr int N = RowVec<T>::N, AHEAD = 4;
    __shared__ double sums[EM_JOIN_WAVES][WAVE * N];
    const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / WAVE);
    const int nfull = a.H / N, rem = a.H % N, nvec = nfull + (rem ? 1 : 0);
    const int entries = a.begin[a.V];
    const int64_t units = (int64_t)((entries + EM_PIECE - 1) / EM_PIECE) * a.slices;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int piece = (int)(u / a.slices), slice = (int)(u % a.slices), v = slice * WAVE + lane;
        const int64_t next = ((int64_t)piece + 1) * EM_PIECE;
        if (next >= entries) continue;
        const int token = a.token[next];
        const int b = a.begin[token], e = a.begin[token + 1];
        if (b / EM_PIECE != piece || b == next) continue;   // it began elsewhere
        const int pieces = (e - 1) / EM_PIECE - piece + 1;
        const int64_t pitch = (int64_t)a.slices * (WAVE * N);
        const float* first = a.part + ((int64_t)piece * 2 + 1) * pitch + (int64_t)v * N;
        const float* rest = a.part + (int64_t)piece * 2 * pitch + (int64_t)v * N;
        double sum[N];
#pragma unroll
        for (int k = 0; k < N; ++k) sum[k] = 0.0;
        const int p0 = (int)((int64_t)pieces * wave / EM_JOIN_WAVES), p1 = (int)((int64_t)pieces * (wave + 1) / EM_JOIN_WAVES);
        if (v < nvec) {
            for (int p = p0; p < p1; p += AHEAD) {
                f32x4 in[AHEAD][N / 4];
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) {
                    const int q = min(p + k, p1 - 1);
                    const float* from = q ? rest + (int64_t)q * 2 * pitch : first;
#pragma unroll
                    for (int c = 0; c < N / 4; ++c) in[k][c] = *reinterpret_cast<const f32x4*>(from + 4 * c);
                }
#pragma unroll
                for (int k = 0; k < AHEAD; ++k)
#pragma unroll
                    for (int c = 0; c < N; ++c) sum[c] += p + k < p1 ? (double)in[k][c / 4][c % 4] : 0.0;
            }
        }
#pragma unroll
        for (int k = 0; k < N; ++k) sums[wave][k * WAVE + lane] = sum[k];
        __syncthreads();
        if (wave == 0 && v < nvec) {
            float f[N];
#pragma unroll
            for (int k = 0; k < N; ++k) {
                for (int w = 1; w < EM_JOIN_WAVES; ++w) sum[k] += sums[w][k * WAVE + lane];
                f[k] = (float)sum[k];
            }
            embed_put<T, NT>(a, token, v, nfull, rem, f);
        }
        __syncthreads();
    }
}

}  // namespace flce
