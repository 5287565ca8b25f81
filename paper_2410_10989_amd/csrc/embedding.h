// Embedding lookup with scaling, and the gradient of the table.  With t_i the token of row i counted from the table's
// first one, live rows those whose t_i is a row of the table and not the ignored token,
//
//     out_i = s E[t_i]   (0 for rows that are not live)          dE_v = (dE_v +) s sum_{i live, t_i = v} dY_i
//
// The gradient's rows are added up in the order of i, whatever the machine does: no atomics on values.
//   1. embed_sort_kernel    the live rows' numbers, those of a token together and in order (a stable counting sort), in one
//                           launch: a workgroup owns every `classes`-th token and looks at all rows, so it counts what
//                           lies before its tokens itself and waits for nobody.  (Neighbouring tokens belong to different
//                           workgroups: the frequent ones are neighbours.  With 512 tokens in a row for each, the first
//                           workgroup had half of 16384 rows to place, 28 us; 10 so.)
//   2. embed_sum_kernel     pieces of consecutive entries of that order, a wavefront per piece and 64 vectors of the row:
//                           the same work for everybody, however often a token comes.  What begins and ends in a
//                           piece is written at once, the rest is left as fp32 sums.  Further workgroups fill the rows
//                           of the table that no token names with zeros.
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
    int classes, class_bits;  // workgroup c of the sort has tokens c, c + classes, ...; a power of two
    int per_class;            // tokens of a class
    int piece;                // entries per piece, a power of two
    int2* span;               // per token, in the order of embed_key: its entries' first and the one behind its last
    int* total;               // entries
    int2* entry;              // (token, row), the tokens in the order of embed_key
    int sum_blocks;           // workgroups of the second launch that add up; the others write zeros
    int zero_rows;            // rows of the table per wavefront of these, at most its lanes
    float* part;              // piece p: row 2 p its first token's sum if that began before, 2 p + 1 its last one's
    int slices;               // of 64 vectors, per row
};

// The row of the table that token t names, or -1.
__device__ __forceinline__ int embed_row(const EmbedArgs& a, int64_t t) {
    const uint64_t v = (uint64_t)t - (uint64_t)a.first;
    return t != a.ignored && t >= a.first && v < (uint64_t)a.V ? (int)v : -1;
}

__device__ __forceinline__ int embed_key(const EmbedArgs& a, int v) { return (v & (a.classes - 1)) * a.per_class + (v >> a.class_bits); }

// LPR lanes per row, K loads of a lane in flight.  One wavefront per row where a row has 64 vectors or more.  Bound by HBM: 16384
// rows of 3584 bf16 38 us, 4.4 TB/s (a row's address waits for its token, and the stores for the row).
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
constexpr int EM_RANGE = 1024;     // most tokens of a class: one per thread
constexpr int EM_LIST = 1024;      // rows of its class that a wavefront of the sort lists
constexpr int EM_PIECE = 32;       // most entries that a wavefront adds up: with one on either side less than its lanes
constexpr int EM_PIECE_MIN = 8;
constexpr int EM_JOIN_PIECES = 2;  // that a workgroup looks at
constexpr int EM_AHEAD = 8;        // loads in flight, per lane
constexpr int EM_JOIN_THREADS = 256, EM_JOIN_WAVES = EM_JOIN_THREADS / WAVE;

// Wavefront w of a workgroup looks at the w-th part of the rows, 16 x 64 of them at a time with the next ones' loads under
// way, and keeps a list of those of its class; the list is then put in order.  Only a wavefront with more than EM_LIST of them
// looks at its rows again, a list for every 1024.  (us, rows dealt by Zipf's law: 16384 10, 32768 15, 131072 45; before the
// lists, every row looked at twice, 21 for 16384 and over 100 for 131072.)
static __global__ __launch_bounds__(EM_SORT_THREADS) void embed_sort_kernel(EmbedArgs a) {
    constexpr int AHEAD = 16;
    __shared__ int count[EM_SORT_WAVES][EM_RANGE];   // later: the next entry of a wavefront's rows of a token
    __shared__ uint32_t list[EM_SORT_WAVES][EM_LIST];   // row, counted from the wavefront's first, and token of the class
    __shared__ int wave_sum_of[EM_SORT_WAVES], before_of[EM_SORT_WAVES];
    const int tid = threadIdx.x, lane = tid % WAVE, wave = __builtin_amdgcn_readfirstlane(tid / WAVE);
    const int mask = a.classes - 1, c = (int)blockIdx.x;
    const uint64_t below = (1ull << lane) - 1;
    const int share = ((a.rows + EM_SORT_WAVES - 1) / EM_SORT_WAVES + WAVE - 1) / WAVE * WAVE;
    const int64_t i0 = (int64_t)wave * share, i1 = min((int64_t)a.rows, i0 + share);
    const int listed = (int64_t)share * EM_RANGE <= ((int64_t)1 << 32) ? EM_LIST : 0;   // (an entry has 32 bits)
    int64_t t[AHEAD];
    auto load = [&](int64_t i) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) t[k] = a.tokens[min(i + k * WAVE + lane, (int64_t)a.rows - 1)];
    };
    load(i0);
    for (int j = lane; j < a.per_class; j += WAVE) count[wave][j] = 0;   // (its own: no barrier)
    int before = 0, mine_all = 0;   // rows before the class's, of the class
    for (int64_t i = i0; i < i1; i += AHEAD * WAVE) {
        int v[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) v[k] = i + k * WAVE + lane < i1 ? embed_row(a, t[k]) : -1;
        if (i + AHEAD * WAVE < i1) load(i + AHEAD * WAVE);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int of = v[k] >= 0 ? v[k] & mask : INT32_MAX;
            before += __popcll(__ballot(of < c));
            const uint64_t here = __ballot(of == c);
            if (!here) continue;
            if (of == c) {
                const int at = mine_all + __popcll(here & below), which = v[k] >> a.class_bits;
                atomicAdd(&count[wave][which], 1);
                if (at < listed) list[wave][at] = (uint32_t)(i - i0 + k * WAVE + lane) * EM_RANGE + which;
            }
            mine_all += __popcll(here);
        }
    }
    if (lane == 0) before_of[wave] = before;
    __syncthreads();
    // per token: where each wavefront's rows begin among them; then where the tokens begin
    int mine = 0;
    static_assert(EM_RANGE == EM_SORT_THREADS, "a token per thread");
    if (tid < a.per_class) {
#pragma unroll
        for (int w = 0; w < EM_SORT_WAVES; ++w) {
            const int here = count[w][tid];
            count[w][tid] = mine;
            mine += here;
        }
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
    if (tid < a.per_class) {
        a.span[c * (int64_t)a.per_class + tid] = int2{at, at + mine};
#pragma unroll
        for (int w = 0; w < EM_SORT_WAVES; ++w) count[w][tid] += at;
    }
    if (tid == EM_SORT_THREADS - 1 && c == mask) *a.total = at + mine;
    __syncthreads();
    // up to 64 rows of the class, in order, each with its token's number in it (or not `here`): to their places
    auto place = [&](bool here, int which, int row) {
        uint64_t peers = __ballot(here);
        // the lanes with the same token, bit by bit
        for (int b = 1; b < a.per_class; b <<= 1) {
            const bool set = which & b;
            const uint64_t with = __ballot(set);
            peers &= set ? with : ~with;
        }
        const int rank = __popcll(peers & below), leader = __ffsll((unsigned long long)peers) - 1;
        int base = 0;
        if (here && rank == 0) base = atomicAdd(&count[wave][which], __popcll(peers));
        base = __shfl(base, max(leader, 0), WAVE);
        if (here) a.entry[base + rank] = int2{(which << a.class_bits) | c, row};
    };
    auto place_list = [&](int n, int64_t first) {
        for (int j = 0; j < n; j += WAVE) {
            const bool here = j + lane < n;
            const uint32_t e = list[wave][here ? j + lane : 0];
            place(here, here ? (int)(e % EM_RANGE) : 0, (int)(first + e / EM_RANGE));
        }
    };
    if (mine_all <= listed) {
        place_list(mine_all, i0);
        return;
    }
    static_assert(AHEAD * WAVE <= EM_LIST, "a round's rows fit the list");
    for (int64_t i = i0; i < i1; i += AHEAD * WAVE) {
        load(i);
        int n = 0;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int v = i + k * WAVE + lane < i1 ? embed_row(a, t[k]) : -1;
            const uint64_t here = __ballot(v >= 0 && (v & mask) == c);
            if (v >= 0 && (v & mask) == c) list[wave][n + __popcll(here & below)] = (uint32_t)(k * WAVE + lane) * EM_RANGE + (v >> a.class_bits);
            n += __popcll(here);
        }
        // (lanes read what others of the wavefront wrote: LDS executes a wavefront's accesses in order)
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        place_list(n, i);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

// Writes (or adds to `base`, what it holds) the finished sum of vector v of a row of the table.
template <typename T>
__device__ __forceinline__ void embed_put(const EmbedArgs& a, int token, int v, int nfull, int rem, const float (&sum)[RowVec<T>::N],
                                          const u32x4& base) {
    constexpr int N = RowVec<T>::N;
    T* to = static_cast<T*>(a.out) + (int64_t)token * a.ldout;
    float f[N];
    RowVec<T>::unpack(base, f);
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = a.add ? f[e] + a.scale * sum[e] : a.scale * sum[e];
    row_store<T, false>(to, v, nfull, rem, f);
}

// Bound by HBM where the whole gradient is written: 16384 rows of 4096 bf16 into 128256, 1.19 GB, 203 to 229 us.
// ADD: a.add.  What finished sums are added to is loaded with the rows of a group, not when a sum is finished (5734 rows
// of 2304, most tokens once or twice: a wait for memory after another, 37 us; 13 so).
template <typename T, bool ADD>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedArgs a) {
    constexpr int N = RowVec<T>::N;
    static_assert(EM_PIECE + 2 <= WAVE, "a lane per entry and one on either side");
    const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / WAVE);
    const int nfull = a.H / N, rem = a.H % N, nvec = nfull + (rem ? 1 : 0);
    if constexpr (!ADD) {
        // zeros: a stretch of zero_rows rows of the table per wavefront, plain stores (what that reaches with nothing else to
        // do: 1.05 GB 172 us, 176 nontemporal; rows dealt round-robin 190 to 205)
        if ((int)blockIdx.x >= a.sum_blocks) {
            const float zero[N] = {};
            const int64_t v0 = (((int64_t)blockIdx.x - a.sum_blocks) * 4 + wave) * a.zero_rows;
            const int2 span = a.span[embed_key(a, (int)min(v0 + lane, (int64_t)a.V - 1))];   // (a lane looks at a row)
            uint64_t empty = __ballot(lane < a.zero_rows && v0 + lane < a.V && span.x == span.y);
            while (empty) {
                const int r = __ffsll((unsigned long long)empty) - 1;
                empty &= empty - 1;
                T* to = static_cast<T*>(a.out) + (v0 + r) * a.ldout;
                for (int v = lane; v < nvec; v += WAVE) row_store<T, false>(to, v, nfull, rem, zero);
            }
            return;
        }
    }
    const int entries = *a.total;
    const int64_t units = (int64_t)((entries + a.piece - 1) / a.piece) * a.slices;
    for (int64_t u = (int64_t)blockIdx.x * 4 + wave; u < units; u += (int64_t)a.sum_blocks * 4) {
        const int piece = (int)(u / a.slices), v = (int)(u % a.slices) * WAVE + lane;
        const int e0 = piece * a.piece, count = min(a.piece, entries - e0);
        // lane 1 + i holds entry i of the piece
        const int at = e0 - 1 + lane;
        const bool there = lane <= a.piece + 1 && at >= 0 && at < entries;
        const int2 mine = there ? a.entry[at] : int2{-1, 0};
        const int tokens = mine.x, rows = mine.y;
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
        auto finish = [&](bool whole, const u32x4& base) {   // the token's entries end here, or the piece does
            if (began && whole) embed_put<T>(a, token, v, nfull, rem, sum, base);
            else leave(began ? 1 : 0);
        };
        for (int g = 0; g < count; g += EM_AHEAD) {
            u32x4 raw[EM_AHEAD], base[ADD ? EM_AHEAD : 1];
            int next[EM_AHEAD];   // the token behind entry g + k
#pragma unroll
            for (int k = 0; k < EM_AHEAD; ++k) {
                const int i = min(g + k, count - 1);
                const T* from = static_cast<const T*>(a.in) + (int64_t)__builtin_amdgcn_readlane(rows, 1 + i) * a.ldin;
                raw[k] = a.H < N ? row_load(from, v, nfull, rem) : row_load_ahead(from, v, nvec, a.H);
                next[k] = __builtin_amdgcn_readlane(tokens, 2 + i);
                if constexpr (ADD) {
                    const int t = __builtin_amdgcn_readlane(tokens, 1 + i);
                    const T* to = static_cast<const T*>(a.out) + (int64_t)t * a.ldout;
                    base[k] = u32x4{0u, 0u, 0u, 0u};
                    if (next[k] != t) base[k] = a.H < N ? row_load(to, v, nfull, rem) : row_load_ahead(to, v, nvec, a.H);
                }
            }
            if (rem && a.H >= N && v == nfull) {
#pragma unroll
                for (int k = 0; k < EM_AHEAD; ++k) {
                    row_shift_tail<T>(raw[k], rem);
                    if constexpr (ADD) row_shift_tail<T>(base[k], rem);
                }
            }
#pragma unroll
            for (int k = 0; k < EM_AHEAD; ++k) {
                if (g + k >= count) break;
                float f[N];
                RowVec<T>::unpack(raw[k], f);
#pragma unroll
                for (int e = 0; e < N; ++e) sum[e] += f[e];
                const bool whole = next[k] != token;
                if (whole || g + k == count - 1) {
                    finish(whole, base[ADD ? k : 0]);
#pragma unroll
                    for (int e = 0; e < N; ++e) sum[e] = 0.f;
                    token = next[k];
                    began = true;
                }
            }
        }
    }
}

// A workgroup per slice and EM_JOIN_PIECES pieces: adds up the sums of the tokens that begin in these and go on behind
// them.
template <typename T>
__global__ __launch_bounds__(EM_JOIN_THREADS) void embed_join_kernel(EmbedArgs a) {
    constexpr int N = RowVec<T>::N, AHEAD = 4;
    __shared__ double sums[EM_JOIN_WAVES][WAVE * N];
    const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / WAVE);
    const int nfull = a.H / N, rem = a.H % N, nvec = nfull + (rem ? 1 : 0);
    const int entries = *a.total;
    const int64_t groups = ((entries + a.piece - 1) / a.piece + EM_JOIN_PIECES - 1) / EM_JOIN_PIECES;
    for (int64_t u = blockIdx.x; u < groups * a.slices; u += gridDim.x) {
        const int piece0 = (int)(u / a.slices) * EM_JOIN_PIECES, v = (int)(u % a.slices) * WAVE + lane;
        // lane i looks at piece i: the token behind it is its last one's, and that began in it
        const int64_t e0 = (int64_t)(piece0 + lane) * a.piece, e1 = e0 + a.piece;
        const bool there = lane < EM_JOIN_PIECES && e1 < entries;
        const int behind = there ? a.entry[e1].x : -1, last = there ? a.entry[e1 - 1].x : -2;
        const int in_front = there && e0 > 0 ? a.entry[e0 - 1].x : -1;
        uint64_t crossed = __ballot(behind == last && in_front != behind);
        while (crossed) {
            const int which = __ffsll((unsigned long long)crossed) - 1;
            crossed &= crossed - 1;
            const int piece = piece0 + which, token = __builtin_amdgcn_readlane(behind, which);
            const int pieces = (a.span[embed_key(a, token)].y - 1) / a.piece - piece + 1;
            const int64_t pitch = (int64_t)a.slices * (WAVE * N);
            const float* first = a.part + ((int64_t)piece * 2 + 1) * pitch + (int64_t)v * N;
            const float* rest = a.part + (int64_t)piece * 2 * pitch + (int64_t)v * N;
            u32x4 base = {0u, 0u, 0u, 0u};
            if (a.add && wave == 0) base = row_load(static_cast<const T*>(a.out) + (int64_t)token * a.ldout, v, nfull, rem);
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
                embed_put<T>(a, token, v, nfull, rem, f, base);
            }
            __syncthreads();
        }
    }
}

}  // namespace flce
