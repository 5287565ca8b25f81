// C ABI of the embedding lookup and its gradient (see embedding.h): argument checks, workspace, launches.
#include "embedding.h"

#include <algorithm>

#include "flce_host.h"

using namespace flce;

namespace {

constexpr int64_t EM_MAX_H = (int64_t)1 << 24;      // keeps vector numbers within 32 bits
constexpr int64_t EM_GRID = (int64_t)1 << 20;       // workgroups of a launch; they go on in strides
// Workgroups of the sort, while each has this many tokens of the table (us with 256 and with 64: 16384 rows of 1024 43.0 and
// 44.5, 512 of 4096 18.0 and 18.9, but 256 of 512 14.5 and 13.8).
constexpr int EM_CUS = 256, EM_RANGE_MIN = 32;
// Wavefronts of the sums, if there is as much to add up: pieces of 32 entries while there are, then of 16 and 8.  us so, with
// pieces of 32 alone and of 8 alone: 5734 rows of 2304 29.7, 33.7, 29.7; 512 of 4096 18.0, 27.7, 17.8; 16384 of 4096
// into a gradient of their own 249.5, 249.0, 260.6.
constexpr int64_t EM_WAVES = 4096;
// Bytes of zeros that a wavefront fills.  us with 4, 8, 16 and 32 KB: 8192 rows into 256000 of 2304 bf16 229.7, 229.8, 244.8,
// 246.6; 1024 into 256000 of 256 37.5, 37.0, 39.1, 43.5; 16384 into 128256 of 4096 244.7, 244.6, 248.3, 249.8.
constexpr int64_t EM_ZERO_BYTES = 8 << 10;
constexpr int64_t EM_CACHE_BYTES = (int64_t)256 << 20;   // memory-side cache

size_t elem(int dtype) { return dtype == FLCE_F32 ? 4 : 2; }
int64_t align64(int64_t n) { return (n + 63) / 64 * 64; }

int check_common(const flce_embedding* b) {
    if (!b) return FLCE_ERR_NULL;
    if (b->size != sizeof(flce_embedding)) return FLCE_ERR_ARG;
    if (b->dtype != FLCE_F32 && b->dtype != FLCE_BF16) return FLCE_ERR_DTYPE;
    if (b->rows < 1 || b->rows > MAX_DIM || b->V < 1 || b->V > MAX_DIM || b->H < 1 || b->H > EM_MAX_H) return FLCE_ERR_SHAPE;
    if (b->scale - b->scale != 0.0f) return FLCE_ERR_ARG;
    if (b->ldtable && b->V > 1 && (b->ldtable < b->H || b->ldtable > MAX_DIM * 4)) return FLCE_ERR_SHAPE;
    if (b->ldrows && b->rows > 1 && (b->ldrows < b->H || b->ldrows > MAX_DIM * 4)) return FLCE_ERR_SHAPE;
    return FLCE_OK;
}
int64_t table_stride(const flce_embedding& b) { return b.ldtable && b.V > 1 ? b.ldtable : b.H; }
int64_t rows_stride(const flce_embedding& b) { return b.ldrows && b.rows > 1 ? b.ldrows : b.H; }

// How the sort deals the tokens, and where the order and the partial sums lie, in bytes from the workspace's start.
struct Plan {
    int class_bits;
    int64_t per_class, slices, piece, pieces;
    size_t span, entry, part, total;
};
Plan plan_of(const flce_embedding& b) {
    const int64_t N = 16 / (int64_t)elem(b.dtype);
    Plan p{};
    while ((b.V - 1) >> p.class_bits >= EM_RANGE || ((int64_t)1 << p.class_bits < EM_CUS && (b.V - 1) >> p.class_bits >= EM_RANGE_MIN)) ++p.class_bits;
    p.per_class = ((b.V - 1) >> p.class_bits) + 1;
    p.slices = ((b.H + N - 1) / N + WAVE - 1) / WAVE;
    // (pieces as long as they may be while there are enough wavefronts to fill the chip)
    p.piece = EM_PIECE;
    while (p.piece > EM_PIECE_MIN && b.rows / p.piece * p.slices < EM_WAVES) p.piece /= 2;
    p.pieces = (b.rows + p.piece - 1) / p.piece;
    p.span = 256;
    p.entry = p.span + (size_t)align64(p.per_class << p.class_bits) * sizeof(int2);
    p.part = p.entry + (size_t)align64(b.rows) * sizeof(int2);
    p.total = p.part + (p.pieces > 1 ? (size_t)p.pieces * 2 * (size_t)(p.slices * WAVE * N) * sizeof(float) : 0);
    return p;
}

EmbedArgs args_of(const flce_embedding& b, const int64_t* tokens) {
    EmbedArgs a{};
    a.tokens = tokens;
    a.first = b.first_token;
    a.ignored = b.ignore_index;
    a.rows = (int)b.rows;
    a.V = (int)b.V;
    a.H = (int)b.H;
    a.scale = b.scale;
    return a;
}

template <typename T, int LPR, int K>
void launch_fwd(const EmbedArgs& a, bool nt, hipStream_t s) {
    constexpr int ROWS = 256 / LPR;
    const dim3 grid((unsigned)std::min<int64_t>(EM_GRID, ((int64_t)a.rows + ROWS - 1) / ROWS));
    if (nt) hipLaunchKernelGGL((embed_fwd_kernel<T, LPR, K, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((embed_fwd_kernel<T, LPR, K, false>), grid, dim3(256), 0, s, a);
}
template <typename T>
int run_fwd(const EmbedArgs& a, bool nt, hipStream_t s) {
    const int64_t nvec = ((int64_t)a.H + RowVec<T>::N - 1) / RowVec<T>::N;
    if (nvec <= 16) launch_fwd<T, 16, 1>(a, nt, s);
    else if (nvec <= 64) launch_fwd<T, 64, 1>(a, nt, s);
    else if (nvec <= 256) launch_fwd<T, 64, 4>(a, nt, s);
    else launch_fwd<T, 64, 8>(a, nt, s);
    HIP_TRY(hipGetLastError());
    return FLCE_OK;
}
template <typename T>
int run_bwd(EmbedArgs& a, const Plan& p, hipStream_t s) {
    hipLaunchKernelGGL(embed_sort_kernel, dim3((unsigned)a.classes), dim3(EM_SORT_THREADS), 0, s, a);
    HIP_TRY(hipGetLastError());
    const int64_t units = p.pieces * p.slices;
    a.sum_blocks = (int)std::min(EM_GRID, (units + 3) / 4);
    if (a.add) {
        hipLaunchKernelGGL((embed_sum_kernel<T, true>), dim3((unsigned)a.sum_blocks), dim3(256), 0, s, a);
    } else {
        a.zero_rows = (int)std::max<int64_t>(1, std::min<int64_t>(WAVE, EM_ZERO_BYTES / ((int64_t)a.H * (int64_t)sizeof(T))));
        const int64_t zeros = ((int64_t)a.V + 4 * a.zero_rows - 1) / (4 * a.zero_rows);
        hipLaunchKernelGGL((embed_sum_kernel<T, false>), dim3((unsigned)(a.sum_blocks + zeros)), dim3(256), 0, s, a);
    }
    HIP_TRY(hipGetLastError());
    if (p.pieces == 1) return FLCE_OK;
    const int64_t groups = (p.pieces + EM_JOIN_PIECES - 1) / EM_JOIN_PIECES;
    hipLaunchKernelGGL((embed_join_kernel<T>), dim3((unsigned)std::min(EM_GRID, groups * p.slices)), dim3(EM_JOIN_THREADS), 0, s, a);
    HIP_TRY(hipGetLastError());
    return FLCE_OK;
}

}  // namespace

extern "C" {

int flce_embedding_fwd(const void* table, const int64_t* tokens, const flce_embedding* args, void* out, void* stream) {
    FLCE_TRY(check_common(args));
    const flce_embedding& b = *args;
    if (!table || !tokens || !out) return FLCE_ERR_NULL;
    const size_t es = elem(b.dtype);
    if (!aligned(table, es) || !aligned(out, es) || !aligned(tokens, 8)) return FLCE_ERR_ALIGN;
    const Span to = span(out, rows_stride(b), b.rows, b.H, es);
    if (overlap(to, span(table, table_stride(b), b.V, b.H, es)) || overlap(to, span(tokens, b.rows, 1, b.rows, 8)))
        return FLCE_ERR_ARG;
    EmbedArgs a = args_of(b, tokens);
    a.in = table;
    a.out = out;
    a.ldin = table_stride(b);
    a.ldout = rows_stride(b);
    // Nontemporal stores where the rows do not fit the memory-side cache anyway: whoever reads them next would miss them
    // there.  us, ordinary / nontemporal, rows of 3584 bf16 alone and with the layer norm that follows: 8192 19 / 16, 41 /
    // 44; 16384 38 / 30, 76 / 80; 24576 54 / 44, 102 / 110.
    const bool nt = b.rows * b.H * (int64_t)es > EM_CACHE_BYTES;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return b.dtype == FLCE_F32 ? run_fwd<float>(a, nt, s) : run_fwd<bf16_t>(a, nt, s);
}

int flce_embedding_bwd(const void* dout, const int64_t* tokens, const flce_embedding* args, void* dtable, void* stream) {
    FLCE_TRY(check_common(args));
    const flce_embedding& b = *args;
    if (!dout || !tokens || !dtable) return FLCE_ERR_NULL;
    if (b.accumulate != 0 && b.accumulate != 1) return FLCE_ERR_ARG;
    const size_t es = elem(b.dtype);
    if (!aligned(dout, es) || !aligned(dtable, es) || !aligned(tokens, 8)) return FLCE_ERR_ALIGN;
    const Span to = span(dtable, table_stride(b), b.V, b.H, es), from = span(dout, rows_stride(b), b.rows, b.H, es);
    const Span which = span(tokens, b.rows, 1, b.rows, 8);
    if (overlap(to, from) || overlap(to, which)) return FLCE_ERR_ARG;
    const Plan p = plan_of(b);
    char* ws = static_cast<char*>(b.workspace);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (ws) {
        if (!aligned(ws, 256)) return FLCE_ERR_ALIGN;
        if (b.workspace_bytes < p.total) return FLCE_ERR_WORKSPACE;
    } else {
        FLCE_TRY(shared_workspace(p.total, &ws, s));
    }
    const Span scratch{ws, p.total, p.total, 1};
    if (overlap(scratch, to) || overlap(scratch, from) || overlap(scratch, which)) return FLCE_ERR_ARG;
    EmbedArgs a = args_of(b, tokens);
    a.in = dout;
    a.out = dtable;
    a.ldin = rows_stride(b);
    a.ldout = table_stride(b);
    a.add = b.accumulate;
    a.class_bits = p.class_bits;
    a.classes = 1 << p.class_bits;
    a.per_class = (int)p.per_class;
    a.total = reinterpret_cast<int*>(ws);
    a.span = reinterpret_cast<int2*>(ws + p.span);
    a.entry = reinterpret_cast<int2*>(ws + p.entry);
    a.part = reinterpret_cast<float*>(ws + p.part);
    a.piece = (int)p.piece;
    a.slices = (int)p.slices;
    return b.dtype == FLCE_F32 ? run_bwd<float>(a, p, s) : run_bwd<bf16_t>(a, p, s);
}

size_t flce_embedding_workspace_bytes(const flce_embedding* args) {
    return check_common(args) == FLCE_OK ? plan_of(*args).total : 0;
}

}  // extern "C"
