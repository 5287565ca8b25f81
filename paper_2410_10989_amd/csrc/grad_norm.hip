// C ABI of the gradient norm and clipping (see grad_norm.h): argument checks, chunks, launches.
#include "grad_norm.h"

#include <algorithm>
#include <new>

#include "flce_host.h"

using namespace flce;

namespace {

constexpr int64_t GN_MAX_COUNT = (int64_t)1 << 40;   // elements of one tensor
constexpr int64_t GN_CHUNK = 64 << 10, GN_CHUNK_MIN = 4 << 10;   // bytes: 16 and 1 accesses per thread
constexpr int GN_BLOCKS = 2048;        // workgroups of all launches of a sweep together: 8 per CU
constexpr int GN_BLOCKS_MIN = 64;      // of one launch

struct Tensors {
    const void* const* in;
    void* const* out;
    const int64_t* count;
    const int* dtype;
    int n;
};

int64_t launches_of(int64_t n) { return std::max<int64_t>(1, (n + GN_TENSORS - 1) / GN_TENSORS); }
int blocks_per_launch(int64_t n) { return (int)std::max<int64_t>(GN_BLOCKS_MIN, GN_BLOCKS / launches_of(n)); }
size_t partial_bytes(int64_t n) { return (size_t)launches_of(n) * blocks_per_launch(n) * sizeof(double); }
size_t bytes_of(const Tensors& t, int i) { return (size_t)t.count[i] * (t.dtype[i] == FLCE_F32 ? 4 : 2); }

int check_tensors(const Tensors& t) {
    if (t.n < 0) return FLCE_ERR_ARG;
    if (t.n && (!t.in || !t.count || !t.dtype)) return FLCE_ERR_NULL;
    for (int i = 0; i < t.n; ++i) {
        if (t.dtype[i] != FLCE_F32 && t.dtype[i] != FLCE_BF16) return FLCE_ERR_DTYPE;
        if (t.count[i] < 0 || t.count[i] > GN_MAX_COUNT) return FLCE_ERR_SHAPE;
        if (!t.count[i]) continue;
        const void* out = t.out ? t.out[i] : t.in[i];
        if (!t.in[i] || !out) return FLCE_ERR_NULL;
        const size_t es = t.dtype[i] == FLCE_F32 ? 4 : 2;
        if (!aligned(t.in[i], es) || !aligned(out, es)) return FLCE_ERR_ALIGN;
    }
    return FLCE_OK;
}

// No two outputs may share memory, and an output may only lie on an input that is its own, exactly.
int check_outputs(const Tensors& t) {
    struct Piece {
        uintptr_t begin, end;
        bool write;
    };
    Piece* pieces = new (std::nothrow) Piece[2 * (size_t)t.n + 1];
    if (!pieces) return FLCE_ERR_WORKSPACE;
    size_t k = 0;
    for (int i = 0; i < t.n; ++i) {
        if (!t.count[i]) continue;
        const void* out = t.out ? t.out[i] : t.in[i];
        const uintptr_t w = reinterpret_cast<uintptr_t>(out), r = reinterpret_cast<uintptr_t>(t.in[i]);
        pieces[k++] = {w, w + bytes_of(t, i), true};
        if (r != w) pieces[k++] = {r, r + bytes_of(t, i), false};
    }
    std::sort(pieces, pieces + k, [](const Piece& a, const Piece& b) { return a.begin < b.begin; });
    uintptr_t any_end = 0, write_end = 0;   // of the pieces so far
    int rc = FLCE_OK;
    for (size_t i = 0; i < k; ++i) {
        if (pieces[i].begin < (pieces[i].write ? any_end : write_end)) rc = FLCE_ERR_ARG;
        any_end = std::max(any_end, pieces[i].end);
        if (pieces[i].write) write_end = std::max(write_end, pieces[i].end);
    }
    delete[] pieces;
    return rc;
}

// The launch of tensors first .. (at most GN_TENSORS of them); blocks: its workgroups, 0 if there is nothing in them.
GnArgs launch_args(const Tensors& t, int first, int64_t chunk_bytes, int max_blocks, int* blocks) {
    GnArgs a{};
    int64_t chunks = 0;
    for (int i = first; i < t.n && i < first + GN_TENSORS; ++i) {
        if (!t.count[i]) continue;
        const int k = a.tensors++;
        a.in[k] = t.in[i];
        a.out[k] = t.out ? t.out[i] : const_cast<void*>(t.in[i]);
        a.count[k] = t.dtype[i] == FLCE_BF16 ? ~t.count[i] : t.count[i];
        chunks += ((int64_t)bytes_of(t, i) + chunk_bytes - 1) / chunk_bytes;
        a.first_chunk[k + 1] = (int)chunks;
    }
    a.chunk_bytes = (int)chunk_bytes;
    *blocks = (int)std::min<int64_t>(chunks, max_blocks);
    return a;
}

// Chunks as long as they may be while there are enough of them for every workgroup.
int64_t chunk_bytes_of(const Tensors& t) {
    size_t total = 0;
    for (int i = 0; i < t.n; ++i) total += bytes_of(t, i);
    int64_t c = GN_CHUNK;
    while (c > GN_CHUNK_MIN && total / (size_t)c < (size_t)GN_BLOCKS) c /= 2;
    // (a launch counts its chunks in 32 bits)
    while (total / (size_t)c > ((size_t)1 << 30)) c *= 2;
    return c;
}

int partial_memory(const Tensors& t, void* workspace, size_t workspace_bytes, double** out) {
    const size_t need = partial_bytes(t.n);
    if (workspace) {
        if (!aligned(workspace, 256)) return FLCE_ERR_ALIGN;
        if (workspace_bytes < need) return FLCE_ERR_WORKSPACE;
        *out = static_cast<double*>(workspace);
        return FLCE_OK;
    }
    char* ws = nullptr;
    FLCE_TRY(shared_workspace(need, &ws));
    *out = reinterpret_cast<double*>(ws);
    return FLCE_OK;
}

// Sweep 1; *partials: the results it leaves.
template <typename Op>
int sweep_norm(const Tensors& t, int64_t chunk_bytes, double* partial, int* partials, hipStream_t s) {
    const int max_blocks = blocks_per_launch(t.n);
    *partials = 0;
    for (int first = 0; first < t.n; first += GN_TENSORS) {
        int blocks;
        GnArgs a = launch_args(t, first, chunk_bytes, max_blocks, &blocks);
        if (!blocks) continue;
        a.partial = partial + *partials;
        hipLaunchKernelGGL((grad_norm_kernel<Op>), dim3((unsigned)blocks), dim3(GN_THREADS), 0, s, a);
        HIP_TRY(hipGetLastError());
        *partials += blocks;
    }
    return FLCE_OK;
}

// Sweep 2, the last tensors first.  The norm is given, or added up from the partial results and stored.
template <typename Op>
int sweep_scale(const Tensors& t, int64_t chunk_bytes, const double* partial, int partials, const float* norm_in,
                float* norm_out, float max_norm, hipStream_t s) {
    const int max_blocks = blocks_per_launch(t.n);
    for (int64_t l = launches_of(t.n) - 1; l >= 0; --l) {
        int blocks;
        GnArgs a = launch_args(t, (int)(l * GN_TENSORS), chunk_bytes, max_blocks, &blocks);
        if (!blocks && !norm_out) continue;
        a.partial = const_cast<double*>(partial);
        a.partials = partials;
        a.norm_in = norm_in;
        a.norm_out = norm_out;
        a.max_norm = max_norm;
        norm_out = nullptr;   // (one launch stores it)
        hipLaunchKernelGGL((grad_scale_kernel<Op>), dim3((unsigned)std::max(1, blocks)), dim3(GN_THREADS), 0, s, a);
        HIP_TRY(hipGetLastError());
    }
    return FLCE_OK;
}

template <typename Op>
int run_norm(const Tensors& t, double* partial, float* norm, hipStream_t s) {
    int partials;
    FLCE_TRY(sweep_norm<Op>(t, chunk_bytes_of(t), partial, &partials, s));
    hipLaunchKernelGGL((grad_norm_final_kernel<Op>), dim3(1), dim3(GN_THREADS), 0, s, partial, partials, norm);
    HIP_TRY(hipGetLastError());
    return FLCE_OK;
}
template <typename Op>
int run_clip(const Tensors& t, double* partial, float max_norm, float* norm, hipStream_t s) {
    int partials;
    const int64_t chunk_bytes = chunk_bytes_of(t);
    FLCE_TRY(sweep_norm<Op>(t, chunk_bytes, partial, &partials, s));
    return sweep_scale<Op>(t, chunk_bytes, partial, partials, nullptr, norm, max_norm, s);
}

bool finite_not_negative(float v) { return v >= 0.0f && v - v == 0.0f; }

}  // namespace

extern "C" {

size_t flce_grad_norm_workspace_bytes(int n_tensors) { return n_tensors < 0 ? 0 : partial_bytes(n_tensors); }

int flce_grad_norm(const void* const* grads, const int64_t* counts, const int* dtypes, int n_tensors, int norm_type,
                   float* norm, void* workspace, size_t workspace_bytes, void* stream) {
    const Tensors t{grads, nullptr, counts, dtypes, n_tensors};
    FLCE_TRY(check_tensors(t));
    if (!norm) return FLCE_ERR_NULL;
    if (!aligned(norm, 4)) return FLCE_ERR_ALIGN;
    if (norm_type != FLCE_NORM_2 && norm_type != FLCE_NORM_INF) return FLCE_ERR_ARG;
    double* partial;
    FLCE_TRY(partial_memory(t, workspace, workspace_bytes, &partial));
    hipStream_t s = static_cast<hipStream_t>(stream);
    return norm_type == FLCE_NORM_2 ? run_norm<GnSumSq>(t, partial, norm, s) : run_norm<GnMax>(t, partial, norm, s);
}

int flce_grad_clip(const void* const* grads, void* const* outs, const int64_t* counts, const int* dtypes, int n_tensors,
                   const float* norm, float max_norm, void* stream) {
    const Tensors t{grads, outs, counts, dtypes, n_tensors};
    FLCE_TRY(check_tensors(t));
    if (!norm) return FLCE_ERR_NULL;
    if (!aligned(norm, 4)) return FLCE_ERR_ALIGN;
    if (!finite_not_negative(max_norm)) return FLCE_ERR_ARG;
    FLCE_TRY(check_outputs(t));
    return sweep_scale<GnSumSq>(t, chunk_bytes_of(t), nullptr, 0, norm, nullptr, max_norm, static_cast<hipStream_t>(stream));
}

int flce_clip_grad_norm(const void* const* grads, void* const* outs, const int64_t* counts, const int* dtypes,
                        int n_tensors, int norm_type, float max_norm, float* norm, void* workspace,
                        size_t workspace_bytes, void* stream) {
    const Tensors t{grads, outs, counts, dtypes, n_tensors};
    FLCE_TRY(check_tensors(t));
    if (!norm) return FLCE_ERR_NULL;
    if (!aligned(norm, 4)) return FLCE_ERR_ALIGN;
    if ((norm_type != FLCE_NORM_2 && norm_type != FLCE_NORM_INF) || !finite_not_negative(max_norm)) return FLCE_ERR_ARG;
    FLCE_TRY(check_outputs(t));
    double* partial;
    FLCE_TRY(partial_memory(t, workspace, workspace_bytes, &partial));
    hipStream_t s = static_cast<hipStream_t>(stream);
    return norm_type == FLCE_NORM_2 ? run_clip<GnSumSq>(t, partial, max_norm, norm, s)
                                    : run_clip<GnMax>(t, partial, max_norm, norm, s);
}

}  // extern "C"
