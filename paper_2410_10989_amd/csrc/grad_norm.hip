// C ABI of the gradient norm and clipping (see grad_norm.h): argument checks, chunks, launches.
#include "grad_norm.h"

#include <algorithm>
#include <new>

#include "flce_host.h"

using namespace flce;

namespace {

constexpr int64_t GN_MAX_COUNT = (int64_t)1 << 40;   // elements of one tensor
constexpr int64_t GN_CHUNK = 32 << 10, GN_CHUNK_MIN = 4 << 10;   // bytes: 8 and 1 accesses per thread
constexpr int GN_BLOCKS = 1024;        // workgroups of a launch: 4 per CU
constexpr int64_t GN_PARTIALS = 8192;  // partial results of all launches, while each has GN_BLOCKS_MIN workgroups
constexpr size_t GN_SMALL_BYTES = 64 << 10;
constexpr size_t GN_CACHE_BYTES = (size_t)256 << 20, GN_KEEP_BYTES = (size_t)192 << 20;   // memory-side cache
constexpr int64_t GN_BLOCKS_MIN = 64;

struct Tensors {
    const void* const* in;
    void* const* out;
    const int64_t* count;
    const int* dtype;
    int n;
};

int64_t launches_of(int64_t n) { return std::max<int64_t>(1, (n + GN_TENSORS - 1) / GN_TENSORS); }
int blocks_per_launch(int64_t n) {
    return (int)std::min<int64_t>(GN_BLOCKS, std::max(GN_BLOCKS_MIN, GN_PARTIALS / launches_of(n)));
}
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
    const int rc = written_twice(pieces, k) ? FLCE_ERR_ARG : FLCE_OK;
    delete[] pieces;
    return rc;
}

// Whether `bytes` bytes at p lie in an output, or (ins) in an input.
bool touches(const Tensors& t, bool ins, const void* p, size_t bytes) {
    const uintptr_t p0 = reinterpret_cast<uintptr_t>(p), p1 = p0 + bytes;
    auto in = [&](const void* q, int i) {
        const uintptr_t q0 = reinterpret_cast<uintptr_t>(q);
        return q0 < p1 && p0 < q0 + bytes_of(t, i);
    };
    for (int i = 0; i < t.n; ++i)
        if (t.count[i] && (in(t.out ? t.out[i] : t.in[i], i) || (ins && in(t.in[i], i)))) return true;
    return false;
}

// How the tensors are cut for both sweeps.
struct Cut {
    size_t total;          // bytes of all tensors
    int64_t chunk_bytes;   // as long as they may be while there are enough of them for every workgroup
    int blocks;            // most workgroups of a launch
};
Cut cut_of(const Tensors& t) {
    Cut c{0, GN_CHUNK, blocks_per_launch(t.n)};
    for (int i = 0; i < t.n; ++i) c.total += bytes_of(t, i);
    while (c.chunk_bytes > GN_CHUNK_MIN && c.total / (size_t)c.chunk_bytes < (size_t)GN_BLOCKS) c.chunk_bytes /= 2;
    while (c.total / (size_t)c.chunk_bytes > ((size_t)1 << 30)) c.chunk_bytes *= 2;   // (counted in 32 bits)
    return c;
}
// The launch of tensors first .. (at most GN_TENSORS of them), whose bytes begin at `at` of all; those below `until`
// are streamed past the cache.  bytes: its bytes; blocks: its workgroups, 0 if there is nothing in them.
GnArgs launch_args(const Tensors& t, int first, const Cut& cut, size_t at, size_t until, size_t* bytes, int* blocks) {
    GnArgs a{};
    int64_t chunks = 0;
    const size_t begin = at;
    a.in_place = 1;
    for (int i = first; i < t.n && i < first + GN_TENSORS; ++i) {
        if (!t.count[i]) continue;
        const int k = a.tensors++;
        a.in[k] = t.in[i];
        a.out[k] = t.out ? t.out[i] : const_cast<void*>(t.in[i]);
        if (a.out[k] != a.in[k]) a.in_place = 0;
        a.count[k] = t.dtype[i] == FLCE_BF16 ? ~t.count[i] : t.count[i];
        const size_t b = bytes_of(t, i), size = (size_t)cut.chunk_bytes;
        if (at < until) a.streamed = (int)(chunks + (std::min(b, until - at) + size - 1) / size);
        chunks += (int64_t)((b + size - 1) / size);
        a.first_chunk[k + 1] = (int)chunks;
        at += b;
    }
    a.chunk_bytes = (int)cut.chunk_bytes;
    *bytes = at - begin;
    *blocks = (int)std::min<int64_t>(chunks, cut.blocks);
    return a;
}

// Few elements: one launch of one workgroup, without partial results.
bool one_workgroup(const Tensors& t, const Cut& cut) { return cut.total <= GN_SMALL_BYTES && t.n <= GN_TENSORS; }

// Memory for the partial results; it may not lie where they or the norm would overwrite what is still read.
int partial_memory(const Tensors& t, const Cut& cut, const float* norm, void* workspace, size_t workspace_bytes,
                   hipStream_t s, double** out) {
    const size_t need = partial_bytes(t.n);
    char* ws = static_cast<char*>(workspace);
    if (workspace) {
        if (!aligned(workspace, 256)) return FLCE_ERR_ALIGN;
        if (workspace_bytes < need) return FLCE_ERR_WORKSPACE;
    }
    *out = nullptr;
    if (one_workgroup(t, cut)) return FLCE_OK;
    if (!workspace) FLCE_TRY(shared_workspace(need, &ws, s));
    const char* n = reinterpret_cast<const char*>(norm);
    if (touches(t, true, ws, need) || (n < ws + need && ws < n + sizeof(float))) return FLCE_ERR_ARG;
    *out = reinterpret_cast<double*>(ws);
    return FLCE_OK;
}

// Sweep 1; *partials: the results it leaves.  Tensors that do not fit the memory-side cache together are read past
// it, but for the end of them where a second sweep follows, which begins there.
template <typename Op>
int sweep_norm(const Tensors& t, const Cut& cut, bool second_sweep, double* partial, int* partials, hipStream_t s) {
    const size_t until = cut.total <= GN_CACHE_BYTES ? 0 : second_sweep ? cut.total - GN_KEEP_BYTES : cut.total;
    size_t at = 0;
    *partials = 0;
    for (int first = 0; first < t.n; first += GN_TENSORS) {
        int blocks;
        size_t bytes;
        GnArgs a = launch_args(t, first, cut, at, until, &bytes, &blocks);
        at += bytes;
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
int sweep_scale(const Tensors& t, const Cut& cut, const double* partial, int partials, const float* norm_in,
                float* norm_out, float max_norm, hipStream_t s) {
    const size_t until = (t.out ? 2 : 1) * cut.total <= GN_CACHE_BYTES ? 0 : cut.total;
    for (int64_t l = launches_of(t.n) - 1; l >= 0; --l) {
        int blocks;
        size_t bytes;
        GnArgs a = launch_args(t, (int)(l * GN_TENSORS), cut, 0, until, &bytes, &blocks);
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

// clip: scale too.
template <typename Op>
int run(const Tensors& t, const Cut& cut, bool clip, double* partial, float max_norm, float* norm, hipStream_t s) {
    int partials;
    if (one_workgroup(t, cut)) {
        size_t bytes;
        GnArgs a = launch_args(t, 0, cut, 0, 0, &bytes, &partials);
        a.norm_out = norm;
        a.max_norm = max_norm;
        hipLaunchKernelGGL((grad_small_kernel<Op>), dim3(1), dim3(GN_THREADS), 0, s, a, clip ? 1 : 0);
        HIP_TRY(hipGetLastError());
        return FLCE_OK;
    }
    FLCE_TRY(sweep_norm<Op>(t, cut, clip, partial, &partials, s));
    // One scaling launch adds the partial results up in each of its workgroups (1 us); several of them, of more
    // partial results, share a launch that does it once (4 us).
    if (clip && launches_of(t.n) == 1) return sweep_scale<Op>(t, cut, partial, partials, nullptr, norm, max_norm, s);
    hipLaunchKernelGGL((grad_norm_final_kernel<Op>), dim3(1), dim3(GN_THREADS), 0, s, partial, partials, norm);
    HIP_TRY(hipGetLastError());
    return clip ? sweep_scale<Op>(t, cut, nullptr, 0, norm, nullptr, max_norm, s) : FLCE_OK;
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
    if (touches(t, true, norm, sizeof(float))) return FLCE_ERR_ARG;
    const Cut cut = cut_of(t);
    double* partial;
    hipStream_t s = static_cast<hipStream_t>(stream);
    FLCE_TRY(partial_memory(t, cut, norm, workspace, workspace_bytes, s, &partial));
    return norm_type == FLCE_NORM_2 ? run<GnSumSq>(t, cut, false, partial, 0.0f, norm, s)
                                    : run<GnMax>(t, cut, false, partial, 0.0f, norm, s);
}

int flce_grad_clip(const void* const* grads, void* const* outs, const int64_t* counts, const int* dtypes, int n_tensors,
                   const float* norm, float max_norm, void* stream) {
    const Tensors t{grads, outs, counts, dtypes, n_tensors};
    FLCE_TRY(check_tensors(t));
    if (!norm) return FLCE_ERR_NULL;
    if (!aligned(norm, 4)) return FLCE_ERR_ALIGN;
    if (!finite_not_negative(max_norm)) return FLCE_ERR_ARG;
    FLCE_TRY(check_outputs(t));
    if (touches(t, false, norm, sizeof(float))) return FLCE_ERR_ARG;
    return sweep_scale<GnSumSq>(t, cut_of(t), nullptr, 0, norm, nullptr, max_norm, static_cast<hipStream_t>(stream));
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
    if (touches(t, true, norm, sizeof(float))) return FLCE_ERR_ARG;
    const Cut cut = cut_of(t);
    double* partial;
    hipStream_t s = static_cast<hipStream_t>(stream);
    FLCE_TRY(partial_memory(t, cut, norm, workspace, workspace_bytes, s, &partial));
    return norm_type == FLCE_NORM_2 ? run<GnSumSq>(t, cut, true, partial, max_norm, norm, s)
                                    : run<GnMax>(t, cut, true, partial, max_norm, norm, s);
}

}  // extern "C"
