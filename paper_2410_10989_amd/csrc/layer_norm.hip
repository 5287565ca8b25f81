// C ABI of the layer norm (see layer_norm.h): argument checks, shapes of the kernels, plan of the backward's sums over
// rows, launches.
#include "layer_norm.h"

#include <algorithm>
#include <type_traits>

#include "flce_host.h"

using namespace flce;

namespace {

constexpr int64_t LN_MAX_H = (int64_t)1 << 24;      // keeps launches and column numbers within 32 bits
constexpr int64_t LN_GRID_X = (int64_t)1 << 20;     // workgroups along x, the rest along y
// Threads per CU that the backward is launched for; more where a workgroup's row is so short that two of them have too little
// on the way.  us with 512 and 768, 8192 rows with a residual: 1280 bf16 30.8 and 28.9, 2304 44.0 and 41.2, 2816 45.5 and
// 44.8, 4096 57.2 and 58.8, 1600 fp32 42.4 and 43.6; several rows per workgroup: 16384 x 1024 bf16 31.3 and 37.4.
constexpr int LN_CU_THREADS = 512, LN_SHORT_CU_THREADS = 768;
constexpr int64_t LN_SHORT_BYTES = 5632;
// Fewest workgroups of a backward with partial sums, while there are rows for them (us with 32, 128 and 256: 128 rows of 4096
// bf16 12.4, 9.2, 9.2; 256 rows 18.9, 11.2, 12.5); rows that one workgroup takes one after the other and writes the sums of
// itself (2 rows of 4096: 5.8, with partial sums 7.0; 4 rows 9.0 and 7.0).
constexpr int64_t LN_CUS = 256, LN_FEW_BLOCKS = 128, LN_ONE_STEPS = 3;
constexpr int64_t LN_CACHE_BYTES = (int64_t)256 << 20;   // memory-side cache

size_t elem(int dtype) { return dtype == FLCE_F32 ? 4 : 2; }

struct Strides {
    int64_t x, y, h, n, dx, dh, dn;
};

int check_common(const flce_layer_norm* b, Strides* st) {
    if (!b) return FLCE_ERR_NULL;
    if (b->size != sizeof(flce_layer_norm)) return FLCE_ERR_ARG;
    if (b->dtype != FLCE_F32 && b->dtype != FLCE_BF16) return FLCE_ERR_DTYPE;
    if (b->rows < 1 || b->rows > MAX_DIM || b->H < 1 || b->H > LN_MAX_H) return FLCE_ERR_SHAPE;
    if (!(b->eps >= 0.0f) || b->eps - b->eps != 0.0f) return FLCE_ERR_ARG;
    const int64_t given[] = {b->ldx, b->ldy, b->ldh, b->ldn, b->lddx, b->lddh, b->lddn};
    int64_t* to[] = {&st->x, &st->y, &st->h, &st->n, &st->dx, &st->dh, &st->dn};
    for (int i = 0; i < 7; ++i) {
        if (given[i] && b->rows > 1 && (given[i] < b->H || given[i] > MAX_DIM * 4)) return FLCE_ERR_SHAPE;
        *to[i] = given[i] && b->rows > 1 ? given[i] : b->H;   // (a single row has no stride)
    }
    return FLCE_OK;
}

// The register forms: TPR threads per row with E elements each (see bn_shape in block_norm.hip for the widths).
struct Shape {
    int tpr, e;   // tpr = 0: the long form
};
Shape shape_of(int64_t H, int dtype, bool backward) {
    if (backward && H < 8) return {0, 0};   // (its loads are whole vectors)
    if (H <= 128) return {16, 8};
    if (H <= 512) return {64, 8};
    if (H <= 1024) return {64, 16};
    if (H <= 2048) return {256, 8};
    if (H <= 4096) return dtype == FLCE_F32 ? Shape{512, 8} : Shape{256, 16};
    if (H <= 8192) return {512, 16};
    if (H <= 16384) return {1024, 16};
    return {0, 0};
}
int threads_of(const Shape& s) { return s.tpr > WAVE ? s.tpr : s.tpr ? 256 : LN_LONG_THREADS; }
int groups_of(const Shape& s) { return s.tpr && s.tpr <= WAVE ? 256 / s.tpr : 1; }

// Nontemporal stores where a call's rows do not fit the memory-side cache anyway.
bool nontemporal(const flce_layer_norm& b, int streams) {
    return (int64_t)streams * b.rows * b.H * (int64_t)elem(b.dtype) > LN_CACHE_BYTES;
}

// Workgroups of the backward, and where its partial sums lie (floats from the workspace's start).
struct Plan {
    int64_t blocks;
    bool one;   // one workgroup holds all rows: no partial sums
    size_t off_beta, total_bytes;
};
Plan plan_for(const Shape& s, const flce_layer_norm& b, bool gamma, bool beta, int64_t blocks) {
    Plan p{};
    p.blocks = std::max<int64_t>(1, std::min(blocks, (b.rows + groups_of(s) - 1) / groups_of(s)));
    p.one = p.blocks == 1 && s.tpr;
    p.off_beta = gamma && !p.one ? (size_t)p.blocks * (size_t)b.H : 0;
    p.total_bytes = (p.off_beta + (beta && !p.one ? (size_t)p.blocks * (size_t)b.H : 0)) * sizeof(float);
    return p;
}
// As many workgroups as fill the chip, fewer for few rows (each costs its partial sums), and no more than `cap` bytes
// of partial sums allow.
Plan plan_of(const Shape& s, const flce_layer_norm& b, bool gamma, bool beta, size_t cap) {
    int64_t target = 1;
    if (!s.tpr || b.rows > LN_ONE_STEPS * groups_of(s)) {
        const bool is_short = s.tpr == 256 && b.H * (int64_t)elem(b.dtype) <= LN_SHORT_BYTES;
        const int64_t most = LN_CUS * std::max(1, (is_short ? LN_SHORT_CU_THREADS : LN_CU_THREADS) / threads_of(s));
        target = std::min(most, std::max({LN_FEW_BLOCKS, std::min<int64_t>(LN_CUS, b.rows / 4), b.rows / 8}));
    }
    for (;; target /= 2) {
        const Plan p = plan_for(s, b, gamma, beta, target);
        if (p.total_bytes <= cap || target == 1) return p;
    }
}

template <typename T, bool NT, int TPR, int E>
void launch_fwd(const LnArgs& a, hipStream_t s) {
    constexpr int GROUPS = row_groups<TPR>;
    const int64_t blocks = ((int64_t)a.rows + GROUPS - 1) / GROUPS;
    const dim3 grid((unsigned)std::min(blocks, LN_GRID_X), (unsigned)((blocks + LN_GRID_X - 1) / LN_GRID_X));
    hipLaunchKernelGGL((layer_norm_fwd_kernel<T, TPR, E / RowVec<T>::N, NT>), grid, dim3(row_block<TPR>), 0, s, a);
}
template <typename T, bool NT>
int run_fwd(const LnArgs& a, hipStream_t s) {
    constexpr bool F32 = std::is_same<T, float>::value;
    const Shape sh = shape_of(a.H, F32 ? FLCE_F32 : FLCE_BF16, false);
    if (sh.tpr == 16) {
        launch_fwd<T, NT, 16, 8>(a, s);
    } else if (sh.tpr == 64 && sh.e == 8) {
        launch_fwd<T, NT, 64, 8>(a, s);
    } else if (sh.tpr == 64) {
        launch_fwd<T, NT, 64, 16>(a, s);
    } else if (sh.tpr == 256 && sh.e == 8) {
        launch_fwd<T, NT, 256, 8>(a, s);
    } else if (sh.tpr == (F32 ? 512 : 256) && sh.e == (F32 ? 8 : 16)) {
        launch_fwd<T, NT, F32 ? 512 : 256, F32 ? 8 : 16>(a, s);
    } else if (sh.tpr == 512) {
        launch_fwd<T, NT, 512, 16>(a, s);
    } else if (sh.tpr == 1024) {
        launch_fwd<T, NT, 1024, 16>(a, s);
    } else {
        const int64_t rows = a.rows;
        const dim3 grid((unsigned)std::min(rows, LN_GRID_X), (unsigned)((rows + LN_GRID_X - 1) / LN_GRID_X));
        hipLaunchKernelGGL((layer_norm_fwd_long<T, NT>), grid, dim3(LN_LONG_THREADS), 0, s, a);
    }
    HIP_TRY(hipGetLastError());
    return FLCE_OK;
}

template <typename T, bool NT, int TPR, int E>
void launch_bwd(const LnArgs& a, const dim3& grid, hipStream_t s) {
    constexpr int NV = E / RowVec<T>::N;
    hipLaunchKernelGGL((layer_norm_bwd_kernel<T, TPR, NV, (NV <= 2 && TPR < 1024), NT>), grid, dim3(row_block<TPR>), 0, s, a);
}
template <typename T, bool NT>
int run_bwd(const LnArgs& a, const Shape& sh, const Plan& p, void* dgamma, void* dbeta, hipStream_t s) {
    constexpr bool F32 = std::is_same<T, float>::value;
    const dim3 grid((unsigned)p.blocks);
    if (sh.tpr == 16) {
        launch_bwd<T, NT, 16, 8>(a, grid, s);
    } else if (sh.tpr == 64 && sh.e == 8) {
        launch_bwd<T, NT, 64, 8>(a, grid, s);
    } else if (sh.tpr == 64) {
        launch_bwd<T, NT, 64, 16>(a, grid, s);
    } else if (sh.tpr == 256 && sh.e == 8) {
        launch_bwd<T, NT, 256, 8>(a, grid, s);
    } else if (sh.tpr == (F32 ? 512 : 256) && sh.e == (F32 ? 8 : 16)) {
        launch_bwd<T, NT, F32 ? 512 : 256, F32 ? 8 : 16>(a, grid, s);
    } else if (sh.tpr == 512) {
        launch_bwd<T, NT, 512, 16>(a, grid, s);
    } else if (sh.tpr == 1024) {
        launch_bwd<T, NT, 1024, 16>(a, grid, s);
    } else {
        hipLaunchKernelGGL((layer_norm_bwd_long<T, NT>), grid, dim3(LN_LONG_THREADS), 0, s, a);
    }
    HIP_TRY(hipGetLastError());
    PartialSums b{};
    int sets = 0;
    auto add = [&](const float* part, void* out) {
        if (!part) return;
        b.part[sets] = part;
        b.out[sets] = out;
        b.ld[sets] = a.H;
        b.parts[sets] = (int)p.blocks;
        b.first[sets] = sets;
        ++sets;
    };
    add(a.part_gamma, dgamma);
    add(a.part_beta, dbeta);
    if (!sets) return FLCE_OK;
    for (int i = sets; i < 4; ++i) b.first[i] = sets;
    hipLaunchKernelGGL((sum_partials_kernel<T>), dim3((unsigned)((a.H + SUM_COLS - 1) / SUM_COLS), (unsigned)sets),
                       dim3(SUM_COLS * SUM_PARTS), 0, s, b, a.H);
    HIP_TRY(hipGetLastError());
    return FLCE_OK;
}

}  // namespace

extern "C" {

int flce_layer_norm_fwd(const void* x, const void* y, const void* gamma, const void* beta, const flce_layer_norm* args,
                        void* h, void* n, void* stream) {
    Strides ld;
    FLCE_TRY(check_common(args, &ld));
    const flce_layer_norm& b = *args;
    if (!x || !n || (y && !h)) return FLCE_ERR_NULL;
    if (!y && h) return FLCE_ERR_ARG;
    const size_t es = elem(b.dtype);
    for (const void* p : {x, y, gamma, beta, static_cast<const void*>(h), static_cast<const void*>(n)})
        if (p && !aligned(p, es)) return FLCE_ERR_ALIGN;
    const Span in[] = {span(x, ld.x, b.rows, b.H, es), span(y, ld.y, b.rows, b.H, es), span(gamma, b.H, 1, b.H, es),
                       span(beta, b.H, 1, b.H, es)};
    const Span oh = span(h, ld.h, b.rows, b.H, es), on = span(n, ld.n, b.rows, b.H, es);
    if (overlap(oh, on)) return FLCE_ERR_ARG;
    for (int i = 0; i < 4; ++i) {
        // h exactly on x, and then on a y that is exactly x too: a thread reads what it overwrites first
        const bool own = i < 2 && same(oh, in[0]) && same(oh, in[i]);
        if ((overlap(oh, in[i]) && !own) || overlap(on, in[i])) return FLCE_ERR_ARG;
    }
    LnArgs a{};
    a.x = x;
    a.y = y;
    a.gamma = gamma;
    a.beta = beta;
    a.out_h = h;
    a.out_n = n;
    a.ldx = ld.x;
    a.ldy = ld.y;
    a.ldh = ld.h;
    a.ldn = ld.n;
    a.rows = (int)b.rows;
    a.H = (int)b.H;
    a.eps = b.eps;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (nontemporal(b, y ? 4 : 2)) return b.dtype == FLCE_F32 ? run_fwd<float, true>(a, s) : run_fwd<bf16_t, true>(a, s);
    return b.dtype == FLCE_F32 ? run_fwd<float, false>(a, s) : run_fwd<bf16_t, false>(a, s);
}

int flce_layer_norm_bwd(const void* h, const void* dn, const void* dh, const void* gamma, const flce_layer_norm* args,
                        void* dx, void* dgamma, void* dbeta, void* stream) {
    Strides ld;
    FLCE_TRY(check_common(args, &ld));
    const flce_layer_norm& b = *args;
    if (!h || !dn) return FLCE_ERR_NULL;
    if ((!gamma && dgamma) || (!dx && !dgamma && !dbeta)) return FLCE_ERR_ARG;
    const size_t es = elem(b.dtype);
    const Span in[] = {span(dh, ld.dh, b.rows, b.H, es), span(h, ld.h, b.rows, b.H, es), span(dn, ld.dn, b.rows, b.H, es),
                       span(gamma, b.H, 1, b.H, es)};
    const Span out[] = {span(dx, ld.dx, b.rows, b.H, es), span(dgamma, b.H, 1, b.H, es), span(dbeta, b.H, 1, b.H, es)};
    for (const Span& i : in)
        if (i.p && !aligned(i.p, es)) return FLCE_ERR_ALIGN;
    for (const Span& o : out)
        if (o.p && !aligned(o.p, es)) return FLCE_ERR_ALIGN;
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return FLCE_ERR_ARG;
        for (int j = 0; j < 4; ++j)
            if (overlap(out[i], in[j]) && !(i == 0 && j == 0 && same(out[0], in[0]))) return FLCE_ERR_ARG;
    }
    if (b.workspace && !aligned(b.workspace, 256)) return FLCE_ERR_ALIGN;
    size_t cap = SIZE_MAX;
    if (b.workspace) {
        cap = b.workspace_bytes;
    } else {
        size_t lent = 0;
        FLCE_TRY(shared_workspace_lent(&lent));
        if (lent) cap = lent;
    }
    const Shape shape = shape_of(b.H, b.dtype, true);
    Plan p;
    char* ws = static_cast<char*>(b.workspace);
    hipStream_t s = static_cast<hipStream_t>(stream);
    for (;;) {   // (again with fewer workgroups where the library finds too little memory for this many)
        p = plan_of(shape, b, dgamma, dbeta, cap);
        if (p.total_bytes > cap) return FLCE_ERR_WORKSPACE;
        if (ws || !p.total_bytes) break;
        const int rc = shared_workspace(p.total_bytes, &ws, s, p.blocks == 1);
        if (rc == FLCE_OK) break;
        if (rc != FLCE_ERR_WORKSPACE || p.blocks == 1) return rc;
        cap = p.total_bytes - 1;
    }
    if (p.total_bytes) {   // partial sums are written while the operands are read
        const Span scratch{ws, p.total_bytes, p.total_bytes, 1};
        for (const Span& i : in)
            if (overlap(scratch, i)) return FLCE_ERR_ARG;
        for (const Span& o : out)
            if (overlap(scratch, o)) return FLCE_ERR_ARG;
    }
    float* f = reinterpret_cast<float*>(ws);
    LnArgs a{};
    a.h = h;
    a.dn = dn;
    a.dh = dh;
    a.gamma = gamma;
    a.dx = dx;
    a.part_gamma = dgamma && !p.one ? f : nullptr;
    a.part_beta = dbeta && !p.one ? f + p.off_beta : nullptr;
    a.dgamma = p.one ? dgamma : nullptr;
    a.dbeta = p.one ? dbeta : nullptr;
    a.ldh = ld.h;
    a.lddn = ld.dn;
    a.lddh = ld.dh;
    a.lddx = ld.dx;
    a.rows = (int)b.rows;
    a.H = (int)b.H;
    a.eps = b.eps;
    if (nontemporal(b, 2 + (dh != nullptr) + (dx != nullptr)))
        return b.dtype == FLCE_F32 ? run_bwd<float, true>(a, shape, p, dgamma, dbeta, s)
                                   : run_bwd<bf16_t, true>(a, shape, p, dgamma, dbeta, s);
    return b.dtype == FLCE_F32 ? run_bwd<float, false>(a, shape, p, dgamma, dbeta, s)
                               : run_bwd<bf16_t, false>(a, shape, p, dgamma, dbeta, s);
}

size_t flce_layer_norm_workspace_bytes(const flce_layer_norm* args) {
    Strides ld;
    if (check_common(args, &ld) != FLCE_OK) return 0;
    return plan_of(shape_of(args->H, args->dtype, true), *args, true, true, SIZE_MAX).total_bytes;
}

}  // extern "C"
