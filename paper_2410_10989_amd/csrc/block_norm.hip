// C ABI of the norms before and after a block (see block_norm.h): argument checks, shapes of the kernels,
// plan of the backward's sums over rows, launches.
#include "block_norm.h"

#include <algorithm>
#include <type_traits>

#include "flce_host.h"

using namespace flce;

namespace {

constexpr int64_t BN_MAX_H = (int64_t)1 << 24;      // keeps launches and column numbers within 32 bits
constexpr int64_t BN_GRID_X = (int64_t)1 << 20;     // workgroups along x, the rest along y
constexpr int BN_CU_THREADS = 512;                 // threads per CU that the backward is launched for
constexpr int BN_CUS = 256;
constexpr int64_t BN_FEW_BLOCKS = 128, BN_ONE_STEPS = 3;
constexpr int64_t BN_ONE_PER_CU_COLS = 2900;
constexpr int64_t BN_CACHE_BYTES = (int64_t)256 << 20;   // memory-side cache

size_t bn_elem(int dtype) { return dtype == FLCE_F32 ? 4 : 2; }

struct Strides {
    int64_t x, y, h, n, gate, dx, dy, dh, dn, dgate;
};

int check_common(const flce_block_norm* b, Strides* st, int64_t* gate_rows) {
    if (!b) return FLCE_ERR_NULL;
    if (b->size != sizeof(flce_block_norm)) return FLCE_ERR_ARG;
    if (b->dtype != FLCE_F32 && b->dtype != FLCE_BF16) return FLCE_ERR_DTYPE;
    if (b->rows < 1 || b->rows > MAX_DIM || b->H < 1 || b->H > BN_MAX_H) return FLCE_ERR_SHAPE;
    if (b->gate_act < FLCE_GATE_LINEAR || b->gate_act > FLCE_GATE_TANH) return FLCE_ERR_ARG;
    if (b->rows_per_gate < 0 || b->rows_per_gate > MAX_DIM) return FLCE_ERR_ARG;
    if (!(b->eps >= 0.0f) || b->eps - b->eps != 0.0f || b->scale - b->scale != 0.0f) return FLCE_ERR_ARG;
    *gate_rows = b->rows_per_gate ? (b->rows + b->rows_per_gate - 1) / b->rows_per_gate : 1;
    const int64_t given[] = {b->ldx, b->ldy, b->ldh, b->ldn, b->ldgate, b->lddx, b->lddy, b->lddh, b->lddn, b->lddgate};
    int64_t* to[] = {&st->x, &st->y, &st->h, &st->n, &st->gate, &st->dx, &st->dy, &st->dh, &st->dn, &st->dgate};
    for (int i = 0; i < 10; ++i) {
        const bool one = (i == 4 || i == 9) ? *gate_rows == 1 : b->rows == 1;   // (a single row has no stride)
        if (given[i] && !one && (given[i] < b->H || given[i] > MAX_DIM * 4)) return FLCE_ERR_SHAPE;
        *to[i] = given[i] && !one ? given[i] : b->H;
    }
    return FLCE_OK;
}

// The register forms: TPR threads per row with E elements each (a table by width, not by size: each row of it was the
// fastest of its neighbours over its range).  Twice the elements per thread halve what a row costs besides them (sums
// over lanes, addresses), half of them leaves registers for more wavefronts: backward, us, 8 / 16 elements: 8192 x 2048
// 41 / 44, 8192 x 2560 55 / 47, 16384 x 512 20 / 22; rows of 513 .. 1024 in one wavefront of 16 elements per lane, or two
// of 8: 16384 x 768 26 / 38 (forward 16.8 / 16.9), 2048 x 1000 9.8 / 12.7.  fp32 rows have half the elements per load
// in flight: 4096 x 4096 66 / 79.
struct BnShape {
    int tpr, e;   // tpr = 0: the long form
};
BnShape bn_shape(int64_t H, int dtype, bool backward, bool three_sums = false) {
    if (backward && H < 8) return {0, 0};   // (its loads are whole vectors)
    if (H <= 128) return {16, 8};
    if (H <= 512) return {64, 8};
    if (H <= 1024) return {64, 16};
    if (H <= 2048) return {256, 8};
    if (H <= 4096) return dtype == FLCE_F32 ? BnShape{512, 8} : BnShape{256, 16};
    if (H <= 8192) return {512, 16};
    if (H <= BN_WIDE_COLS && !backward) return {1024, 16};
    if (H <= (three_sums ? BN_WIDE_COLS_3 : BN_WIDE_COLS) && backward) return {512, 32};
    return {0, 0};
}
int bn_threads(const BnShape& s) { return s.tpr > WAVE ? s.tpr : s.tpr ? 256 : BN_LONG_THREADS; }
int bn_groups(const BnShape& s) { return s.tpr && s.tpr <= WAVE ? 256 / s.tpr : 1; }

// Nontemporal stores where a call's rows do not fit the memory-side cache anyway: what the call reads then stays in
// it.  us, ordinary / nontemporal: 402 MB of rows 76 / 60 (backward), 470 MB 89 / 68 (forward); between a kernel that
// writes y and one that reads n: 470 MB 161 / 149, 403 MB 139 / 128, but 268 MB 85 / 87.
bool bn_nontemporal(const flce_block_norm& b, int streams) {
    return (int64_t)streams * b.rows * b.H * (int64_t)bn_elem(b.dtype) > BN_CACHE_BYTES;
}

// How the backward deals rows to workgroups, and where its partial sums lie (floats from the workspace's start).
struct BnPlan {
    int64_t blocks, segments, parts, per;
    bool direct;   // a segment holds all rows of its gate row
    bool one;      // one workgroup holds all rows: no partial sums of the gammas
    size_t off_post, off_gate, total_bytes;
};

// per: rows per gate row where rows share one, else all rows; gate_sum: its gradient is wanted.
BnPlan bn_plan_for(const BnShape& s, int64_t rows, int64_t H, int64_t per, bool pre, bool post, bool gate_sum,
                   int64_t target) {
    const int64_t groups = bn_groups(s);
    BnPlan p{};
    p.per = std::min(per, rows);
    const int64_t G = (rows + p.per - 1) / p.per;
    p.parts = 1;
    if (G == 1) {
        p.parts = std::max<int64_t>(1, std::min(target, (rows + groups - 1) / groups));
    } else if (G < target) {
        // rounds of segments over the workgroups times the steps of one (a step is `groups` rows; writing a
        // segment's sums counts as one).  The search costs the host up to 5 us of a call (2 gate rows; 4: 2, 16:
        // 0.7).  From G = target on gate rows stay whole, and a last round of few of them is as long as a full one.
        int64_t best = INT64_MAX;
        for (int64_t c = 1; c <= std::min<int64_t>(p.per, 4 * ((target + G - 1) / G)); ++c) {
            const int64_t cost = ((G * c + target - 1) / target) * (((p.per + c - 1) / c + groups - 1) / groups + 1);
            if (cost < best) {
                best = cost;
                p.parts = c;
            }
        }
    }
    p.segments = G * p.parts;
    p.blocks = std::min(p.segments, target);
    p.direct = gate_sum && p.parts == 1;
    const int64_t gate_rows = !gate_sum ? 0 : p.direct ? (s.tpr ? 0 : p.blocks) : p.segments;
    p.one = p.blocks == 1 && s.tpr;
    size_t at = 0;
    auto take = [&](int64_t n) {
        const size_t here = at;
        at += (size_t)n * (size_t)H;
        return here;
    };
    take(pre && !p.one ? p.blocks : 0);
    p.off_post = take(post && !p.one ? p.blocks : 0);
    p.off_gate = take(gate_rows);
    p.total_bytes = at * sizeof(float);
    return p;
}
// Workgroups of the backward.  Up to two of 256 threads per CU (or one of 512), but one where a row fills most of the
// (256, 16) form's vectors: their loads a row ahead fill the memory pipes, and every workgroup more costs its
// partial sums (us, 256 / 512 workgroups, inputs not in the cache: 8192 rows with one sum, H = 2304 49.8 / 44.4, 2816
// 49.2 / 48.6, 3200 53.4 / 54.6, 3584 58.3 / 60.2, 4096 65.7 / 68.1; 16384 rows 2816 89.5 / 88.1, 3200 97.3 / 98.7; 3000
// rows with two sums 2816 31.2 / 31.1, 3200 32.1 / 34.3.  Three sums, 8192 rows: 2304 69.2 / 74.2, 4096 83.8 / 91.7.  Rows
// that do not start on 16 bytes, 8192 x 3583: 93 / 72).  Small batches: few rows
// per workgroup, because sums of few rows cost as much as the rows (512 / 256 / 128 workgroups, H = 4096 with a norm
// after the block: 256 rows 12.9 / 13.0 / 11.9, 1024 rows 19.8 / 19.2 / 22.8, 4096 x 2048 24.1 / 29.0 / 48.0; below 128
// rows one each).
// A handful of rows: one workgroup, which needs no second launch (us on the GPU, one / several: 2 x 4096 6.4 / 7.6, 8 x
// 1000 in two steps 6.6 / 7.4, 3 x 4096 8.0 / 7.6, 4 x 4096 9.6 / 7.6; a call that is not captured 15.5 / 18.3).
int64_t bn_target(const BnShape& s, int64_t rows, int64_t H) {
    if (s.tpr && rows <= BN_ONE_STEPS * bn_groups(s)) return 1;
    int64_t most = BN_CUS * std::max(1, BN_CU_THREADS / bn_threads(s));
    if (s.tpr == 256 && s.e == 16 && H >= BN_ONE_PER_CU_COLS && H % 8 == 0) most = BN_CUS;
    return std::min(most, std::max({BN_FEW_BLOCKS, std::min<int64_t>(BN_CUS, rows / 4), rows / 8}));
}
// That plan, or the largest power-of-two fraction of it whose sums fit `cap` bytes.
BnPlan bn_plan(const BnShape& s, int64_t rows, int64_t H, int64_t per, bool pre, bool post, bool gate_sum, size_t cap) {
    for (int64_t target = bn_target(s, rows, H);; target /= 2) {
        const BnPlan p = bn_plan_for(s, rows, H, per, pre, post, gate_sum, target);
        if (p.total_bytes <= cap || target == 1) return p;
    }
}

template <typename T, bool NT, int TPR, int E>
void launch_fwd(const BnArgs& a, hipStream_t s) {
    constexpr int NV = E / RowVec<T>::N, GROUPS = row_groups<TPR>;
    const int64_t blocks = (a.rows + GROUPS - 1) / GROUPS;
    const dim3 grid((unsigned)std::min(blocks, BN_GRID_X), (unsigned)((blocks + BN_GRID_X - 1) / BN_GRID_X));
    const dim3 block(row_block<TPR>);
#define BN_FWD(POST, GATE) hipLaunchKernelGGL((block_norm_fwd_kernel<T, TPR, NV, POST, GATE, NT>), grid, block, 0, s, a)
    if (a.gpost) {
        if (a.gate) BN_FWD(true, true); else BN_FWD(true, false);
    } else {
        if (a.gate) BN_FWD(false, true); else BN_FWD(false, false);
    }
#undef BN_FWD
}
template <typename T, bool NT, int TPR, int E>
void launch_bwd(const BnArgs& a, const dim3& grid, hipStream_t s) {
    constexpr int NV = E / RowVec<T>::N;
    const dim3 block(row_block<TPR>);
#define BN_BWD(POST, GATE) \
    hipLaunchKernelGGL((block_norm_bwd_kernel<T, TPR, NV, POST, GATE, (NV <= 2), (E == 32), NT>), grid, block, 0, s, a)
#define BN_BWD_GATE(POST)                             \
    do {                                              \
        if (!a.gate) BN_BWD(POST, BN_GATE_NONE);      \
        else if (a.by_row) BN_BWD(POST, BN_GATE_ROW); \
        else BN_BWD(POST, BN_GATE_SUM);               \
    } while (0)
    if (a.gpost) BN_BWD_GATE(true); else BN_BWD_GATE(false);
#undef BN_BWD_GATE
#undef BN_BWD
}
template <typename T, bool NT>
int run_fwd(const BnArgs& a, hipStream_t s) {
    constexpr bool F32 = std::is_same<T, float>::value;
    const BnShape sh = bn_shape(a.H, F32 ? FLCE_F32 : FLCE_BF16, false);
    if (sh.tpr == 16 && sh.e == 8) {
        launch_fwd<T, NT, 16, 8>(a, s);
    } else if (sh.tpr == 64 && sh.e == 8) {
        launch_fwd<T, NT, 64, 8>(a, s);
    } else if (sh.tpr == 64 && sh.e == 16) {
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
        const dim3 grid((unsigned)std::min(rows, BN_GRID_X), (unsigned)((rows + BN_GRID_X - 1) / BN_GRID_X));
        hipLaunchKernelGGL((block_norm_fwd_long<T, NT>), grid, dim3(BN_LONG_THREADS), 0, s, a);
    }
    HIP_TRY(hipGetLastError());
    return FLCE_OK;
}
template <typename T, bool NT>
int run_bwd(const BnArgs& a, const BnShape& sh, const BnPlan& p, void* dgamma_pre, void* dgamma_post, hipStream_t s) {
    constexpr bool F32 = std::is_same<T, float>::value;
    const dim3 grid((unsigned)p.blocks);
    if (sh.tpr == 16 && sh.e == 8) {
        launch_bwd<T, NT, 16, 8>(a, grid, s);
    } else if (sh.tpr == 64 && sh.e == 8) {
        launch_bwd<T, NT, 64, 8>(a, grid, s);
    } else if (sh.tpr == 64 && sh.e == 16) {
        launch_bwd<T, NT, 64, 16>(a, grid, s);
    } else if (sh.tpr == 256 && sh.e == 8) {
        launch_bwd<T, NT, 256, 8>(a, grid, s);
    } else if (sh.tpr == (F32 ? 512 : 256) && sh.e == (F32 ? 8 : 16)) {
        launch_bwd<T, NT, F32 ? 512 : 256, F32 ? 8 : 16>(a, grid, s);
    } else if (sh.tpr == 512 && sh.e == 16) {
        launch_bwd<T, NT, 512, 16>(a, grid, s);
    } else if (sh.tpr == 512) {
        launch_bwd<T, NT, 512, 32>(a, grid, s);
    } else {
        hipLaunchKernelGGL((block_norm_bwd_long<T, NT>), grid, dim3(BN_LONG_THREADS), 0, s, a);
    }
    HIP_TRY(hipGetLastError());
    PartialSums b{};
    int set = 0, rows = 0;
    auto add = [&](const float* part, void* out, int64_t ld, int64_t parts, int64_t out_rows) {
        b.part[set] = part;
        b.out[set] = out;
        b.ld[set] = ld;
        b.parts[set] = (int)parts;
        b.first[set] = rows;
        rows += (int)out_rows;
        ++set;
    };
    if (a.part_pre) add(a.part_pre, dgamma_pre, a.H, p.blocks, 1);
    if (a.part_post) add(a.part_post, dgamma_post, a.H, p.blocks, 1);
    if (a.part_gate && !p.direct) add(a.part_gate, a.dgate, a.lddgate, p.parts, p.segments / p.parts);
    if (!rows) return FLCE_OK;
    for (int i = set; i < 4; ++i) b.first[i] = rows;
    const int col_blocks = (a.H + SUM_COLS - 1) / SUM_COLS;
    hipLaunchKernelGGL((sum_partials_kernel<T>), dim3((unsigned)col_blocks, (unsigned)rows), dim3(SUM_COLS * SUM_PARTS),
                       0, s, b, a.H);
    HIP_TRY(hipGetLastError());
    return FLCE_OK;
}

}  // namespace

extern "C" {

int flce_block_norm_fwd(const void* x, const void* y, const void* gate, const void* gamma_post, const void* gamma_pre,
                        const flce_block_norm* args, void* h, void* n, void* stream) {
    Strides ld;
    int64_t gate_rows;
    FLCE_TRY(check_common(args, &ld, &gate_rows));
    const flce_block_norm& b = *args;
    if ((!x && !y) || (y && !h) || (gamma_pre && !n)) return FLCE_ERR_NULL;
    if ((!y && (gate || gamma_post || h)) || (!gamma_pre && n) || (!y && !gamma_pre)) return FLCE_ERR_ARG;
    const size_t es = bn_elem(b.dtype);
    for (const void* p : {x, y, gate, gamma_post, gamma_pre, static_cast<const void*>(h), static_cast<const void*>(n)})
        if (p && !aligned(p, es)) return FLCE_ERR_ALIGN;
    const Span in[] = {span(x, ld.x, b.rows, b.H, es), span(y, ld.y, b.rows, b.H, es),
                       span(gate, ld.gate, gate_rows, b.H, es), span(gamma_post, b.H, 1, b.H, es), span(gamma_pre, b.H, 1, b.H, es)};
    const Span oh = span(h, ld.h, b.rows, b.H, es), on = span(n, ld.n, b.rows, b.H, es);
    if (overlap(oh, on)) return FLCE_ERR_ARG;
    for (int i = 0; i < 5; ++i) {
        // h exactly on x, and then on a y or a gate per row that is exactly x too: a thread reads what it overwrites
        // first.  Not on what other rows read, nor on a gamma, which the long form reads after it has written h.
        const bool own = i < 3 && same(oh, in[0]) && same(oh, in[i]) && in[i].rows == b.rows;
        if (overlap(oh, in[i]) && !own) return FLCE_ERR_ARG;
        if (overlap(on, in[i])) return FLCE_ERR_ARG;
    }
    BnArgs a{};
    a.x = x;
    a.y = y;
    a.gate = gate;
    a.gpost = gamma_post;
    a.gpre = gamma_pre;
    a.out_h = h;
    a.out_n = n;
    a.ldx = ld.x;
    a.ldy = ld.y;
    a.ldgate = ld.gate;
    a.ldh = ld.h;
    a.ldn = ld.n;
    a.rows = (int)b.rows;
    a.H = (int)b.H;
    a.per = (int)(b.rows_per_gate ? b.rows_per_gate : MAX_DIM);
    a.act = b.gate_act;
    a.scale = b.scale;
    a.eps = b.eps;
    const bool by_row = gate && b.rows_per_gate == 1;
    const bool nt = bn_nontemporal(b, (x != nullptr) + 2 * (y != nullptr) + (gamma_pre != nullptr) + by_row);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (nt) return b.dtype == FLCE_F32 ? run_fwd<float, true>(a, s) : run_fwd<bf16_t, true>(a, s);
    return b.dtype == FLCE_F32 ? run_fwd<float, false>(a, s) : run_fwd<bf16_t, false>(a, s);
}

int flce_block_norm_bwd(const void* h, const void* dn, const void* dh, const void* y, const void* gate,
                        const void* gamma_post, const void* gamma_pre, const flce_block_norm* args, void* dx, void* dy,
                        void* dgate, void* dgamma_post, void* dgamma_pre, void* stream) {
    Strides ld;
    int64_t gate_rows;
    FLCE_TRY(check_common(args, &ld, &gate_rows));
    const flce_block_norm& b = *args;
    if ((gamma_pre && (!h || !dn)) || (!gamma_pre && !dh) || ((gate || gamma_post || dy) && !y)) return FLCE_ERR_NULL;
    if ((!gamma_pre && (h || dn || dgamma_pre)) || (!gate && dgate) || (!gamma_post && dgamma_post) ||
        (!dx && !dy && !dgate && !dgamma_post && !dgamma_pre))
        return FLCE_ERR_ARG;
    const size_t es = bn_elem(b.dtype);
    const Span in[] = {span(dh, ld.dh, b.rows, b.H, es),        span(h, ld.h, b.rows, b.H, es),
                       span(dn, ld.dn, b.rows, b.H, es),        span(y, ld.y, b.rows, b.H, es),
                       span(gate, ld.gate, gate_rows, b.H, es), span(gamma_post, b.H, 1, b.H, es),
                       span(gamma_pre, b.H, 1, b.H, es)};
    const Span out[] = {span(dx, ld.dx, b.rows, b.H, es), span(dy, ld.dy, b.rows, b.H, es),
                        span(dgate, ld.dgate, gate_rows, b.H, es), span(dgamma_post, b.H, 1, b.H, es),
                        span(dgamma_pre, b.H, 1, b.H, es)};
    for (const Span& i : in)
        if (i.p && !aligned(i.p, es)) return FLCE_ERR_ALIGN;
    for (const Span& o : out)
        if (o.p && !aligned(o.p, es)) return FLCE_ERR_ALIGN;
    for (int i = 0; i < 5; ++i) {
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return FLCE_ERR_ARG;
        for (int j = 0; j < 7; ++j)
            if (overlap(out[i], in[j]) && !(i == 0 && j == 0 && same(out[0], in[0]))) return FLCE_ERR_ARG;
    }
    if (b.workspace && !aligned(b.workspace, 256)) return FLCE_ERR_ALIGN;

    const bool by_row = gate && b.rows_per_gate == 1 && b.rows > 1;
    const bool sums = dgate && !by_row;
    const int64_t per = b.rows_per_gate ? b.rows_per_gate : b.rows;
    size_t cap = SIZE_MAX;
    if (b.workspace) cap = b.workspace_bytes;
    else {
        size_t lent = 0;
        FLCE_TRY(shared_workspace_lent(&lent));
        if (lent) cap = lent;
    }
    const BnShape shape = bn_shape(b.H, b.dtype, true, gamma_post && gate && !by_row);
    BnPlan p;
    char* ws = static_cast<char*>(b.workspace);
    hipStream_t s = static_cast<hipStream_t>(stream);
    for (;;) {   // (again with fewer workgroups where the library finds too little memory for this many)
        p = bn_plan(shape, b.rows, b.H, gate && !by_row ? per : b.rows, dgamma_pre, dgamma_post, sums, cap);
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
    BnArgs a{};
    a.h = h;
    a.dn = dn;
    a.dh = dh;
    a.y = y;
    a.gate = gate;
    a.gpost = gamma_post;
    a.gpre = gamma_pre;
    a.dx = dx;
    a.dy = dy;
    a.dgate = dgate;
    a.ldh = ld.h;
    a.lddn = ld.dn;
    a.lddh = ld.dh;
    a.ldy = ld.y;
    a.ldgate = ld.gate;
    a.lddx = ld.dx;
    a.lddy = ld.dy;
    a.lddgate = ld.dgate;
    a.part_pre = dgamma_pre && !p.one ? f : nullptr;
    a.part_post = dgamma_post && !p.one ? f + p.off_post : nullptr;
    a.dpre = p.one ? dgamma_pre : nullptr;
    a.dpost = p.one ? dgamma_post : nullptr;
    a.part_gate = sums && (!p.direct || !shape.tpr) ? f + p.off_gate : nullptr;
    a.rows = (int)b.rows;
    a.H = (int)b.H;
    a.per = (int)p.per;
    a.act = b.gate_act;
    a.scale = b.scale;
    a.eps = b.eps;
    a.segments = (int)p.segments;
    a.parts = (int)p.parts;
    a.by_row = by_row;
    a.gate_direct = p.direct;
    const bool nt = bn_nontemporal(b, 2 * (h != nullptr) + (dh != nullptr) + (y != nullptr) + (dx != nullptr) +
                                          (dy != nullptr) + by_row + (by_row && dgate));
    if (nt)
        return b.dtype == FLCE_F32 ? run_bwd<float, true>(a, shape, p, dgamma_pre, dgamma_post, s)
                                   : run_bwd<bf16_t, true>(a, shape, p, dgamma_pre, dgamma_post, s);
    return b.dtype == FLCE_F32 ? run_bwd<float, false>(a, shape, p, dgamma_pre, dgamma_post, s)
                               : run_bwd<bf16_t, false>(a, shape, p, dgamma_pre, dgamma_post, s);
}

size_t flce_block_norm_workspace_bytes(const flce_block_norm* args) {
    Strides ld;
    int64_t gate_rows;
    if (check_common(args, &ld, &gate_rows) != FLCE_OK) return 0;
    const int64_t per = args->rows_per_gate ? args->rows_per_gate : args->rows;
    const int64_t rows = args->rows, H = args->H;
    // three sets of sums, or (a gate row per row, or none) the gammas' alone, each in a plan of its own
    auto bytes = [&](bool post, bool gate) {
        return bn_plan(bn_shape(H, args->dtype, true, post && gate), rows, H, gate ? per : rows, true, post, gate, SIZE_MAX)
            .total_bytes;
    };
    return std::max({bytes(true, true), bytes(false, true), bytes(true, false)});
}

}  // extern "C"
