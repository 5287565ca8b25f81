// C ABI of the orthogonalisation (see orthogonalize.h): argument checks, the powers of two that keep the iterates in
// fp16's range, workspace, launches.
#include "orthogonalize.h"

#include <math.h>

#include <algorithm>
#include <new>
#include <type_traits>

#include "flce_host.h"

using namespace flce;
static_assert(OR_SMALL <= 256, "one tile of 256");

namespace {

constexpr int64_t OR_MAX_DIM = (int64_t)1 << 20;         // a tile's rows stay below 2^31 bytes apart
constexpr int64_t OR_MAX_ELEMENTS = (int64_t)1 << 28;    // of a padded matrix: its planes stay below 2^30 bytes
// n / m from which two steps are taken at a time.  24 matrices, us in pairs and step by step: bf16 1024 x 1024 827 and 805,
// 1024 x 2048 1078 and 1207, 1024 x 4096 1640 and 2098; fp32 1024 x 1024 2007 and 1884, 1024 x 1536 2435 and 2562, 1024 x 2048
// 2627 and 2870, 1024 x 4096 3970 and 5030.
constexpr int64_t OR_PAIR_LENGTH = 2;
// Most that the first of two such steps may multiply by (its largest |a + b l + c l^2|).  What rounding B' B to 11 or 22 bits
// leaves of the large singular values in the directions of the small ones grows with that, and no A of an X between sees
// it.  Matrices of rank 2, 30 to 300 times as large as noise, 320 x 704 bf16, off by so much step by step and in pairs:
// 3.44 (the usual steps) 1.7e-3 .. 2.5e-3 and 1.8e-3 .. 3.2e-3; 4.08 and less 1.8e-3 .. 2.5e-3 and 2.2e-3 .. 6.8e-3; 8 twice 2.0e-3 ..
// 2.7e-3 and 1.2e-2 .. 2.5e-2.
constexpr double OR_PAIR_GROWTH = 3.5;
constexpr double OR_ITERATE_GROWTH = 20000.0;            // of a rounding error of A (see or_iterate_kernel)
constexpr double OR_MAX_NORM = 1024.0;                   // that a singular value of an iterate may reach
constexpr double OR_LIFT = 4.0;                          // see steps_of (fp16 has room for another 4)
// Fewest tiles of 256 that a launch takes those for, and that two steps at a time take.  Whole calls in tiles of 256 and of
// 128, us: bf16 2 x 2048 x 2048 (128 tiles) 557 and 505, 1 x 4096 x 4096 (136) 1528 and 1605, 16 x 1024 x 1024 (160) 598 and
// 628; 1 x 4096 x 14336 (136), two steps at a time or one, bf16 3170 and 4350, fp32 8540 and 11100.  Operands in two planes, whose
// tiles of 128 take both at a time: 4 x 2048 x 2048 fp32 (144 and 256 tiles) 2192 with both in tiles of 256, 2046 with the
// larger ones so, 2101 with none.
constexpr int64_t OR_TILES_256 = 132, OR_TILES_256_PLANES = 256;
static_assert(OR_MATRICES < OR_TILES_256, "Gram products of up to OR_SMALL rows never take them");
constexpr int64_t OR_SLOTS_128 = 256;                    // workgroups that ranges of K may make: one per CU
// Fewest turns of a range's K loop, most ranges, and turns one after the other that ranges have to save (a turn: 64 of K and
// one product).  us: a range of 8 turns or of 4: 512 x 512 fp32 198 and 223, 256 x 4096 bf16 168 and 182; ranges that
// save 20 turns or none: 1024 x 1024 bf16 199 and 259; 20 or 32: 512 x 2048 bf16 164 and 191.
constexpr int64_t OR_RANGE_STEPS = 8, OR_MAX_RANGES = 16, OR_SAVED_STEPS = 20;
constexpr int64_t OR_ROUNDS = 1024;                      // tiles of a launch that more matrices would not fill better
constexpr float OR_USUAL[3] = {3.4445f, -4.7750f, 2.0315f};

size_t elem(int dtype) { return dtype == FLCE_F32 ? 4 : 2; }
int64_t padded(int64_t v) { return (v + OR_PAD - 1) / OR_PAD * OR_PAD; }
size_t aligned_bytes(size_t n) { return (n + 255) / 256 * 256; }

struct OrStep {
    float a, b, c;
    int e_x, e_a, e_b;   // X, A and B are held times 2 to these
    bool lo;             // X is needed in two planes
    double most_b;       // B's largest eigenvalue
    int growth;          // see OrLoadArgs
};
struct OrPlan {
    int64_t mp, np, ldx, lda;
    int planes;                       // that POLY and APPLY multiply, and of A and B
    int gram_planes;                  // that GRAM multiplies
    bool iterate;                     // all steps in m x m matrices alone (or_iterate_kernel)
    int b_matrices;                   // that there is room for
    int64_t group;                    // matrices at a time
    size_t x_bytes, a_bytes, bytes;   // of one matrix: X (there are two), A (and B); all of them, and its partial sums
    int64_t tiles;                    // of 128, of the product with the most of them
    OrStep steps[OR_MAX_STEPS];
};

// The exponent that brings values of up to `most` below 2^14.
int exponent_for(double most) { return 14 - (int)ceil(log2(std::max(most, 0x1p-40))); }

// What a step's polynomial a + b l + c l^2, l = x^2, does to singular values x of up to s: its largest magnitude, and the
// largest singular value that follows.
struct OrRange {
    double most_b, most_x;
};
OrRange range_of(double A, double B, double C, double s) {
    const double l1 = s * s;
    auto poly = [&](double l) { return fabs(A + B * l + C * l * l); };
    auto next = [&](double l) { return sqrt(l) * poly(l); };
    OrRange r{std::max(poly(0.0), poly(l1)), next(l1)};
    auto at = [&](double l, auto f, double& most) {
        if (l > 0.0 && l < l1) most = std::max(most, f(l));
    };
    if (C != 0.0) {
        at(-B / (2.0 * C), poly, r.most_b);
        const double disc = 9.0 * B * B - 20.0 * A * C;
        if (disc >= 0.0) {
            at((-3.0 * B + sqrt(disc)) / (10.0 * C), next, r.most_x);
            at((-3.0 * B - sqrt(disc)) / (10.0 * C), next, r.most_x);
        }
    } else if (B != 0.0) {
        at(-A / (3.0 * B), next, r.most_x);
    }
    return r;
}

// Singular values of X_k lie in [0, s]; every step's polynomial says where those of X_{k+1} do.  What is held lies in
// [0, held]: an operand's rounding lifts a singular value by up to `rounding` of it, which polynomials that are steep there
// multiply, step after step (five that stay below 2 from 1 on make 3056 of 1.001).  That decides about exponents alone, not
// about what is taken, and up to OR_LIFT times: what is lifted higher is rounding errors, and the room for them would
// cost the others their bits.
int steps_of(const flce_orthogonalize_args& b, double rounding, OrStep* to) {
    double s = 1.0, held = 1.0, small = 1.0;   // small: what singular values far below 1 grow by at most
    int growth = 0;
    for (int k = 0; k < b.steps; ++k) {
        const float* p = !b.coefficients ? OR_USUAL : b.coefficients + (b.per_step ? 3 * k : 0);
        for (int i = 0; i < 3; ++i)
            if (p[i] - p[i] != 0.0f) return FLCE_ERR_ARG;
        const OrRange lifted = range_of(p[0], p[1], p[2], held);
        growth = std::max(growth, (int)ceil(log2(small)) + exponent_for(held) - 14);   // (never less: they stay in range anyway)
        to[k] = {p[0], p[1], p[2], exponent_for(held), exponent_for(held * held), exponent_for(lifted.most_b), false, lifted.most_b, growth};
        small = std::min(std::max(small * lifted.most_b * (1.0 + rounding), 0x1p-1000), 0x1p1000);
        s = std::max(range_of(p[0], p[1], p[2], s).most_x, 0x1p-20);
        if (!(s <= OR_MAX_NORM)) return FLCE_ERR_ARG;
        held = std::min(std::max(lifted.most_x, 0x1p-20) * (1.0 + rounding), OR_LIFT * s);
    }
    float grows = 1.0f;   // what an error of X_k may be multiplied by in what follows
    for (int k = b.steps - 1; k >= 0; --k) {
        grows = std::min(grows * std::max(1.0f, fabsf(to[k].a)), 1e30f);
        to[k].lo = k > 0 && grows > OR_CARRY;
    }
    return FLCE_OK;
}

// Workspace of a group: its matrices' and the sums of K ranges.
size_t part_bytes(const OrPlan& p, int64_t group) {
    return (size_t)std::min(OR_SLOTS_128, OR_MAX_RANGES * p.tiles * group) * 128 * 128 * sizeof(float);
}
size_t group_bytes(const OrPlan& p, int64_t group) { return part_bytes(p, group) + (size_t)group * p.bytes; }

int or_plan(const flce_orthogonalize_args* args, int n, OrPlan* p) {
    if (!args) return FLCE_ERR_NULL;
    const flce_orthogonalize_args& b = *args;
    if (b.size != sizeof(flce_orthogonalize_args) || n < 0) return FLCE_ERR_ARG;
    if (b.dtype != FLCE_F32 && b.dtype != FLCE_BF16) return FLCE_ERR_DTYPE;
    if (b.rows < 1 || b.rows > OR_MAX_DIM || b.cols < 1 || b.cols > OR_MAX_DIM) return FLCE_ERR_SHAPE;
    if (b.steps < 1 || b.steps > OR_MAX_STEPS || (b.per_step != 0 && b.per_step != 1)) return FLCE_ERR_ARG;
    if (b.scale - b.scale != 0.0f || !(b.eps >= 0.0f) || b.eps - b.eps != 0.0f) return FLCE_ERR_ARG;
    p->mp = padded(std::min(b.rows, b.cols));
    p->np = padded(std::max(b.rows, b.cols));
    if (p->mp * p->np > OR_MAX_ELEMENTS) return FLCE_ERR_SHAPE;
    p->gram_planes = b.dtype == FLCE_F32 ? 2 : 1;
    FLCE_TRY(steps_of(b, p->gram_planes == 2 ? 0x1p-20 : 0x1p-10, p->steps));
    p->planes = b.dtype == FLCE_F32 || p->mp <= OR_SMALL ? 2 : 1;
    p->ldx = 2 * p->np;
    p->lda = p->planes * p->mp;
    p->x_bytes = aligned_bytes((size_t)(p->mp * p->ldx) * sizeof(f16_t));
    p->a_bytes = aligned_bytes((size_t)(p->mp * p->lda) * sizeof(f16_t));
    double growth = 1.0;
    for (int k = 0; k + 1 < b.steps; ++k) growth = std::min(growth * std::max(1.0, p->steps[k].most_b * p->steps[k].most_b), 1e30);
    const bool small = b.dtype == FLCE_BF16 && p->mp <= OR_ITERATE_MOST;
    p->iterate = small && b.steps <= OR_ITERATE_STEPS && growth <= OR_ITERATE_GROWTH;
    p->b_matrices = small ? 1 + OR_ITERATE_STEPS : 2;   // (whatever the steps are)
    p->bytes = 2 * p->x_bytes + (1 + p->b_matrices) * p->a_bytes + aligned_bytes(OR_NORM_BLOCKS * sizeof(double)) +
               aligned_bytes(OR_MAX_STEPS * sizeof(double));
    p->tiles = ((p->mp + 127) / 128) * ((p->np + 127) / 128);
    // Matrices at a time: until the launch with the fewest tiles has several rounds of them.
    const int64_t t = (p->mp + 255) / 256, tiles = t * (t + 1) / 2;
    p->group = std::max<int64_t>(1, std::min<int64_t>({n, OR_MATRICES, (OR_ROUNDS + tiles - 1) / tiles}));
    return FLCE_OK;
}

// A product of all matrices of a group.  Tiles of 128 that leave CUs idle are cut into ranges of K, at most as many as
// run at a time.
template <int PRODUCT, int PL, int OUT, typename OutT, bool TALL>
int launch_product(OrArgs& a, hipStream_t s) {
    constexpr bool SYMMETRIC = PRODUCT <= OR_MULTIPLY;
    auto tiles_of = [&](int64_t tile) {
        a.tiles_m = (int)((a.mp + tile - 1) / tile);
        a.tiles_n = SYMMETRIC ? a.tiles_m : (int)((a.np + tile - 1) / tile);
        const int64_t tiles = SYMMETRIC ? (int64_t)a.tiles_m * (a.tiles_m + 1) / 2 : (int64_t)a.tiles_m * a.tiles_n;
        a.tiles = (int)tiles;
        return tiles * a.count;
    };
    auto grid = [](int64_t total) { return dim3((unsigned)((total + FG_XCDS - 1) / FG_XCDS * FG_XCDS)); };
    constexpr bool PAIRED = PRODUCT == OR_MULTIPLY;    // only of two steps at a time: its launches fill the chip (run_group)
    if constexpr (PRODUCT != OR_GRAM || PL == OUT) {   // (else OR_MATRICES tiles of 256 at most: see OR_SMALL)
        const int64_t large = tiles_of(256);
        if ((PAIRED && PL == 1) || large >= (PL == 2 ? OR_TILES_256_PLANES : OR_TILES_256)) {
            hipLaunchKernelGGL((or_product_kernel<PRODUCT, PL, OUT, 256, OutT, TALL, OR_WHOLE>), grid(large), dim3(FG_THREADS), 0, s, a);
            HIP_TRY(hipGetLastError());
            return FLCE_OK;
        }
    }
    if constexpr (!PAIRED || PL == 2) {
        const int64_t total = tiles_of(128);
        if constexpr (!PAIRED) {
            const int64_t steps = (PRODUCT == OR_GRAM ? a.np : a.mp) / FG_BK, turns = steps * (PL == 2 ? 3 : 1);
            a.ranges = (int)std::min({OR_MAX_RANGES, OR_SLOTS_128 / total, turns / OR_RANGE_STEPS, steps});
            if (a.ranges > 1 && turns - turns / a.ranges >= OR_SAVED_STEPS) {
                hipLaunchKernelGGL((or_product_kernel<PRODUCT, PL, OUT, 128, OutT, TALL, OR_RANGES>), grid(total * a.ranges), dim3(FG_THREADS), 0, s, a);
                HIP_TRY(hipGetLastError());
                hipLaunchKernelGGL((or_product_kernel<PRODUCT, PL, OUT, 128, OutT, TALL, OR_JOIN>), grid(2 * total), dim3(FG_THREADS), 0, s, a);
                HIP_TRY(hipGetLastError());
                return FLCE_OK;
            }
        }
        hipLaunchKernelGGL((or_product_kernel<PRODUCT, PL, OUT, 128, OutT, TALL, OR_WHOLE>), grid(total), dim3(FG_THREADS), 0, s, a);
        HIP_TRY(hipGetLastError());
    }
    return FLCE_OK;
}

// What or_iterate_kernel needs for it->steps steps; returns the exponent that Q is held with.
int iterate_args(const OrPlan& p, OrIterateArgs* it) {
    const OrStep* steps = p.steps;
    const int last = it->steps - 1;
    double most_q = steps[last].most_b;
    int e_q = steps[last].e_b;
    for (int i = last; i >= 0; --i) {
        const OrStep& st = steps[i];
        it->square[i] = ldexpf(st.c, st.e_b - 2 * st.e_a);
        it->linear[i] = ldexpf(st.b, st.e_b - st.e_a);
        it->diagonal[i] = ldexpf(st.a, st.e_b);
        if (i == last) continue;
        const int e_t = exponent_for(st.most_b * ldexp(1.0, 14 - st.e_a));   // (A's eigenvalues: at most 2^(14 - e_a))
        it->t[i] = ldexpf(1.0f, e_t - st.e_b - st.e_a);
        it->next[i] = ldexpf(1.0f, steps[i + 1].e_a - e_t - st.e_b);
        most_q *= st.most_b;
        const int e = exponent_for(most_q);
        it->q[i] = ldexpf(1.0f, e - e_q - st.e_b);
        e_q = e;
    }
    return e_q;
}

// `count` matrices, in the workspace from ws on.  GP: planes that GRAM multiplies, PL: that the others do.
template <typename T, int GP, int PL>
int run_group(const flce_orthogonalize_args& b, const OrPlan& p, const void* const* in, void* const* out, int count, char* ws, hipStream_t s) {
    const bool tall = b.rows > b.cols;
    size_t at = part_bytes(p, count);
    auto take = [&](size_t bytes) {
        char* here = ws + at;
        at += aligned_bytes(bytes);
        return here;
    };
    f16_t* X[2];
    for (f16_t*& x : X) x = reinterpret_cast<f16_t*>(take(count * p.x_bytes));
    f16_t* A = reinterpret_cast<f16_t*>(take(count * p.a_bytes));
    f16_t* B = reinterpret_cast<f16_t*>(take(count * p.b_matrices * p.a_bytes));
    OrLoadArgs l{};
    l.partial = reinterpret_cast<double*>(take(count * OR_NORM_BLOCKS * sizeof(double)));
    l.size = reinterpret_cast<double*>(take(count * OR_MAX_STEPS * sizeof(double)));
    l.X = X[0];
    l.stride_x = (int64_t)(p.x_bytes / sizeof(f16_t));
    l.rows = (int)b.rows;
    l.cols = (int)b.cols;
    l.mp = (int)p.mp;
    l.np = (int)p.np;
    l.ldx = (int)p.ldx;
    l.planes = PL;
    l.exponent = p.steps[0].e_x;
    l.eps = b.eps;
    l.steps = b.steps;
    for (int k = 0; k < b.steps; ++k) l.growth[k] = (int16_t)p.steps[k].growth;
    for (int i = 0; i < count; ++i) l.in[i] = in[i];
    hipLaunchKernelGGL((or_norm_kernel<T>), dim3(OR_NORM_BLOCKS, (unsigned)count), dim3(256), 0, s, l);
    HIP_TRY(hipGetLastError());
    const dim3 blocks((unsigned)(p.mp / 64 * (p.np / 64)), (unsigned)count);
    if (tall) hipLaunchKernelGGL((or_load_kernel<T, true>), blocks, dim3(256), 0, s, l);
    else hipLaunchKernelGGL((or_load_kernel<T, false>), blocks, dim3(256), 0, s, l);
    HIP_TRY(hipGetLastError());
    OrArgs a{};
    a.A = A;
    a.B = B;
    a.stride_x = l.stride_x;
    a.stride_a = (int64_t)(p.a_bytes / sizeof(f16_t));
    a.mp = l.mp;
    a.np = l.np;
    a.ldx = (int)p.ldx;
    a.lda = (int)p.lda;
    a.count = count;
    a.rows = l.rows;
    a.cols = l.cols;
    a.part = reinterpret_cast<float*>(ws);
    a.size = l.size;
    for (int i = 0; i < count; ++i) a.out[i] = out[i];
    // Small matrices: all steps between the first and the last product with X in one launch.
    if constexpr (GP == 1 && PL == 2) {
        if (p.iterate) {
            a.X = X[0];
            a.to = A;
            a.alpha = ldexpf(1.0f, p.steps[0].e_a - 2 * p.steps[0].e_x);
            FLCE_TRY((launch_product<OR_GRAM, GP, PL, float, false>(a, s)));
            OrIterateArgs it{};
            it.A = A;
            it.Q = B;
            it.B = B + count * a.stride_a;
            it.stride_a = a.stride_a;
            it.lda = a.lda;
            it.steps = b.steps;
            const int e_q = iterate_args(p, &it);
            if (p.mp == 64) hipLaunchKernelGGL((or_iterate_kernel<64>), dim3((unsigned)count), dim3(256), 0, s, it);
            else hipLaunchKernelGGL((or_iterate_kernel<128>), dim3((unsigned)count), dim3(256), 0, s, it);
            HIP_TRY(hipGetLastError());
            a.B = B;
            a.alpha = ldexpf(b.scale, -e_q - p.steps[0].e_x);
            return tall ? launch_product<OR_LAST, PL, 2, T, true>(a, s) : launch_product<OR_LAST, PL, 2, T, false>(a, s);
        }
    }
    // Two steps at a time where launches fill the chip and X is long (see orthogonalize.h), never twice in a row.
    const int64_t t = (p.mp + 255) / 256;
    const bool pairs = p.np >= OR_PAIR_LENGTH * p.mp && t * (t + 1) / 2 * count >= OR_TILES_256;
    f16_t* spare = B + count * a.stride_a;
    bool paired = false;
    for (int k = 0, x = 0; k < b.steps; x ^= 1) {
        const OrStep* st = &p.steps[k];
        const int first_x = st->e_x;
        const bool lo = st->lo;
        a.step = k;
        a.X = X[x];
        a.A = A;
        a.to = A;
        a.alpha = ldexpf(1.0f, st->e_a - 2 * st->e_x);
        a.beta = 0.0f;
        a.add_lo = 0;
        FLCE_TRY((launch_product<OR_GRAM, GP, PL, float, false>(a, s)));
        auto poly = [&](f16_t* to) {
            a.to = to;
            a.alpha = ldexpf(st->c, st->e_b - 2 * st->e_a);
            a.beta = ldexpf(st->b, st->e_b - st->e_a);
            a.diagonal = ldexpf(st->a, st->e_b);
            return launch_product<OR_POLY, PL, PL, float, false>(a, s);
        };
        auto multiply = [&](const f16_t* left, const f16_t* right, f16_t* to, int exponent) {
            a.A = left;
            a.B = right;
            a.to = to;
            a.alpha = ldexpf(1.0f, exponent);
            return launch_product<OR_MULTIPLY, PL, PL, float, false>(a, s);
        };
        FLCE_TRY(poly(B));
        a.B = B;
        int e_b = st->e_b;
        float carried = st->a;
        paired = pairs && !paired && k + 1 < b.steps && st->most_b <= OR_PAIR_GROWTH;
        if (paired) {
            const OrStep* second = st + 1;
            const int e_t = exponent_for(st->most_b * ldexp(1.0, 14 - st->e_a));   // (A's eigenvalues: at most 2^(14 - e_a))
            FLCE_TRY(multiply(B, A, spare, e_t - st->e_b - st->e_a));
            FLCE_TRY(multiply(spare, B, A, second->e_a - e_t - st->e_b));
            const double most = st->most_b * second->most_b;
            st = second;
            a.A = A;
            FLCE_TRY(poly(spare));
            const int e = exponent_for(most);
            FLCE_TRY(multiply(spare, B, A, e - st->e_b - e_b));
            a.B = A;
            e_b = e;
            carried *= st->a;
            ++k;
        }
        ++k;
        const bool last = k == b.steps;
        a.next = k;
        const float scale = last ? b.scale : ldexpf(1.0f, p.steps[k].e_x);
        a.to = X[x ^ 1];
        a.alpha = ldexpf(scale, -e_b - first_x);
        a.beta = ldexpf(scale * carried, -first_x);
        a.add_lo = PL == 1 && lo;
        a.put_lo = !last && p.steps[k].lo;
        if (!last) FLCE_TRY((launch_product<OR_APPLY, PL, 2, float, false>(a, s)));
        else if (tall) FLCE_TRY((launch_product<OR_LAST, PL, 2, T, true>(a, s)));
        else FLCE_TRY((launch_product<OR_LAST, PL, 2, T, false>(a, s)));
    }
    return FLCE_OK;
}

}  // namespace

extern "C" {

int flce_orthogonalize(const void* const* in, void* const* out, int n_matrices, const flce_orthogonalize_args* args, void* stream) {
    OrPlan p;
    FLCE_TRY(or_plan(args, n_matrices, &p));
    const flce_orthogonalize_args& b = *args;
    if (!n_matrices) return FLCE_OK;
    if (!in) return FLCE_ERR_NULL;
    if (!out) out = const_cast<void* const*>(in);
    const size_t es = elem(b.dtype), bytes = (size_t)b.rows * (size_t)b.cols * es;
    for (int i = 0; i < n_matrices; ++i) {
        if (!in[i] || !out[i]) return FLCE_ERR_NULL;
        if (!aligned(in[i], es) || !aligned(out[i], es)) return FLCE_ERR_ALIGN;
    }
    if (b.workspace && !aligned(b.workspace, 256)) return FLCE_ERR_ALIGN;
    // the workspace: for a group, or for as many of its matrices as there is room for
    hipStream_t s = static_cast<hipStream_t>(stream);
    char* ws = static_cast<char*>(b.workspace);
    size_t cap = SIZE_MAX;
    if (ws) {
        cap = b.workspace_bytes;
    } else {
        size_t lent = 0;
        FLCE_TRY(shared_workspace_lent(&lent));
        if (lent) cap = lent;
    }
    while (p.group > 1 && group_bytes(p, p.group) > cap) --p.group;
    if (group_bytes(p, p.group) > cap) return FLCE_ERR_WORKSPACE;
    while (!ws) {
        const int rc = shared_workspace(group_bytes(p, p.group), &ws, s, p.group == 1);
        if (rc == FLCE_OK) break;
        if (rc != FLCE_ERR_WORKSPACE || p.group == 1) return rc;
        p.group = (p.group + 1) / 2;
    }
    Piece* pieces = new (std::nothrow) Piece[2 * (size_t)n_matrices + 1];
    if (!pieces) return FLCE_ERR_WORKSPACE;
    size_t k = 0;
    for (int i = 0; i < n_matrices; ++i) {
        const uintptr_t w = reinterpret_cast<uintptr_t>(out[i]), r = reinterpret_cast<uintptr_t>(in[i]);
        pieces[k++] = {w, w + bytes, true};
        if (r != w) pieces[k++] = {r, r + bytes, false};
    }
    pieces[k++] = {reinterpret_cast<uintptr_t>(ws), reinterpret_cast<uintptr_t>(ws) + group_bytes(p, p.group), true};
    const bool shared = written_twice(pieces, k);
    delete[] pieces;
    if (shared) return FLCE_ERR_ARG;
    for (int i = 0; i < n_matrices; i += (int)p.group) {
        const int count = (int)std::min<int64_t>(p.group, n_matrices - i);
        FLCE_TRY(p.gram_planes == 2 ? (run_group<float, 2, 2>(b, p, in + i, out + i, count, ws, s))
                 : p.planes == 2    ? (run_group<bf16_t, 1, 2>(b, p, in + i, out + i, count, ws, s))
                                    : (run_group<bf16_t, 1, 1>(b, p, in + i, out + i, count, ws, s)));
    }
    return FLCE_OK;
}

size_t flce_orthogonalize_workspace_bytes(int n_matrices, const flce_orthogonalize_args* args) {
    OrPlan p;
    return or_plan(args, n_matrices, &p) == FLCE_OK && n_matrices ? group_bytes(p, p.group) : 0;
}

}  // extern "C"
