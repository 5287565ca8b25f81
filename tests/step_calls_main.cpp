// The launches of the operators of a step with a tied embedding, on a HIP runtime that is stood in for: memory comes from
// the host (up to a limit that a scenario sets), launches are looked at and do nothing.
// Usage: step_calls <libflce.so> <scenario>; prints "ok" and returns 0, or says what failed.
#include <dlfcn.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <vector>

#include "../include/flce.h"

struct Dim3 {
    unsigned x, y, z;
};
namespace {
size_t g_limit = (size_t)1 << 40, g_most = 0;   // a larger hipMalloc finds too little memory; the largest that did not
int g_launches = 0, g_failed = 0;
struct Launch {
    Dim3 grid, block;
} g_pushed;

#define CHECK(cond)                                              \
    do {                                                         \
        if (!(cond)) {                                           \
            printf("line %d: %s does not hold\n", __LINE__, #cond); \
            ++g_failed;                                          \
        }                                                        \
    } while (0)
}   // namespace

extern "C" {
int hipGetDevice(int* d) { *d = 0; return 0; }
int hipGetLastError() { return 0; }
int hipDeviceSynchronize() { return 0; }
int hipMalloc(void** p, size_t n) {
    if (n > g_limit) return 2;
    g_most = std::max(g_most, n);
    static char* next = reinterpret_cast<char*>((uintptr_t)3 << 45);   // (never touched)
    *p = next;
    next += (n + 4095) / 4096 * 4096;
    return 0;
}
int hipFree(void*) { return 0; }
int hipStreamIsCapturing(void*, int* status) { *status = 0; return 0; }
int hipLaunchKernel(const void*, Dim3 grid, Dim3 block, void**, size_t, void*) {
    ++g_launches;
    // what the runtime takes: 1 .. 1024 threads to a workgroup, below 2^32 along each direction
    const uint64_t threads = (uint64_t)block.x * block.y * block.z;
    CHECK(threads >= 1 && threads <= 1024);
    CHECK(grid.x >= 1 && grid.y >= 1 && grid.z >= 1 && grid.y <= 65535 && grid.z <= 65535);
    CHECK((uint64_t)grid.x * block.x < ((uint64_t)1 << 32));
    return 0;
}
int __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t, void*) {
    g_pushed = {grid, block};
    return 0;
}
int __hipPopCallConfiguration(Dim3* g, Dim3* b, size_t* m, void** s) {
    *g = g_pushed.grid;
    *b = g_pushed.block;
    *m = 0;
    *s = nullptr;
    return 0;
}
void** __hipRegisterFatBinary(const void*) { static void* handle; return &handle; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void*, char*, const char*, unsigned, void*, void*, void*, void*, int*) {}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
int hipGetSymbolAddress(void** p, const void* s) { *p = const_cast<void*>(s); return 0; }
int hipEventCreate(void**) { return 0; }
int hipEventDestroy(void*) { return 0; }
int hipEventRecord(void*, void*) { return 0; }
int hipEventSynchronize(void*) { return 0; }
int hipEventElapsedTime(float* ms, void*, void*) { *ms = 0; return 0; }
}

namespace {
#define ENTRIES(E) \
    E(flce_embedding_fwd) E(flce_embedding_bwd) E(flce_embedding_workspace_bytes) E(flce_layer_norm_fwd) E(flce_layer_norm_bwd) \
    E(flce_layer_norm_workspace_bytes) E(flce_orthogonalize) E(flce_orthogonalize_workspace_bytes) E(flce_release_workspace)
#define ENTRY(name) decltype(&::name) name##_;
struct Library {
    ENTRIES(ENTRY)
} L;
#undef ENTRY

// Addresses that are never touched: operands of the calls.
char* operand(int i) { return reinterpret_cast<char*>((uintptr_t)1 << 44) + ((uintptr_t)i << 38); }

const int64_t SIZES[] = {1, 2, 63, 64, 65, 1000, 4096, 65537, (int64_t)1 << 20, ((int64_t)1 << 24) + 3, (int64_t)1 << 30, ((int64_t)1 << 31) - 1};
bool too_large(int64_t n) { return n > (int64_t)1 << 30; }

void embeddings() {
    for (int dtype : {FLCE_F32, FLCE_BF16})
        for (int64_t rows : SIZES)
            for (int64_t V : SIZES)
                for (int64_t H : {1, 7, 64, 513, 4096, 16384}) {
                    const int64_t es = dtype == FLCE_F32 ? 4 : 2;
                    if (rows * H > ((int64_t)1 << 38) / es || V * H > ((int64_t)1 << 38) / es) continue;
                    flce_embedding b{};
                    b.size = sizeof b;
                    b.rows = rows;
                    b.V = V;
                    b.H = H;
                    b.dtype = dtype;
                    b.ignore_index = -100;
                    b.scale = 1.0f;
                    const int64_t* tokens = reinterpret_cast<const int64_t*>(operand(1));
                    int n = g_launches;
                    if (too_large(rows) || too_large(V)) {
                        CHECK(L.flce_embedding_fwd_(operand(0), tokens, &b, operand(2), nullptr) == FLCE_ERR_SHAPE);
                        CHECK(L.flce_embedding_bwd_(operand(0), tokens, &b, operand(2), nullptr) == FLCE_ERR_SHAPE);
                        CHECK(L.flce_embedding_workspace_bytes_(&b) == 0 && g_launches == n);
                        continue;
                    }
                    CHECK(L.flce_embedding_fwd_(operand(0), tokens, &b, operand(2), nullptr) == FLCE_OK && g_launches == n + 1);
                    for (b.accumulate = 0; b.accumulate < 2; ++b.accumulate) {
                        n = g_launches;
                        const size_t bytes = L.flce_embedding_workspace_bytes_(&b);
                        CHECK(bytes > 0 && bytes < ((size_t)1 << 40));
                        const int rc = L.flce_embedding_bwd_(operand(0), tokens, &b, operand(2), nullptr);
                        CHECK(rc == FLCE_OK && g_launches >= n + 2 && g_launches <= n + 3);
                    }
                }
}

void layer_norms() {
    for (int dtype : {FLCE_F32, FLCE_BF16})
        for (int64_t rows : SIZES)
            for (int64_t H : {(int64_t)1, (int64_t)7, (int64_t)8, (int64_t)128, (int64_t)513, (int64_t)1025, (int64_t)2304, (int64_t)4097,
                              (int64_t)16384, (int64_t)16385, ((int64_t)1 << 24)}) {
                if (rows * H > (int64_t)1 << 36) continue;
                flce_layer_norm b{};
                b.size = sizeof b;
                b.rows = rows;
                b.H = H;
                b.dtype = dtype;
                b.eps = 1e-5f;
                int n = g_launches;
                if (too_large(rows)) {
                    CHECK(L.flce_layer_norm_fwd_(operand(0), operand(1), operand(2), operand(3), &b, operand(4), operand(5), nullptr) == FLCE_ERR_SHAPE);
                    CHECK(L.flce_layer_norm_bwd_(operand(0), operand(1), operand(2), operand(3), &b, operand(4), operand(5), operand(6), nullptr) == FLCE_ERR_SHAPE);
                    CHECK(L.flce_layer_norm_workspace_bytes_(&b) == 0 && g_launches == n);
                    continue;
                }
                CHECK(L.flce_layer_norm_fwd_(operand(0), operand(1), operand(2), operand(3), &b, operand(4), operand(5), nullptr) == FLCE_OK);
                CHECK(g_launches == n + 1);
                n = g_launches;
                CHECK(L.flce_layer_norm_bwd_(operand(0), operand(1), operand(2), operand(3), &b, operand(4), operand(5), operand(6), nullptr) == FLCE_OK);
                CHECK(g_launches >= n + 1 && g_launches <= n + 2);
            }
}

int orthogonalize(int count, int64_t rows, int64_t cols, int dtype, int steps = 5) {
    flce_orthogonalize_args b{};
    b.size = sizeof b;
    b.rows = rows;
    b.cols = cols;
    b.dtype = dtype;
    b.steps = steps;
    b.scale = 1.0f;
    b.eps = 1e-7f;
    std::vector<const void*> in;
    std::vector<void*> out;
    const size_t bytes = ((size_t)rows * (size_t)cols * 4 + 255) / 256 * 256;
    for (int i = 0; i < count; ++i) {
        in.push_back(operand(0) + i * bytes);
        out.push_back(operand(16) + i * bytes);
    }
    return L.flce_orthogonalize_(in.data(), out.data(), count, &b, nullptr);
}

void orthogonalisations() {
    for (int dtype : {FLCE_F32, FLCE_BF16})
        for (int count : {1, 2, 119, 120, 121, 1000})
            for (int64_t rows : {1, 64, 65, 128, 129, 300, 1024, 16384, 1 << 20})
                for (int64_t cols : {1, 64, 100, 256, 257, 2048, 16384, 1 << 20}) {
                    const int64_t all = (rows + 63) / 64 * 64 * ((cols + 63) / 64 * 64);
                    const int n = g_launches, rc = orthogonalize(count, rows, cols, dtype);
                    if (all > (int64_t)1 << 28) CHECK(rc == FLCE_ERR_SHAPE && g_launches == n);
                    else CHECK(rc == FLCE_OK && g_launches > n);
                }
}

// Fewer matrices at a time where memory is short, and an error, without a launch, where it is too short for one.
void orthogonalisation_with_little_memory() {
    flce_orthogonalize_args b{};
    b.size = sizeof b;
    b.rows = 1024;
    b.cols = 768;
    b.dtype = FLCE_BF16;
    b.steps = 5;
    b.scale = 1.0f;
    const size_t one = L.flce_orthogonalize_workspace_bytes_(1, &b), many = L.flce_orthogonalize_workspace_bytes_(40, &b);
    CHECK(one > 0 && many > 3 * one);
    int before = 0;
    for (size_t room : {many, many / 3, 3 * one, one}) {
        CHECK(L.flce_release_workspace_() == FLCE_OK);
        g_limit = room;
        g_most = 0;
        const int n = g_launches;
        CHECK(orthogonalize(40, 1024, 768, FLCE_BF16) == FLCE_OK);
        CHECK(g_most <= room && g_launches - n > before);
        before = g_launches - n;
    }
    CHECK(L.flce_release_workspace_() == FLCE_OK);
    g_limit = one - 1;
    const int n = g_launches;
    CHECK(orthogonalize(40, 1024, 768, FLCE_BF16) == FLCE_ERR_WORKSPACE && g_launches == n);
}
}   // namespace

int main(int argc, char** argv) {
    if (argc != 3) return 2;
    void* lib = dlopen(argv[1], RTLD_NOW);
    if (!lib) {
        printf("%s\n", dlerror());
        return 2;
    }
#define ENTRY(name) L.name##_ = reinterpret_cast<decltype(L.name##_)>(dlsym(lib, #name));
    ENTRIES(ENTRY)
#undef ENTRY
    const struct {
        const char* name;
        void (*run)();
    } scenarios[] = {{"embeddings", embeddings}, {"layer_norms", layer_norms}, {"orthogonalisations", orthogonalisations},
                     {"orthogonalisation_with_little_memory", orthogonalisation_with_little_memory}};
    for (const auto& s : scenarios)
        if (!strcmp(s.name, argv[2])) {
            s.run();
            printf("%s\n", g_failed ? "failed" : "ok");
            fflush(stdout);
            _Exit(g_failed ? 1 : 0);
        }
    printf("no such scenario\n");
    return 2;
}
