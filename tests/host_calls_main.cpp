// The library's host side on a HIP runtime that is stood in for: memory comes from the host (up to a limit that a
// scenario sets), launches are counted and do nothing.  What a call allocates, frees and launches can so be seen
// where there is no GPU.  Usage: host_calls <libflce.so> <scenario>; prints "ok" and returns 0, or says what failed.
#include <dlfcn.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <set>
#include <vector>

#include "../include/flce.h"

namespace {
size_t g_limit = (size_t)1 << 40;   // a larger hipMalloc finds too little memory
bool g_capturing = false;
int g_mallocs = 0, g_refused = 0, g_frees = 0, g_launches = 0;
std::set<void*> g_live;
std::vector<size_t> g_sizes;   // of the allocations that succeeded
constexpr int OUT_OF_MEMORY = 2;
}   // namespace

struct Dim3 {
    unsigned x, y, z;
};
extern "C" {
int hipGetDevice(int* d) { *d = 0; return 0; }
int hipGetLastError() { return 0; }
int hipDeviceSynchronize() { return 0; }
int hipMalloc(void** p, size_t n) {
    if (n > g_limit) {
        ++g_refused;
        return OUT_OF_MEMORY;
    }
    ++g_mallocs;
    g_sizes.push_back(n);
    *p = aligned_alloc(256, 256);   // (nothing is stored in it)
    g_live.insert(*p);
    return 0;
}
int hipFree(void* p) {
    ++g_frees;
    g_live.erase(p);
    return 0;   // (kept, so that no two allocations have one address)
}
int hipStreamIsCapturing(void*, int* status) { *status = g_capturing ? 1 : 0; return 0; }
int hipLaunchKernel(const void*, Dim3, Dim3, void**, size_t, void*) { ++g_launches; return 0; }
int __hipPushCallConfiguration(Dim3, Dim3, size_t, void*) { return 0; }
int __hipPopCallConfiguration(Dim3* g, Dim3* b, size_t* m, void** s) {
    *g = *b = {1, 1, 1};
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
#define ENTRY(name) decltype(&::name) name##_;
struct Library {
    ENTRY(flce_clip_grad_norm)
    ENTRY(flce_grad_norm)
    ENTRY(flce_block_norm_bwd)
    ENTRY(flce_block_norm_workspace_bytes)
    ENTRY(flce_cross_entropy_inplace)
    ENTRY(flce_release_workspace)
} L;
#undef ENTRY

int g_failed = 0;
#define CHECK(cond)                                              \
    do {                                                         \
        if (!(cond)) {                                           \
            printf("line %d: %s does not hold\n", __LINE__, #cond); \
            ++g_failed;                                          \
        }                                                        \
    } while (0)

// Addresses that are never touched: operands of the calls.
char* operand(int i) { return reinterpret_cast<char*>((uintptr_t)1 << 44) + ((uintptr_t)i << 36); }

int clip(int64_t count, void* stream = nullptr) {
    const void* grads[1] = {operand(0)};
    const int dtypes[1] = {FLCE_F32};
    return L.flce_clip_grad_norm_(grads, nullptr, &count, dtypes, 1, FLCE_NORM_2, 1.0f, reinterpret_cast<float*>(operand(1)),
                                  nullptr, 0, stream);
}

// Lists that one workgroup takes leave no partial results and need no memory for them.
void short_lists() {
    CHECK(clip(1000) == FLCE_OK && clip(16384) == FLCE_OK);
    float* norm = reinterpret_cast<float*>(operand(1));
    CHECK(L.flce_grad_norm_(nullptr, nullptr, nullptr, 0, FLCE_NORM_INF, norm, nullptr, 0, nullptr) == FLCE_OK);
    CHECK(g_mallocs == 0 && g_launches == 3);
    CHECK(clip(16385) == FLCE_OK);
    CHECK(g_mallocs == 1 && g_launches == 5);
}

int backward(int64_t rows, int64_t H, void* stream = nullptr) {   // both norms, a gate per channel
    flce_block_norm b{};
    b.size = sizeof b;
    b.rows = rows;
    b.H = H;
    b.dtype = FLCE_BF16;
    b.scale = 1.0f;
    b.eps = 1e-6f;
    auto at = [](int i) { return static_cast<void*>(operand(2 + i)); };
    return L.flce_block_norm_bwd_(at(0), at(1), at(2), at(3), at(4), at(5), at(6), &b, at(7), at(8), at(9), at(10), at(11),
                                  stream);
}

// Where the library's own memory cannot grow to the whole plan, the backward runs with fewer workgroups.
void backward_with_little_memory() {
    flce_block_norm b{};
    b.size = sizeof b;
    b.rows = 8192;
    b.H = 2048;
    b.dtype = FLCE_BF16;
    const size_t need = L.flce_block_norm_workspace_bytes_(&b);
    CHECK(need > ((size_t)4 << 20));
    g_limit = need / 3;
    CHECK(backward(8192, 2048) == FLCE_OK);
    CHECK(g_mallocs == 1 && g_refused > 0 && g_launches == 2 && g_sizes[0] <= g_limit && g_sizes[0] > need / 8);
    const int refused = g_refused;   // the next call does not try again
    CHECK(backward(8192, 2048) == FLCE_OK);
    CHECK(g_mallocs == 1 && g_refused == refused && g_launches == 4);
    CHECK(L.flce_release_workspace_() == FLCE_OK);
    g_limit = need;   // ... but behind a release it does
    CHECK(backward(8192, 2048) == FLCE_OK);
    CHECK(g_mallocs == 2 && g_sizes[1] == need && g_launches == 6);
    CHECK(L.flce_release_workspace_() == FLCE_OK);
    g_limit = 0;   // one workgroup that holds its rows in registers needs none
    CHECK(backward(8192, 2048) == FLCE_OK && g_launches == 7);
    g_launches = 0;
    CHECK(backward(8192, 20000) == FLCE_ERR_WORKSPACE && g_launches == 0);   // 12 H bytes at the least
    g_limit = 12 * 20000;
    CHECK(backward(8192, 20000) == FLCE_OK && g_sizes.back() == 12 * 20000);
}
// A captured graph holds the address of the shared workspace: it stays when a later call makes the workspace grow.
void workspace_of_a_captured_call() {
    void* const stream = operand(20);
    auto cross_entropy = [&](int64_t rows) {
        return L.flce_cross_entropy_inplace_(operand(0), reinterpret_cast<int64_t*>(operand(1)), rows, 512, 512, -100,
                                             FLCE_BF16, reinterpret_cast<float*>(operand(2)), stream);
    };
    // a call that is captured in each of the ways to use the workspace, then a larger one that is not
    int (*const clip_list)(void*) = [](void* s) { return clip(1 << 20, s); };
    int (*const norms)(void*) = [](void* s) { return backward(2048, 1024, s); };
    for (int kind = 0; kind < 3; ++kind) {
        auto small = [&] { return kind == 0 ? cross_entropy(4) : kind == 1 ? clip_list(stream) : norms(stream); };
        CHECK(L.flce_release_workspace_() == FLCE_OK && g_live.empty());
        CHECK(small() == FLCE_OK && g_live.size() == 1);
        void* const first = *g_live.begin();
        g_capturing = true;
        CHECK(small() == FLCE_OK && g_live.size() == 1);
        g_capturing = false;
        CHECK(backward(16384, 8192, stream) == FLCE_OK);
        CHECK(g_live.size() == 2 && g_live.count(first));
        CHECK(backward(16384, 16000, stream) == FLCE_OK);   // the second one has not been captured: it goes
        CHECK(g_live.size() == 2 && g_live.count(first));
        g_capturing = true;
        CHECK(backward(16384, 16000, stream) == FLCE_OK);
        g_capturing = false;
        CHECK(backward(16384, 40000, stream) == FLCE_OK);
        CHECK(g_live.size() == 3 && g_live.count(first));
        g_capturing = true;
        CHECK(backward(16384, 40000, stream) == FLCE_OK);
        g_capturing = false;
        g_limit = 0;   // (what could not be outgrown goes on serving, with fewer workgroups)
        CHECK(backward(16384, 60000, stream) == FLCE_OK && g_live.size() == 3);
        g_limit = (size_t)1 << 40;
        CHECK(L.flce_release_workspace_() == FLCE_OK && g_live.empty());
    }
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
    ENTRY(flce_clip_grad_norm)
    ENTRY(flce_grad_norm)
    ENTRY(flce_block_norm_bwd)
    ENTRY(flce_block_norm_workspace_bytes)
    ENTRY(flce_cross_entropy_inplace)
    ENTRY(flce_release_workspace)
#undef ENTRY
    const struct {
        const char* name;
        void (*run)();
    } scenarios[] = {{"short_lists", short_lists}, {"backward_with_little_memory", backward_with_little_memory},
                     {"workspace_of_a_captured_call", workspace_of_a_captured_call}};
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
