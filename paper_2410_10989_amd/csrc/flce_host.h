// Host-side helpers that the library's translation units share.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/flce.h"

#define HIP_TRY(expr)                          \
    do {                                       \
        if ((expr) != hipSuccess) {            \
            (void)hipGetLastError();           \
            return FLCE_ERR_HIP;               \
        }                                      \
    } while (0)

#define FLCE_TRY(expr)                 \
    do {                               \
        const int rc_ = (expr);        \
        if (rc_ != FLCE_OK) return rc_; \
    } while (0)

namespace flce {

constexpr int64_t MAX_DIM = (int64_t)1 << 30;   // per-dimension limit, keeps int tile math safe

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// A strided matrix in memory.
struct Span {
    const char* p;
    size_t pitch, width;   // bytes from row to row, bytes of a row
    int64_t rows;
};
inline Span span(const void* p, int64_t ld, int64_t rows, int64_t H, size_t es) {
    return {static_cast<const char*>(p), (size_t)ld * es, (size_t)H * es, rows};
}
// Whether two of them share a byte.  A single row may lie between the rows of the other, column windows of one wider
// buffer (equal pitch) may interleave; with different pitches any common stretch of addresses counts.
inline bool overlap(const Span& a, const Span& b) {
    if (!a.p || !b.p) return false;
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
    const uintptr_t a1 = a0 + (a.rows - 1) * a.pitch + a.width, b1 = b0 + (b.rows - 1) * b.pitch + b.width;
    if (a1 <= b0 || b1 <= a0) return false;
    if (a.rows == 1 || b.rows == 1) {
        const Span &m = a.rows == 1 ? b : a, &v = a.rows == 1 ? a : b;
        const uintptr_t m0 = reinterpret_cast<uintptr_t>(m.p), v0 = reinterpret_cast<uintptr_t>(v.p);
        if (v0 <= m0) return true;
        const size_t off = (v0 - m0) % m.pitch;   // from the row that begins before v
        return off < m.width || ((int64_t)((v0 - m0) / m.pitch) + 1 < m.rows && off + v.width > m.pitch);
    }
    if (a.pitch != b.pitch) return true;
    const size_t off = b0 >= a0 ? (b0 - a0) % a.pitch : (a.pitch - (a0 - b0) % a.pitch) % a.pitch;
    return off < a.width || a.pitch - off < b.width;
}
inline bool same(const Span& a, const Span& b) { return a.p == b.p && (a.pitch == b.pitch || a.rows == 1); }

// Stretches of memory that a call reads or writes; whether one that is written shares a byte with any other.
struct Piece {
    uintptr_t begin, end;
    bool write;
};
inline bool written_twice(Piece* pieces, size_t n) {
    std::sort(pieces, pieces + n, [](const Piece& a, const Piece& b) { return a.begin < b.begin; });
    uintptr_t any_end = 0, write_end = 0;   // of the pieces so far
    bool found = false;
    for (size_t i = 0; i < n; ++i) {
        if (pieces[i].begin < (pieces[i].write ? any_end : write_end)) found = true;
        any_end = std::max(any_end, pieces[i].end);
        if (pieces[i].write) write_end = std::max(write_end, pieces[i].end);
    }
    return found;
}

// The current device's shared workspace (see Scratch memory in flce.h), at least `need` bytes of it, for a call on s.
// last: the caller has no plan that needs less (without one, an allocation that found too little memory is not tried
// again every call).
int shared_workspace(size_t need, char** out, hipStream_t s, bool last = true);
// Bytes of the buffer lent to the current device (flce_set_workspace), 0 if there is none.
int shared_workspace_lent(size_t* bytes);

}  // namespace flce
