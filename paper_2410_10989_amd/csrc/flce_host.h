// Host-side helpers that the library's translation units share.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

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

// The current device's shared workspace (see Scratch memory in flce.h), at least `need` bytes of it, for a call on s.
// last: the caller has no plan that needs less (without one, an allocation that found too little memory is not tried
// again every call).
int shared_workspace(size_t need, char** out, hipStream_t s, bool last = true);
// Bytes of the buffer lent to the current device (flce_set_workspace), 0 if there is none.
int shared_workspace_lent(size_t* bytes);

}  // namespace flce
