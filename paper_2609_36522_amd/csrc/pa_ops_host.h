// Host helpers of the operators' entry points (paraanya_ops.cpp, paraanya_block_ops.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "pa_host.h"
#include "pa_ops.h"

namespace pa {

inline size_t round256(size_t n) { return (n + 255) / 256 * 256; }

inline int element_size(int dtype) { return dtype == PA_F32 ? 4 : 2; }

inline bool misaligned(const void* p, int size) { return reinterpret_cast<uintptr_t>(p) % size != 0; }

inline int check_workspace(const void* ws, size_t have, size_t need, const char* what = "workspace") {
    if (need == 0) return PA_OK;
    if (!ws) return fail(PA_ERR_INVALID_ARG, "%s is NULL (%zu bytes needed)", what, need);
    if (misaligned(ws, 256)) return fail(PA_ERR_INVALID_ARG, "%s must be 256-byte aligned", what);
    if (have < need) return fail(PA_ERR_INVALID_ARG, "%s of %zu bytes too small: %zu needed", what, have, need);
    return PA_OK;
}

inline int launched(hipError_t e, const char* what) { return e == hipSuccess ? PA_OK : hip_fail(e, what); }

// No C++ exception (std::bad_alloc of an error text) crosses the C ABI.
template <class F>
int guarded(F f) noexcept {
    try {
        return f();
    } catch (...) {
        return PA_ERR_OOM;
    }
}

// Parts of a workspace, in order; of one that is not there only the size is wanted.
struct Parts {
    char* at;
    size_t used = 0;
    explicit Parts(void* ws) : at(static_cast<char*>(ws)) {}
    void* take(size_t bytes) {
        char* p = at ? at + used : nullptr;
        used += round256(bytes);
        return p;
    }
};

}  // namespace pa
