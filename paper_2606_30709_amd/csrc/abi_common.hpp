// Host-side helpers of the C entry points: status reporting and the argument
// checks they share (defined in hga_abi.cpp).
#pragma once

#include <hip/hip_runtime.h>

#include "hga.h"

namespace hga {
namespace abi {

// Records the calling thread's error message and returns `st`.
hga_status fail(hga_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
hga_status hip_fail(hipError_t e, const char* what);

bool aligned(const void* p, size_t a);
hga_status check_plan(const hga_plan* plan);
// A tensor pointer: not NULL, 16-byte aligned; an index pointer: 4-byte.
hga_status check_tensor(const void* p, const char* name);
hga_status check_index(const void* p, const char* name);
// A caller workspace: NULL with 0 bytes, or 16-byte aligned with > 0 bytes.
hga_status check_workspace(const void* workspace, int64_t workspace_bytes);
hga_status launched(hipError_t e, const char* what);

// A launch reports its error through hipGetLastError(), which also returns
// errors that earlier, unrelated runtime calls on this thread left behind;
// clear those first so a launch is charged only with its own failure.
inline void clear_stale_error() { (void)hipGetLastError(); }

}  // namespace abi
}  // namespace hga

#define HGA_TRY(x)                      \
    do {                                \
        hga_status st_ = (x);           \
        if (st_ != HGA_OK) return st_;  \
    } while (0)
