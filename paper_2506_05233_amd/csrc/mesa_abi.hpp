// Host-side helpers of the C ABI's entry points: byte ranges for the overlap checks and the
// status a call returns once its work is enqueued.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdlib.h>
#include <string.h>

#include "libmesa.h"

namespace mesa {

// Byte range [p, p + n) of a device array, for overlap checks.
struct Range {
    uintptr_t lo, hi;
};
inline Range range_of(const void* p, int64_t bytes) { return {uintptr_t(p), uintptr_t(p) + uintptr_t(bytes)}; }
inline bool overlaps(Range a, Range b) { return a.lo < b.hi && b.lo < a.hi; }

// MESA_SYNC_AFTER_LAUNCH (read once, at the first call): when set to anything but
// "" or "0", every entry point synchronises its stream after its launches and turns
// an execution error into MESA_ERR_HIP.
inline bool sync_after_launch()
{
    static const bool on = [] {
        const char* e = getenv("MESA_SYNC_AFTER_LAUNCH");
        return e != nullptr && e[0] != '\0' && strcmp(e, "0") != 0;
    }();
    return on;
}

// A launch's error as a status; a grid that one launch cannot hold is refused as a size.
inline int launch_status(hipError_t e)
{
    return e == hipSuccess ? MESA_OK : e == hipErrorInvalidConfiguration ? MESA_ERR_SHAPE : MESA_ERR_HIP;
}

// The status an entry point returns once its launches are enqueued on `stream`.
inline int finish(int status, void* stream)
{
    if (status != MESA_OK || !sync_after_launch()) return status;
    if (hipStreamSynchronize(static_cast<hipStream_t>(stream)) != hipSuccess) return MESA_ERR_HIP;
    return hipGetLastError() == hipSuccess ? MESA_OK : MESA_ERR_HIP;
}

}  // namespace mesa
