// Host-side helpers of the C ABI's entry points: byte ranges for the overlap checks and the
// status a call returns once its work is enqueued.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdlib.h>
#include <string.h>

#include <initializer_list>

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

constexpr int64_t kMostElements = int64_t(1) << 40;   // of one array: byte offsets stay far inside 64 bits

// Whether the product of non-negative factors stays within kMostElements.
inline bool product_ok(std::initializer_list<int64_t> factors)
{
    int64_t p = 1;
    for (int64_t f : factors) {
        if (f == 0) return true;
        if (f > kMostElements / p) return false;
        p *= f;
    }
    return true;
}

inline bool float_type(int dtype) { return dtype == MESA_DTYPE_F32 || dtype == MESA_DTYPE_BF16; }
inline int64_t bytes_of(int dtype) { return dtype == MESA_DTYPE_BF16 ? 2 : dtype == MESA_DTYPE_Q8 ? 1 : 4; }
inline bool aligned(const void* p, int64_t bytes) { return uintptr_t(p) % uintptr_t(bytes) == 0; }
inline bool all_aligned(std::initializer_list<const void*> ptrs, int64_t bytes)
{
    for (const void* p : ptrs)
        if (!aligned(p, bytes)) return false;
    return true;
}
inline bool any_null(std::initializer_list<const void*> ptrs)
{
    for (const void* p : ptrs)
        if (p == nullptr) return true;
    return false;
}

// A device array as `rows` pieces of `bytes`, `pitch` apart (absent: a null pointer or no bytes).
struct Rows {
    const void* p;
    int64_t rows, bytes, pitch;
    bool empty() const { return p == nullptr || rows <= 0 || bytes <= 0; }
    Range span() const { return range_of(p, (rows - 1) * pitch + bytes); }
};
inline Rows dense(const void* p, int64_t bytes) { return {p, 1, bytes, bytes}; }
inline Rows tokens(const void* p, int64_t n, int64_t width, int64_t stride, int dtype)
{
    return {p, n, width * bytes_of(dtype), stride * bytes_of(dtype)};
}

// Whether two arrays share a byte.  Slices of one array (the same pitch) interleave freely.
inline bool touch(const Rows& a, const Rows& b)
{
    if (a.empty() || b.empty() || !overlaps(a.span(), b.span())) return false;
    if (a.pitch != b.pitch || a.rows == 1 || b.rows == 1) return true;
    int64_t d = (int64_t(uintptr_t(b.p)) - int64_t(uintptr_t(a.p))) % a.pitch;
    if (d < 0) d += a.pitch;
    return d < a.bytes || a.pitch - d < b.bytes;
}

// Outputs must overlap neither an input nor each other.
inline bool clash(std::initializer_list<Rows> ins, std::initializer_list<Rows> outs)
{
    for (const Rows* o = outs.begin(); o != outs.end(); ++o) {
        for (const Rows& i : ins)
            if (touch(*o, i)) return true;
        for (const Rows* q = o + 1; q != outs.end(); ++q)
            if (touch(*o, *q)) return true;
    }
    return false;
}

inline int status_of(hipError_t e, void* stream) { return finish(launch_status(e), stream); }

}  // namespace mesa
