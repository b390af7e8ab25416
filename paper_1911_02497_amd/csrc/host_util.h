// Host-side pieces that every source of the library shares: status of runtime calls, launch count, buffer-overlap checks.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>

#include "common.h"

namespace condensa {

extern std::atomic<int> g_last_hip_error;
extern std::atomic<uint64_t> g_launches;        // kernels enqueued since the library was loaded (diagnostic)

#define CONDENSA_HIP(expr)                                                      \
    do {                                                                        \
        hipError_t err__ = (expr);                                              \
        if (err__ != hipSuccess) {                                              \
            ::condensa::g_last_hip_error.store(static_cast<int>(err__));        \
            return CONDENSA_ERR_HIP;                                            \
        }                                                                       \
    } while (0)

#define CONDENSA_LAUNCH_CHECK()                                                 \
    do {                                                                        \
        ::condensa::g_launches.fetch_add(1, std::memory_order_relaxed);         \
        CONDENSA_HIP(hipGetLastError());                                        \
    } while (0)

inline size_t align_up(size_t x, size_t a = 256) { return (x + a - 1) / a * a; }

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Byte ranges of the buffers of one call.  A call is rejected when an output overlaps any other range.
// An input that the call also writes in place (theta == w, lambda updated in place) is entered once, as
// an output.
struct ByteRange {
    uintptr_t begin, end;
    bool written;
};
inline ByteRange byte_range(const void* p, u64 bytes, bool written) {
    const uintptr_t b = reinterpret_cast<uintptr_t>(p);
    return ByteRange{b, b + static_cast<uintptr_t>(p ? bytes : 0), written};
}
// Sorts `r` by start address; true when some written range overlaps another range.
inline bool ranges_conflict(ByteRange* r, size_t n) {
    std::sort(r, r + n, [](const ByteRange& x, const ByteRange& y) { return x.begin < y.begin; });
    uintptr_t end_any = 0, end_written = 0;          // furthest end among the ranges seen so far
    for (size_t i = 0; i < n; ++i) {
        if (r[i].begin == r[i].end) continue;        // empty
        if (r[i].written ? r[i].begin < end_any : r[i].begin < end_written) return true;
        if (r[i].end > end_any) end_any = r[i].end;
        if (r[i].written && r[i].end > end_written) end_written = r[i].end;
    }
    return false;
}

}  // namespace condensa
