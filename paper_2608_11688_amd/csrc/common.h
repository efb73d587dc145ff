// Internal helpers of the APEX library: error reporting and argument checks.
#pragma once

#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <string>

#include "apex.h"

namespace apex {

// Records the message for apex_last_error() on the calling thread and returns `st`.
apex_status fail(apex_status st, const char *fmt, ...);

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// T rows of `bytes` each, `stride` bytes apart.
struct Rows {
    const void *at;
    int64_t stride, bytes;
    int64_t row(int64_t t) const { return static_cast<int64_t>(reinterpret_cast<uintptr_t>(at)) + t * stride; }
};

// Whether T >= 1 rows of a and as many of b, of which neither's own overlap, have a byte in common.
inline bool rows_overlap(const Rows &a, const Rows &b, int64_t T) {
    if (a.row(T - 1) + a.bytes <= b.row(0) || b.row(T - 1) + b.bytes <= a.row(0)) return false;
    if (a.stride == b.stride) {       // row t of b begins `in` bytes behind row t + k of a
        const int64_t d = b.row(0) - a.row(0), k = d / a.stride - (d % a.stride < 0), in = d - k * a.stride;
        return (in < a.bytes && k > -T && k < T) || (in + b.bytes > a.stride && k + 1 > -T && k + 1 < T);
    }
    for (int64_t i = 0, j = 0; i < T && j < T;) {
        if (a.row(i) + a.bytes <= b.row(j)) ++i;
        else if (b.row(j) + b.bytes <= a.row(i)) ++j;
        else return true;
    }
    return false;
}

}  // namespace apex

#define APEX_REQUIRE(cond, ...)                                  \
    do {                                                         \
        if (!(cond)) return ::apex::fail(APEX_E_INVAL, __VA_ARGS__); \
    } while (0)

#define APEX_HIP(call)                                                          \
    do {                                                                        \
        hipError_t apex_err_ = (call);                                          \
        if (apex_err_ != hipSuccess)                                            \
            return ::apex::fail(APEX_E_HIP, "%s failed: %s", #call,            \
                                hipGetErrorString(apex_err_));                  \
    } while (0)
