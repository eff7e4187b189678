// What the entry points of operators share: refusals, alignment and overlap of
// operands, and the status of a launch.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdio>

#include "../include/pipeboost.h"

__attribute__((visibility("hidden"))) int pb_fail_status(int code, const char* msg);  // model.cpp

namespace pb {

__attribute__((format(printf, 1, 2))) inline int refuse(const char* fmt, ...) {
    char buf[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof(buf), fmt, ap);
    va_end(ap);
    return pb_fail_status(PB_EINVAL, buf);
}

inline int launched(const char* op, hipError_t e) {
    if (e == hipSuccess) return PB_OK;
    char buf[256];
    snprintf(buf, sizeof(buf), "%s: launch failed: %s", op, hipGetErrorString(e));
    return pb_fail_status(PB_EHIP, buf);
}

inline bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    return a && b && na && nb && (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}

}  // namespace pb
