// Division by a number fixed at launch (host and device; no HIP needed).
#pragma once

#include <stdint.h>

#if defined(__HIP__)
#define PB_HOST_DEVICE __host__ __device__ inline
#else
#define PB_HOST_DEVICE inline
#endif

namespace pb {

// Quotients by a divisor fixed at launch, exact for 0 <= n < 2^31: with
// s = ceil(log2 d) and m = floor(2^(31 + s) / d) + 1, n / d = (2 n m) >> (32 + s)
// (m d - 2^(31 + s) <= d <= 2^s, so the error n (m d - 2^(31+s)) / (d 2^(31+s)) is
// below 1 / d; m < 2^32 because d > 2^(s-1)).
struct FastDiv {
    uint32_t m, s, d;
    FastDiv(uint32_t div = 1) : d(div) {
        s = 0;
        while ((1u << s) < div) ++s;
        m = (uint32_t)((((uint64_t)1 << (31 + s)) / div) + 1);
    }
    PB_HOST_DEVICE uint32_t quot(uint32_t n) const { return (uint32_t)(((uint64_t)(n << 1) * m) >> 32) >> s; }
};

}  // namespace pb
