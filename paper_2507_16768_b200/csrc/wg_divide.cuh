// Division by a number that is fixed for a launch.
#pragma once

#include <cuda_runtime.h>
#include <cstdint>

// n / d for n < 2^31 by a multiplication: M = ceil(2^(31 + k) / d) with 2^(k - 1) < d <= 2^k fits 32 bits, and
// n * (M * d - 2^(31 + k)) < 2^31 * 2^k, so the quotient is exact.
struct Divisor {
    uint32_t d, mul;
    int32_t shift;
    static Divisor of(uint32_t d) {
        int k = 0;
        while ((1ull << k) < d) ++k;
        return {d, (uint32_t)(((1ull << (31 + k)) + d - 1) / d), 31 + k};
    }
    __device__ __forceinline__ uint32_t quotient(uint32_t n) const { return (uint32_t)(((uint64_t)n * mul) >> shift); }
};
