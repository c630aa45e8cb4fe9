// Division of 32-bit numbers by one that is known before the launch.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mlda {

// Quotients of 32-bit numbers below 2^31 by one that the host knows.
struct Divisor {
    uint32_t by, factor, shift;
    __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return by == 1 ? n : __umulhi(n, factor) >> shift; }
};

// With l = ceil(log2 by) and factor = floor(2^(31 + l) / by) + 1, n factor / 2^(31 + l) lies above n / by by less than 1 / by for n < 2^31.
inline Divisor divisor(uint32_t by) {
    uint32_t l = 0;
    while (l < 31 && (1u << l) < by) ++l;
    return Divisor{by, l ? (uint32_t)(((uint64_t)1 << (31 + l)) / by + 1) : 0, l ? l - 1 : 0};
}

}  // namespace mlda
