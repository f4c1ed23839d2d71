// Division of 0 <= n < 2^31 by an invariant 1 <= d < 2^31 as a multiplication: q = (n * mul) >> shift in 64 bits.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace vitq {

struct FastDiv { uint32_t mul, shift; };

inline FastDiv fast_div(uint32_t d) {
    // l = ceil(log2 d), mul = ceil(2^(31+l) / d) < 2^32 with mul*d - 2^(31+l) = e < d <= 2^l: n*e < 2^(31+l) for n < 2^31,
    // so n*mul / 2^(31+l) exceeds n / d by less than 1 / d and has the same floor
    uint32_t l = 0;
    while ((uint64_t(1) << l) < d) ++l;
    const uint64_t num = uint64_t(1) << (31 + l);
    FastDiv f;
    f.shift = 31 + l; f.mul = (uint32_t)((num + d - 1) / d);
    return f;
}
__device__ __forceinline__ uint32_t divide(uint32_t n, const FastDiv &f) { return (uint32_t)(((uint64_t)n * f.mul) >> f.shift); }

}  // namespace vitq
