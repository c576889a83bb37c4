// Division of indices by numbers that the host knows, without a division.
#pragma once

#include <stdint.h>

namespace psk {

// x / d for 0 <= x < 2^31, 0 < d < 2^31: multiplication by ceil(2^(31 + s) / d), 2^s >= d (the error of the reciprocal times x
// stays below 1/d).
struct FastDiv {
    uint32_t d, mul, shift;
    void set(uint32_t v) {
        d = v;
        shift = 0;
        while ((1ull << shift) < v) ++shift;
        mul = v == 1 ? 0 : (uint32_t)(((1ull << (31 + shift)) + v - 1) / v);
    }
    __device__ __forceinline__ uint32_t div(uint32_t x) const { return mul == 0 ? x : __umulhi(x, mul) >> (shift - 1); }
};

}  // namespace psk
