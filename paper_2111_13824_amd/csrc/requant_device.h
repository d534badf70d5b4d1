// Dyadic requantization of one int32 value (the integer form of Supplement A.1).
#pragma once

#include <hip/hip_runtime.h>

namespace fqvit {

// y = clip(((N2 q + 2^(N1-1)) >> N1) + zp, 0, 2^b - 1) in the int8 container.
__device__ __forceinline__ int requant_one(int32_t q, int64_t N2, int N1, int64_t zp, int64_t hi,
                                           int half) {
    const int64_t prod = N2 * (int64_t)q;
    const int64_t w = N1 > 0 ? (prod + ((int64_t)1 << (N1 - 1))) >> N1 : prod;
    const int64_t yu = w + zp;
    const int64_t yc = yu < 0 ? 0 : (yu > hi ? hi : yu);
    return (int)yc - half;
}

// The same for N1 >= 32 (every M below 1/2): the rounding term enters the 64-bit
// multiply-add, the shift leaves the high word alone, and a value outside
// [-2^31, 2^31) after zp cannot arise (|w| < 2^30 there).  Six instructions an
// element instead of twenty: 768 x 197 x 64 elements, after the attention from Q and
// K (both): 37.7 -> 36.8 us.
__device__ __forceinline__ int requant_hi(int32_t q, int32_t N2, uint64_t half_ulp, int sh, int zp_c,
                                          int lo, int hi) {
    const int64_t prod = (int64_t)N2 * (int64_t)q + (int64_t)half_ulp;
    const int w = (int)(prod >> 32) >> sh;
    return min(max(w + zp_c, lo), hi);
}

}  // namespace fqvit
