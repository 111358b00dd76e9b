// 4-bit floating point with a power-of-two scale for each block of 32: what a kernel that writes such a matrix needs.
#pragma once

#include <cuda_fp4.h>

#include "dst_tied.cuh"

namespace dst {

// As in 8 bits, with 6 = 1.5 * 2^2 the largest value: the smallest power of two 2^e with amax <= 6 * 2^e, as an exponent plus 127;
// 255 (NaN) where the block holds an infinity or a NaN.
constexpr unsigned kLeastAmax4 = 0x0D800000u;               // 2^-100
__device__ __forceinline__ unsigned block_exponent4(unsigned amax) {
    return amax >= 0x7F800000u ? 255u : ((max(amax, kLeastAmax4) + 0x3FFFFFu) >> 23) - 2u;
}
// 2^-e, exact (any number where the scale is NaN)
__device__ __forceinline__ float block_inverse4(unsigned amax) {
    return __uint_as_float((0x807FFFFFu - 0x3FFFFFu - max(amax, kLeastAmax4)) & 0xFF800000u);
}
// four floats to four e2m1 elements, the first in the lowest bits, round to nearest even
__device__ __forceinline__ unsigned to_e2m1x4(float a, float b, float c, float d) {
    const unsigned lo = __nv_cvt_float2_to_fp4x2(make_float2(a, b), __NV_E2M1, cudaRoundNearest);
    const unsigned hi = __nv_cvt_float2_to_fp4x2(make_float2(c, d), __NV_E2M1, cudaRoundNearest);
    return lo | hi << 8;
}

}  // namespace dst
