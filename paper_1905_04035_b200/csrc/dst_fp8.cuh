// 8-bit floating point with a power-of-two scale for each block: what a kernel that writes such a matrix needs.
#pragma once

#include <cuda_fp8.h>

#include "dst_tied.cuh"

namespace dst {

__device__ __forceinline__ unsigned float_abs(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// The scale of a block whose largest magnitude has the bits `amax`, as an exponent plus 127: the smallest power of two
// 2^e with amax <= 448 * 2^e.  448 = 1.75 * 2^8, so e is amax's exponent less 8, one more where its mantissa is above
// 1.75: adding all that 1.75 leaves of a mantissa, less one, carries exactly there.  255 (NaN) where the block holds an
// infinity or a NaN (their bits are the largest).
constexpr unsigned kLeastAmax = 0x0D800000u;                // 2^-100
__device__ __forceinline__ unsigned block_exponent(unsigned amax) {
    return amax >= 0x7F800000u ? 255u : ((max(amax, kLeastAmax) + 0x1FFFFFu) >> 23) - 8u;
}
// 2^-e, exact (any number where the scale is NaN): the exponent field 262 less the carried one above, in one subtraction
// whose lower bits never borrow
__device__ __forceinline__ float block_inverse(unsigned amax) {
    return __uint_as_float((0x837FFFFFu - 0x1FFFFFu - max(amax, kLeastAmax)) & 0xFF800000u);
}
__device__ __forceinline__ uint8_t* scale_byte(const Fp8View& m, long long row, long long block) {
    return m.scale + ((row >> 7) * m.ld_scale + (block >> 2)) * kScaleTile + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3);
}
// four floats to four e4m3 bytes, round to nearest even
__device__ __forceinline__ unsigned to_e4m3x4(float a, float b, float c, float d) {
    const unsigned lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const unsigned hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
    return lo | hi << 16;
}

}  // namespace dst
