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

// Four neighbouring elements as they are stored; the largest magnitudes of four rows' elements in each of the columns.
template <typename T> struct Four;
template <> struct Four<float> {
    float4 v;
    __device__ __forceinline__ void clear() { v = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void set(int j, float x) { (j == 0 ? v.x : j == 1 ? v.y : j == 2 ? v.z : v.w) = x; }
    __device__ __forceinline__ float get(int j) const { return j == 0 ? v.x : j == 1 ? v.y : j == 2 ? v.z : v.w; }
    __device__ __forceinline__ unsigned abs(int j) const { return __float_as_uint(get(j)) & 0x7FFFFFFFu; }
    __device__ __forceinline__ unsigned amax() const { return max(max(abs(0), abs(1)), max(abs(2), abs(3))); }
    __device__ static __forceinline__ void column_amax(const Four (&w)[4], unsigned (&top)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) top[i] = max(max(w[0].abs(i), w[1].abs(i)), max(w[2].abs(i), w[3].abs(i)));
    }
};
template <> struct Four<__nv_bfloat16> {
    uint2 v;
    __device__ __forceinline__ void clear() { v = make_uint2(0u, 0u); }
    __device__ __forceinline__ void set(int j, __nv_bfloat16 x) {
        unsigned& w = j < 2 ? v.x : v.y;
        const unsigned b = __bfloat16_as_ushort(x);
        w = j & 1 ? (w & 0xFFFFu) | b << 16 : (w & 0xFFFF0000u) | b;
    }
    __device__ __forceinline__ float get(int j) const {
        const unsigned w = j < 2 ? v.x : v.y;
        return __uint_as_float(j & 1 ? w & 0xFFFF0000u : w << 16);
    }
    __device__ __forceinline__ unsigned amax() const {
        const unsigned m = __vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu);
        return max(m << 16, m & 0xFFFF0000u);
    }
    __device__ static __forceinline__ void column_amax(const Four (&w)[4], unsigned (&top)[4]) {
        const unsigned k = 0x7FFF7FFFu;
        const unsigned a = __vmaxu2(__vmaxu2(w[0].v.x & k, w[1].v.x & k), __vmaxu2(w[2].v.x & k, w[3].v.x & k));
        const unsigned b = __vmaxu2(__vmaxu2(w[0].v.y & k, w[1].v.y & k), __vmaxu2(w[2].v.y & k, w[3].v.y & k));
        top[0] = a << 16; top[1] = a & 0xFFFF0000u; top[2] = b << 16; top[3] = b & 0xFFFF0000u;
    }
};

}  // namespace dst
