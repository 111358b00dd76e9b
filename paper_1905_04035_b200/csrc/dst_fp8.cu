// 8-bit floating point with a power-of-two scale for each block of 128: quantisation and the product of two such matrices.
#include <cuda_fp8.h>

#include "dst_tied.cuh"

namespace dst {

// ---- quantisation -----------------------------------------------------------------
// The scale of a block whose largest magnitude has the bits `amax`: the smallest power of two 2^e with
// amax <= 448 * 2^e.  448 = 1.75 * 2^8, so e is amax's exponent less 8, one more where its mantissa is above 1.75.
// NaN where the block holds an infinity or a NaN (their bits are the largest).
__device__ __forceinline__ float block_scale(unsigned amax) {
    if (amax >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
    const unsigned low = 0x0D800000u;                       // 2^-100
    if (amax < low) amax = low;
    const unsigned e = (amax >> 23) - 8u + ((amax & 0x7FFFFFu) > 0x600000u ? 1u : 0u);
    return __uint_as_float(e << 23);
}
// its reciprocal: exact, a power of two
__device__ __forceinline__ float block_unscale(float scale) { return __uint_as_float(0x7F000000u - __float_as_uint(scale)); }
__device__ __forceinline__ unsigned abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// four floats to four e4m3 bytes, round to nearest even
__device__ __forceinline__ unsigned to_e4m3x4(float a, float b, float c, float d) {
    const unsigned lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const unsigned hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
    return lo | hi << 16;
}

constexpr int kQuantThreads = 256;

// A CTA takes 128 x 128 elements: each is read once, into shared memory, and rounded for the matrix and for its
// transpose from there.  Rows of the tile are 129 floats apart, so that lanes on neighbouring columns and lanes on
// neighbouring rows both find 32 different banks.
template <typename T, bool SQUARE>
__global__ void __launch_bounds__(kQuantThreads) k_quantize_tile(const __grid_constant__ QuantParams p) {
    extern __shared__ float tile[];                          // [128][129]
    __shared__ unsigned warp_max[kQuantThreads / 32];
    pdl_trigger();
    pdl_wait();
    const long long r0 = (long long)blockIdx.y * 128, c0 = (long long)blockIdx.x * 128;
    const int nr = (int)(p.rows - r0 < 128 ? p.rows - r0 : 128), nc = (int)(p.cols - c0 < 128 ? p.cols - c0 : 128);
    const int lane = lane_id(), warp = warp_id();
    constexpr int kWarps = kQuantThreads / 32;
    const T* x = static_cast<const T*>(p.x);
    unsigned top = 0;
    for (int r = warp; r < 128; r += kWarps)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = j * 32 + lane;
            const float v = r < nr && c < nc ? to_float(x[(r0 + r) * p.ldx + c0 + c]) : 0.f;
            tile[r * 129 + c] = v;
            top = max(top, abs_bits(v));
        }
    float square = 0.f;
    if (SQUARE) {
        top = __reduce_max_sync(0xFFFFFFFFu, top);
        if (lane == 0) warp_max[warp] = top;
    }
    __syncthreads();
    if (SQUARE) {
        for (int w = 0; w < kWarps; ++w) top = max(top, warp_max[w]);
        square = block_scale(top);
        if (threadIdx.x == 0) {
            if (p.q.q) p.q.scale[(long long)blockIdx.x * p.q.ld_scale + blockIdx.y] = square;
            if (p.qt.q) p.qt.scale[(long long)blockIdx.y * p.qt.ld_scale + blockIdx.x] = square;
        }
    }
    if (p.q.q)
        for (int r = warp; r < nr; r += kWarps) {
            float v[4];
            unsigned m = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) { v[j] = tile[r * 129 + lane * 4 + j]; m = max(m, abs_bits(v[j])); }
            float s = square;
            if (!SQUARE) {
                s = block_scale(__reduce_max_sync(0xFFFFFFFFu, m));
                if (lane == 0) p.q.scale[(long long)blockIdx.x * p.q.ld_scale + r0 + r] = s;
            }
            const float u = block_unscale(s);
            if (lane * 4 < nc)
                *reinterpret_cast<unsigned*>(p.q.q + (r0 + r) * p.q.ld + c0 + lane * 4) = to_e4m3x4(v[0] * u, v[1] * u, v[2] * u, v[3] * u);
        }
    if (p.qt.q)
        for (int c = warp; c < nc; c += kWarps) {
            float v[4];
            unsigned m = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) { v[j] = tile[(lane * 4 + j) * 129 + c]; m = max(m, abs_bits(v[j])); }
            float s = square;
            if (!SQUARE) {
                s = block_scale(__reduce_max_sync(0xFFFFFFFFu, m));
                if (lane == 0) p.qt.scale[(long long)blockIdx.y * p.qt.ld_scale + c0 + c] = s;
            }
            const float u = block_unscale(s);
            if (lane * 4 < nr)
                *reinterpret_cast<unsigned*>(p.qt.q + (c0 + c) * p.qt.ld + r0 + lane * 4) = to_e4m3x4(v[0] * u, v[1] * u, v[2] * u, v[3] * u);
        }
}

template <typename T, bool SQUARE>
static cudaError_t quantize_t(const QuantParams& p, cudaStream_t stream) {
    static SmemOptIn opt;
    const size_t smem = 128 * 129 * sizeof(float);
    const cudaError_t e = ensure_dynamic_smem(k_quantize_tile<T, SQUARE>, smem, opt);
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)((p.cols + 127) / 128), (unsigned)((p.rows + 127) / 128));
    return launch_pdl(k_quantize_tile<T, SQUARE>, grid, dim3(kQuantThreads), smem, stream, p);
}

cudaError_t launch_quantize(const QuantParams& p, int x_type, int, cudaStream_t stream) {
    const bool square = (p.q.q ? p.q.shift : p.qt.shift) != 0;
    if (x_type == DST_F32) return square ? quantize_t<float, true>(p, stream) : quantize_t<float, false>(p, stream);
    return square ? quantize_t<__nv_bfloat16, true>(p, stream) : quantize_t<__nv_bfloat16, false>(p, stream);
}

// ---- product ----------------------------------------------------------------------
size_t matmul_fp8_workspace(long long, long long, long long) { return 0; }

__device__ __forceinline__ float from_e4m3(uint8_t v) {
    return __half2float(__half(__nv_cvt_fp8_to_halfraw(v, __NV_E4M3)));
}

// 16 x 16 outputs a CTA, one a thread
template <typename OT>
__global__ void __launch_bounds__(256) k_matmul_fp8(Fp8View a, Fp8View b, OT* out, long long ldo) {
    __shared__ float ta[16][129], tb[16][129];
    pdl_trigger();
    pdl_wait();
    const long long m0 = (long long)blockIdx.y * 16, n0 = (long long)blockIdx.x * 16;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const long long m = m0 + ty, n = n0 + tx;
    float acc = 0.f;
    for (long long k0 = 0; k0 < a.cols; k0 += 128) {
        __syncthreads();
        for (int i = threadIdx.x; i < 16 * 128; i += 256) {
            const int r = i >> 7, c = i & 127;
            ta[r][c] = m0 + r < a.rows && k0 + c < a.cols ? from_e4m3(a.q[(m0 + r) * a.ld + k0 + c]) : 0.f;
            tb[r][c] = n0 + r < b.rows && k0 + c < b.cols ? from_e4m3(b.q[(n0 + r) * b.ld + k0 + c]) : 0.f;
        }
        __syncthreads();
        float part = 0.f;
        for (int c = 0; c < 128; ++c) part = fmaf(ta[ty][c], tb[tx][c], part);
        if (m < a.rows && n < b.rows)
            acc = fmaf(part, a.scale[(k0 >> 7) * a.ld_scale + (m >> a.shift)] * b.scale[(k0 >> 7) * b.ld_scale + (n >> b.shift)], acc);
    }
    if (m < a.rows && n < b.rows) out[m * ldo + n] = from_float<OT>(acc);
}

cudaError_t launch_matmul_fp8(const Fp8View& a, const Fp8View& b, void* out, long long ldo, int out_type, void*, int, cudaStream_t stream) {
    const dim3 grid((unsigned)((b.rows + 15) / 16), (unsigned)((a.rows + 15) / 16));
    if (out_type == DST_F32) return launch_pdl(k_matmul_fp8<float>, grid, dim3(256), 0, stream, a, b, static_cast<float*>(out), ldo);
    return launch_pdl(k_matmul_fp8<__nv_bfloat16>, grid, dim3(256), 0, stream, a, b, static_cast<__nv_bfloat16*>(out), ldo);
}

}  // namespace dst
