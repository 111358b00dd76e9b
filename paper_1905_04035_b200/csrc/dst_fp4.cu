// 4-bit floating point with a power-of-two scale for each block of 32 columns of a row: quantisation, and the product's entries.
#include "dst_block_matmul.cuh"

namespace dst {

// ---- quantisation -----------------------------------------------------------------
// A warp takes 256 columns of a row at a time, eight neighbouring ones a lane, so that four lanes hold a block, a lane's elements are a
// word and the four scales of 128 columns are one too.  ROWS rows are in flight: many where the matrix is large, one where it would
// not fill the device otherwise.
// Measured: 33,708 x 1024 fp32 26 us (138 MB in, 18 out: 24 at the copy rate).
constexpr int kQuant4Warps = 8;

template <typename T, bool VEC, int ROWS>
__global__ void __launch_bounds__(kQuant4Warps * 32) k_quantize4(const __grid_constant__ QuantParams p) {
    constexpr int kRows = ROWS;
    const int lane = lane_id(), col_tiles = (int)((p.cols + 255) >> 8);
    const long long tile = blockIdx.x / col_tiles;
    const long long c0 = (long long)(blockIdx.x - tile * col_tiles) * 256 + lane * 8, r0 = (tile * kQuant4Warps + warp_id()) * kRows;
    pdl_trigger();
    pdl_wait();
    float v[kRows][8];
    const T* const x = static_cast<const T*>(p.x) + r0 * p.ldx + c0;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        if (VEC && r0 + i < p.rows && c0 + 8 <= p.cols) load8<T>(x + i * p.ldx, v[i]);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = r0 + i < p.rows && c0 + j < p.cols ? to_float<T>(x[i * p.ldx + j]) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        if (r0 + i >= p.rows) break;
        const long long row = r0 + i;
        unsigned top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, float_abs(v[i][j]));
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        const float u = block_inverse4(top);
        unsigned e = block_exponent4(top);
        e |= __shfl_down_sync(0xFFFFFFFFu, e, 4) << 8;
        e |= __shfl_down_sync(0xFFFFFFFFu, e, 8) << 16;     // lanes 0 and 16: the four scales of 128 columns (those past the row for zeros)
        if (c0 >= p.cols) continue;
        // (up to three bytes of a row's padding are written too)
        *reinterpret_cast<unsigned*>(p.q.q + row * p.q.ld + (c0 >> 1)) =
            to_e2m1x4(v[i][0] * u, v[i][1] * u, v[i][2] * u, v[i][3] * u) | to_e2m1x4(v[i][4] * u, v[i][5] * u, v[i][6] * u, v[i][7] * u) << 16;
        if ((lane & 15) == 0)
            *reinterpret_cast<unsigned*>(p.q.scale + ((row >> 7) * p.q.ld_scale + (c0 >> 7)) * kScaleTile + (row & 31) * 16 + ((row >> 5) & 3) * 4) = e;
    }
}

template <typename T, bool VEC, int ROWS>
static cudaError_t quantize4_run(const QuantParams& p, cudaStream_t stream) {
    constexpr long long kRows = kQuant4Warps * ROWS;
    const dim3 grid((unsigned)(((p.rows + kRows - 1) / kRows) * ((p.cols + 255) / 256)));
    return launch_pdl(k_quantize4<T, VEC, ROWS>, grid, dim3(kQuant4Warps * 32), 0, stream, p);
}
template <typename T>
static cudaError_t quantize4_t(const QuantParams& p, cudaStream_t stream) {
    constexpr int kMany = sizeof(T) == 4 ? 4 : 8;
    const bool vec = (reinterpret_cast<uintptr_t>(p.x) & 15u) == 0 && p.ldx * sizeof(T) % 16 == 0;
    const bool large = p.rows * ((p.cols + 255) / 256) >= 32ll * kSmCount * kMany;   // a row and 256 columns a warp: 32 warps for each SM and more
    if (large) return vec ? quantize4_run<T, true, kMany>(p, stream) : quantize4_run<T, false, kMany>(p, stream);
    return vec ? quantize4_run<T, true, 1>(p, stream) : quantize4_run<T, false, 1>(p, stream);
}
cudaError_t launch_quantize_fp4(const QuantParams& p, int x_type, cudaStream_t stream) {
    return x_type == DST_F32 ? quantize4_t<float>(p, stream) : quantize4_t<__nv_bfloat16>(p, stream);
}

// ---- product (dst_block_matmul.cuh) -----------------------------------------------
size_t matmul_fp4_workspace(long long M, long long N, long long K) { return block_matmul_workspace<Fp4Kind>(M, N, K); }
size_t matmul_fp4_workspace_bound(long long M, long long N, long long K) { return block_matmul_workspace_bound<Fp4Kind>(M, N, K); }
cudaError_t launch_matmul_fp4(const Fp8View& a, const Fp8View& b, void* out, long long ldo, int out_type, void* workspace, int sms, cudaStream_t stream) {
    return launch_block_matmul<Fp4Kind>(a, b, out, ldo, out_type, workspace, sms, stream);
}

// A few rows of x are quantised by every CTA for itself while the weight's first tiles are on their way: up to 12 blocks of 256, where the
// two forms cost the same (in one kernel and in two, 33,708 x 1024: 1 row 5.8 and 6.7 us, 3 rows 6.4 and 6.8, 4 rows 7.2 and 6.7, 8 rows 9.5
// and 7.0; x 512: 1 row 4.3 and 4.7, 6 rows 5.3 and 4.7; x 64: 1 row 4.2 and 4.7, 10 rows 5.4 and 5.7, 16 rows 6.3 and 5.7; x 2048: 1 row 8.5 and
// 9.7; 1000 x 1024: 1 row 4.1 and 4.2, 3 rows 4.8 and 4.2).
bool linear_fp4_fused(long long M, long long N, long long K) {
    const MatmulPlan L = plan_matmul<Fp4Kind>(M, N, K);
    return block_linear_fits<Fp4Kind>(L) && M * L.blocks <= 12;
}
cudaError_t launch_linear_fp4_fused(const void* x, long long ldx, int x_type, long long M, const Fp8View& w, void* out, long long ldo, int out_type,
                                    int sms, cudaStream_t stream) {
    return launch_block_linear<Fp4Kind>(x, ldx, x_type, M, w, out, ldo, out_type, sms, stream);
}

}  // namespace dst
