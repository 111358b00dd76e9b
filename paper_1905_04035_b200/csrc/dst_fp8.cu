// 8-bit floating point with a power-of-two scale for each block of 128: quantisation, and the product's entries.
#include "dst_block_matmul.cuh"

namespace dst {

// ---- quantisation -----------------------------------------------------------------
// fp32 tiles take twice the warps: a warp then holds eight rows, 32 registers a lane, and two CTAs share an SM
template <typename T> struct QuantShape {
    static constexpr int kThreads = sizeof(T) == 4 ? 512 : 256, kWarps = kThreads / 32, kRows = 128 / kWarps, kCtas = sizeof(T) == 4 ? 2 : 4;
};
constexpr int kQuantPitch = 132;                           // elements between rows of the staged tile

// A CTA takes 128 x 128 elements, read once: a warp holds whole rows of the tile, four neighbouring columns a lane,
// so a row's largest magnitude is one reduction over the warp and its 128 bytes go out in one store.  For the transpose
// the tile passes through shared memory: row r is kept in place (r % 4) * 32 + r / 4, so that a lane that wants rows
// 4 l .. 4 l + 3 (the four bytes of a transposed row it writes) reads, with the whole warp, neighbouring places.
// VEC: rows are aligned to four elements.  FULL: the whole tile is inside the matrix.
// Measured: 33,708 x 1024 fp32, square blocks, both ways 37 us (5600 GB/s of 6551); 8111 x 33,708 bf16 both ways 255 us (4290;
// bound by the integer pipe: unpacking, maxima, packing), one way 5700 GB/s.
template <typename T, bool SQUARE, bool VEC, bool FULL>
__device__ __forceinline__ void quantize_tile(const QuantParams& p, T* tile, unsigned* warp_max, long long rb, long long cb) {
    using S = QuantShape<T>;
    const long long r0 = rb * 128, c0 = cb * 128;
    const int nr = FULL ? 128 : (int)min(p.rows - r0, 128ll), nc = FULL ? 128 : (int)min(p.cols - c0, 128ll);
    const int lane = lane_id(), warp = warp_id();
    using Raw = decltype(Four<T>::v);
    Four<T> v[S::kRows];
    {
        const T* x = static_cast<const T*>(p.x) + (r0 + warp) * p.ldx + c0 + lane * 4;
#pragma unroll
        for (int i = 0; i < S::kRows; ++i, x += S::kWarps * p.ldx) {
            if (VEC && FULL) { v[i].v = __ldcs(reinterpret_cast<const Raw*>(x)); continue; }
            v[i].clear();
            if (i * S::kWarps + warp >= nr) continue;
            if (VEC && lane * 4 + 4 <= nc) v[i].v = __ldcs(reinterpret_cast<const Raw*>(x));
            else
#pragma unroll
                for (int j = 0; j < 4; ++j) if (lane * 4 + j < nc) v[i].set(j, x[j]);
        }
    }
    if (SQUARE) {
        unsigned top = 0;
#pragma unroll
        for (int i = 0; i < S::kRows; ++i) top = max(top, v[i].amax());
        top = __reduce_max_sync(0xFFFFFFFFu, top);
        if (lane == 0) warp_max[warp] = top;
    }
    if (p.qt.q) {
#pragma unroll
        for (int i = 0; i < S::kRows; ++i) {
            const int r = i * S::kWarps + warp;
            *reinterpret_cast<Raw*>(tile + ((r & 3) * 32 + (r >> 2)) * kQuantPitch + lane * 4) = v[i].v;
        }
    }
    if (SQUARE || p.qt.q) __syncthreads();
    float u = 0.f;
    if (SQUARE) {
        unsigned top = 0;
        for (int w = 0; w < S::kWarps; ++w) top = max(top, warp_max[w]);
        u = block_inverse(top);
        const uint8_t e = (uint8_t)block_exponent(top);
        if (threadIdx.x < 128) {                            // every row's byte, as the product wants it
            if (p.q.q) *scale_byte(p.q, r0 + threadIdx.x, cb) = e;
            if (p.qt.q) *scale_byte(p.qt, c0 + threadIdx.x, rb) = e;
        }
    }
    if (p.q.q) {
        uint8_t* q = p.q.q + (r0 + warp) * p.q.ld + c0 + lane * 4;
        unsigned mine = 0;                                  // lane i: the largest magnitude of the warp's i-th row
#pragma unroll
        for (int i = 0; i < S::kRows; ++i, q += S::kWarps * p.q.ld) {
            if (!SQUARE) {
                const unsigned top = __reduce_max_sync(0xFFFFFFFFu, v[i].amax());
                if (lane == i) mine = top;
                u = block_inverse(top);
            }
            if (FULL || (i * S::kWarps + warp < nr && lane * 4 < nc))   // (up to three bytes of a row's padding are written too)
                *reinterpret_cast<unsigned*>(q) = to_e4m3x4(v[i].get(0) * u, v[i].get(1) * u, v[i].get(2) * u, v[i].get(3) * u);
        }
        if (!SQUARE && lane < S::kRows && lane * S::kWarps + warp < nr) *scale_byte(p.q, r0 + lane * S::kWarps + warp, cb) = (uint8_t)block_exponent(mine);
    }
    if (p.qt.q) {
        constexpr int kCols = 128 / S::kWarps;              // of the warp, consecutive
        uint8_t* q = p.qt.q + (c0 + warp * kCols) * p.qt.ld + r0 + lane * 4;
        const T* from = tile + lane * kQuantPitch + warp * kCols;
        unsigned mine = 0;
#pragma unroll
        for (int k = 0; k < kCols; k += 4) {                // four columns, rows 4 lane .. 4 lane + 3
            Four<T> w[4];
            unsigned top[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j].v = *reinterpret_cast<const Raw*>(from + j * 32 * kQuantPitch + k);
            if (!SQUARE) Four<T>::column_amax(w, top);
#pragma unroll
            for (int i = 0; i < 4; ++i, q += p.qt.ld) {
                if (!SQUARE) {
                    const unsigned most = __reduce_max_sync(0xFFFFFFFFu, top[i]);
                    if (lane == k + i) mine = most;
                    u = block_inverse(most);
                }
                if (FULL || (warp * kCols + k + i < nc && lane * 4 < nr))
                    *reinterpret_cast<unsigned*>(q) = to_e4m3x4(w[0].get(i) * u, w[1].get(i) * u, w[2].get(i) * u, w[3].get(i) * u);
            }
        }
        if (!SQUARE && lane < kCols && warp * kCols + lane < nc) *scale_byte(p.qt, c0 + warp * kCols + lane, rb) = (uint8_t)block_exponent(mine);
    }
}

template <typename T, bool SQUARE, bool VEC>
__global__ void __launch_bounds__(QuantShape<T>::kThreads, QuantShape<T>::kCtas) k_quantize(const __grid_constant__ QuantParams p) {
    extern __shared__ __align__(16) unsigned char dyn[];
    __shared__ unsigned warp_max[QuantShape<T>::kWarps];
    pdl_trigger();
    pdl_wait();
    const int col_tiles = (int)((p.cols + 127) >> 7), rb = blockIdx.x / col_tiles, cb = blockIdx.x - rb * col_tiles;
    if (rb * 128ll + 128 <= p.rows && cb * 128ll + 128 <= p.cols) quantize_tile<T, SQUARE, VEC, true>(p, reinterpret_cast<T*>(dyn), warp_max, rb, cb);
    else quantize_tile<T, SQUARE, VEC, false>(p, reinterpret_cast<T*>(dyn), warp_max, rb, cb);
}

template <typename T, bool SQUARE, bool VEC>
static cudaError_t quantize_v(const QuantParams& p, cudaStream_t stream) {
    static SmemOptIn opt;
    const size_t smem = p.qt.q ? 128 * kQuantPitch * sizeof(T) : 0;
    const cudaError_t e = ensure_dynamic_smem(k_quantize<T, SQUARE, VEC>, smem, opt);
    if (e != cudaSuccess) return e;
    const long long tiles = ((p.cols + 127) / 128) * ((p.rows + 127) / 128);
    return launch_pdl(k_quantize<T, SQUARE, VEC>, dim3((unsigned)tiles), dim3(QuantShape<T>::kThreads), smem, stream, p);
}
template <typename T>
static cudaError_t quantize_t(const QuantParams& p, cudaStream_t stream) {
    const bool square = p.q.q ? p.q.square : p.qt.square;
    const bool vec = (reinterpret_cast<uintptr_t>(p.x) & (4 * sizeof(T) - 1)) == 0 && p.ldx % 4 == 0;
    if (square) return vec ? quantize_v<T, true, true>(p, stream) : quantize_v<T, true, false>(p, stream);
    return vec ? quantize_v<T, false, true>(p, stream) : quantize_v<T, false, false>(p, stream);
}
cudaError_t launch_quantize(const QuantParams& p, int x_type, cudaStream_t stream) {
    return x_type == DST_F32 ? quantize_t<float>(p, stream) : quantize_t<__nv_bfloat16>(p, stream);
}

// ---- product (dst_block_matmul.cuh) -----------------------------------------------
size_t matmul_fp8_workspace(long long M, long long N, long long K) { return block_matmul_workspace<Fp8Kind>(M, N, K); }
size_t matmul_fp8_workspace_bound(long long M, long long N, long long K) { return block_matmul_workspace_bound<Fp8Kind>(M, N, K); }
cudaError_t launch_matmul_fp8(const Fp8View& a, const Fp8View& b, void* out, long long ldo, int out_type, void* workspace, int sms, cudaStream_t stream) {
    return launch_block_matmul<Fp8Kind>(a, b, out, ldo, out_type, workspace, sms, stream);
}

// A few rows of x against a whole weight, quantised by every CTA for itself while the weight's first tiles are on their way:
// where they fit next to the ring of stages, the inner dimension stays whole, and the blocks are few enough for the four
// epilogue warps (against the two-kernel form, 33,708 x 1024: 1 row 7.9 and 10.3 us, 4 rows 9.1 and 10.3, 6 rows 10.8 and 10.7,
// 16 rows 15.0 and 11.0).  The work before the first tile is the same whatever the vocabulary, and the limit holds for small
// ones and for few columns too: at the most rows it takes, 6.2 and 6.3 us for 16 rows of 33,708 x 256, 5.2 and 6.0 of x 128, 15.6 and
// 17.2 for 2 rows of x 2048; 4.7 and 5.9 for 16 rows of 1000 x 64, 5.9 and 6.6 for 8 of x 512, 7.3 and 8.1 for 4 of x 1024;
// 4.4 and 5.4 for 16 of 200 x 128.
bool linear_fp8_fused(long long M, long long N, long long K) {
    const MatmulPlan L = plan_matmul<Fp8Kind>(M, N, K);
    return block_linear_fits<Fp8Kind>(L) && M * L.blocks <= 40;
}
cudaError_t launch_linear_fp8_fused(const void* x, long long ldx, int x_type, long long M, const Fp8View& w, void* out, long long ldo, int out_type,
                                    int sms, cudaStream_t stream) {
    return launch_block_linear<Fp8Kind>(x, ldx, x_type, M, w, out, ldo, out_type, sms, stream);
}

}  // namespace dst
