// Root-mean-square norm of the residual stream with the addition of a sub-layer's output, to 32, 16 or 8 bits, and its gradient.
//
// A row belongs to as many warps as hold it at 32 elements a lane (1 up to 1024 columns, 16 at most), four neighbouring
// columns a lane and load, so that the 128 columns of a warp's load are one block of the 8-bit form.  Every element is read
// once, stays in registers while the row's sum of squares is formed, and is written once: memory's time is the floor.
#include "dst_step.cuh"
#include "dst_fp8.cuh"

namespace dst {

constexpr int kNormWarps = 8;                // of a CTA, or the row's warps where they are more
constexpr int kNormGroups = 8;               // groups of four elements a lane
constexpr int kNormWarpCols = kNormGroups * 128;

// four neighbouring elements, aligned to their size together (VEC) or not
template <typename T, bool VEC> __device__ __forceinline__ void load4(const T* p, int n, float (&v)[4]) {
    if constexpr (VEC) {
        if constexpr (sizeof(T) == 4) {
            const float4 a = *reinterpret_cast<const float4*>(p);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        } else {
            const uint2 a = *reinterpret_cast<const uint2*>(p);
            v[0] = __uint_as_float(a.x << 16); v[1] = __uint_as_float(a.x & 0xFFFF0000u);
            v[2] = __uint_as_float(a.y << 16); v[3] = __uint_as_float(a.y & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < n ? to_float<T>(p[i]) : 0.f;
    }
}
template <typename T, bool VEC> __device__ __forceinline__ void store4(T* p, int n, const float (&v)[4]) {
    if constexpr (VEC) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
        else *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) if (i < n) p[i] = from_float<T>(v[i]);
    }
}

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
    return x;
}
// over the `team` warps of a row; every thread of the CTA takes part.  `part` is used by turns, so that a row's sums are read
// before the row after the next one writes
__device__ __forceinline__ float row_sum(float x, int team, float* part) {
    x = warp_sum(x);
    if (team == 1) return x;
    if (lane_id() == 0) part[warp_id()] = x;
    __syncthreads();
    float s = 0.f;
    const int first = warp_id() / team * team;
    for (int w = 0; w < team; ++w) s += part[first + w];
    return s;
}

template <typename XT, typename ST, typename OT, bool VEC>
__global__ void __launch_bounds__(512) k_rmsnorm(const __grid_constant__ NormParams p, int team) {
    __shared__ float parts[16];
    const int lane = lane_id(), teams = blockDim.x / 32 / team;
    const long long row = (long long)blockIdx.x * teams + warp_id() / team;
    const int col0 = warp_id() % team * kNormWarpCols + lane * 4;
    const bool mine = row < p.rows;
    pdl_trigger();
    pdl_wait();
    float h[kNormGroups][4];
    const XT* const x = static_cast<const XT*>(p.x) + row * p.ldx + col0;
#pragma unroll
    for (int j = 0; j < kNormGroups; ++j) {
        const int left = mine ? p.d - col0 - j * 128 : 0;
        if (left > 0) load4<XT, VEC>(x + j * 128, left, h[j]);
        else h[j][0] = h[j][1] = h[j][2] = h[j][3] = 0.f;
    }
    if (p.residual) {
        const ST* const r = static_cast<const ST*>(p.residual) + row * p.ldr + col0;
        float v[kNormGroups][4];
#pragma unroll
        for (int j = 0; j < kNormGroups; ++j) {
            const int left = mine ? p.d - col0 - j * 128 : 0;
            if (left > 0) load4<ST, VEC>(r + j * 128, left, v[j]);
            else v[j][0] = v[j][1] = v[j][2] = v[j][3] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < kNormGroups; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) h[j][i] += v[j][i];
    }
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < kNormGroups; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (p.keep) h[j][i] = to_float<ST>(from_float<ST>(h[j][i]));   // the norm is that of the stream as it is stored
            sum = fmaf(h[j][i], h[j][i], sum);
        }
    if (p.sum_out) {
        ST* const s = static_cast<ST*>(p.sum_out) + row * p.lds + col0;
#pragma unroll
        for (int j = 0; j < kNormGroups; ++j) {
            const int left = mine ? p.d - col0 - j * 128 : 0;
            if (left > 0) store4<ST, VEC>(s + j * 128, left, h[j]);
        }
    }
    const float inv = rsqrtf(row_sum(sum, team, parts) / (float)p.d + p.eps);
    if (!mine) return;
    if (p.inv_rms && col0 == 0) p.inv_rms[row] = inv;
    OT* const out = static_cast<OT*>(p.out) + row * p.ldo + col0;
#pragma unroll
    for (int j = 0; j < kNormGroups; ++j) {
        const int left = p.d - col0 - j * 128;
        if (left + lane * 4 <= 0) break;                                   // (the whole warp's columns are past the row)
        float y[4] = {0.f, 0.f, 0.f, 0.f};
        if (left > 0) {
            float w[4] = {1.f, 1.f, 1.f, 1.f};
            if (p.weight) load4<float, VEC>(p.weight + col0 + j * 128, left, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = i < left ? h[j][i] * inv * w[i] : 0.f;
            if (p.out) store4<OT, VEC>(out + j * 128, left, y);
        }
        if (p.q.q) {
            const unsigned top = __reduce_max_sync(0xFFFFFFFFu, max(max(float_abs(y[0]), float_abs(y[1])), max(float_abs(y[2]), float_abs(y[3]))));
            const float u = block_inverse(top);
            if (left > 0) *reinterpret_cast<unsigned*>(p.q.q + row * p.q.ld + col0 + j * 128) = to_e4m3x4(y[0] * u, y[1] * u, y[2] * u, y[3] * u);
            if (lane == 0) *scale_byte(p.q, row, (col0 + j * 128) >> 7) = (uint8_t)block_exponent(top);
        }
    }
}

// A CTA takes every gridDim.x-th group of rows and keeps its columns' share of the weight's gradient in registers; the CTAs' shares
// are added in their order by k_norm_dweight.
template <typename DT, typename HT, typename XT, bool VEC>
__global__ void __launch_bounds__(512) k_rmsnorm_backward(const __grid_constant__ NormBackParams p, int team) {
    extern __shared__ float shares[];                                      // [teams][team * kNormWarpCols], teams > 1
    __shared__ float parts[2][16];
    const int lane = lane_id(), teams = blockDim.x / 32 / team;
    const int col0 = warp_id() % team * kNormWarpCols + lane * 4;
    float w[kNormGroups][4], dw[kNormGroups][4];
    pdl_trigger();
    pdl_wait();
#pragma unroll
    for (int j = 0; j < kNormGroups; ++j) {
        const int left = p.d - col0 - j * 128;
#pragma unroll
        for (int i = 0; i < 4; ++i) { w[j][i] = 1.f; dw[j][i] = 0.f; }
        if (p.weight && left > 0) load4<float, VEC>(p.weight + col0 + j * 128, left, w[j]);
    }
    int turn = 0;
    for (long long row0 = (long long)blockIdx.x * teams; row0 < p.rows; row0 += (long long)gridDim.x * teams, turn ^= 1) {
        const long long row = row0 + warp_id() / team;
        const bool mine = row < p.rows;
        const float inv = mine ? p.inv_rms[row] : 0.f;
        float u[kNormGroups][4], g[kNormGroups][4];
        const DT* const dy = static_cast<const DT*>(p.dy) + row * p.ldy + col0;
        const HT* const h = static_cast<const HT*>(p.h) + row * p.ldh + col0;
#pragma unroll
        for (int j = 0; j < kNormGroups; ++j) {
            const int left = mine ? p.d - col0 - j * 128 : 0;
            if (left > 0) { load4<DT, VEC>(dy + j * 128, left, g[j]); load4<HT, VEC>(h + j * 128, left, u[j]); }
            else { g[j][0] = g[j][1] = g[j][2] = g[j][3] = 0.f; u[j][0] = u[j][1] = u[j][2] = u[j][3] = 0.f; }
        }
        float along = 0.f;
#pragma unroll
        for (int j = 0; j < kNormGroups; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                u[j][i] *= inv;
                dw[j][i] = fmaf(g[j][i], u[j][i], dw[j][i]);
                g[j][i] *= w[j][i];
                along = fmaf(g[j][i], u[j][i], along);
            }
        along = row_sum(along, team, parts[turn]) / (float)p.d;
        if (!mine) continue;
        XT* const dx = static_cast<XT*>(p.dx) + row * p.lddx + col0;
        const XT* const ds = static_cast<const XT*>(p.dsum) + row * p.ldds + col0;
#pragma unroll
        for (int j = 0; j < kNormGroups; ++j) {
            const int left = p.d - col0 - j * 128;
            if (left <= 0) break;
            float v[4] = {0.f, 0.f, 0.f, 0.f};
            if (p.dsum) load4<XT, VEC>(ds + j * 128, left, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = fmaf(inv, fmaf(-u[j][i], along, g[j][i]), v[i]);
            store4<XT, VEC>(dx + j * 128, left, v);
        }
    }
    if (!p.parts) return;
    float* const out = p.parts + (long long)blockIdx.x * p.d;
    if (teams > 1) {
        const int pitch = team * kNormWarpCols;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kNormGroups; ++j) *reinterpret_cast<float4*>(shares + warp_id() / team * pitch + col0 + j * 128) = make_float4(dw[j][0], dw[j][1], dw[j][2], dw[j][3]);
        __syncthreads();
        for (int c = threadIdx.x; c < p.d; c += blockDim.x) {
            float v = 0.f;
            for (int t = 0; t < teams; ++t) v += shares[t * pitch + c];
            out[c] = v;
        }
    } else {
#pragma unroll
        for (int j = 0; j < kNormGroups; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) if (col0 + j * 128 + i < p.d) out[col0 + j * 128 + i] = dw[j][i];
    }
}

// dweight[c] = the CTAs' shares in their order: 32 columns a CTA, its eight warps an eighth of the shares each
__global__ void __launch_bounds__(256) k_norm_dweight(const float* __restrict__ parts, int n, int d, float* __restrict__ dweight) {
    __shared__ float sums[8][32];
    pdl_trigger();
    pdl_wait();
    const int c = blockIdx.x * 32 + lane_id(), from = n * warp_id() / 8, to = n * (warp_id() + 1) / 8;
    float v = 0.f;
    if (c < d) for (int i = from; i < to; ++i) v += parts[(long long)i * d + c];
    sums[warp_id()][lane_id()] = v;
    __syncthreads();
    if (warp_id() == 0 && c < d) {
        for (int w = 1; w < 8; ++w) v += sums[w][lane_id()];
        dweight[c] = v;
    }
}

static int norm_team(int d) {
    int t = 1;
    while (t * kNormWarpCols < d) t *= 2;
    return t;
}
static bool rows_aligned(const void* p, long long ld, size_t size) { return !p || ((reinterpret_cast<uintptr_t>(p) & (4 * size - 1)) == 0 && ld % 4 == 0); }
static size_t bytes_of(int type) { return type == DST_F32 ? 4 : 2; }

template <typename XT, typename ST, typename OT>
static cudaError_t norm_t(const NormParams& p, bool vec, cudaStream_t stream) {
    const int team = norm_team(p.d), warps = team > kNormWarps ? team : kNormWarps, teams = warps / team;
    const dim3 grid((unsigned)((p.rows + teams - 1) / teams)), block(warps * 32);
    return vec ? launch_pdl(k_rmsnorm<XT, ST, OT, true>, grid, block, 0, stream, p, team) : launch_pdl(k_rmsnorm<XT, ST, OT, false>, grid, block, 0, stream, p, team);
}
template <typename XT, typename ST>
static cudaError_t norm_o(const NormParams& p, int out_type, bool vec, cudaStream_t stream) {
    return out_type == DST_F32 ? norm_t<XT, ST, float>(p, vec, stream) : norm_t<XT, ST, __nv_bfloat16>(p, vec, stream);
}
template <typename XT>
static cudaError_t norm_s(const NormParams& p, int sum_type, int out_type, bool vec, cudaStream_t stream) {
    return sum_type == DST_F32 ? norm_o<XT, float>(p, out_type, vec, stream) : norm_o<XT, __nv_bfloat16>(p, out_type, vec, stream);
}
cudaError_t launch_rmsnorm(const NormParams& p, int x_type, int sum_type, int out_type, cudaStream_t stream) {
    const bool vec = p.d % 4 == 0 && rows_aligned(p.x, p.ldx, bytes_of(x_type)) && rows_aligned(p.residual, p.ldr, bytes_of(sum_type)) &&
                     rows_aligned(p.sum_out, p.lds, bytes_of(sum_type)) && rows_aligned(p.out, p.ldo, bytes_of(out_type)) && rows_aligned(p.weight, 0, 4);
    return x_type == DST_F32 ? norm_s<float>(p, sum_type, out_type, vec, stream) : norm_s<__nv_bfloat16>(p, sum_type, out_type, vec, stream);
}

// CTAs of the backward pass: two for each SM of a B200 (not the device's: the order of the weight's sums follows from the sizes)
static long long norm_back_ctas(long long rows, int team) {
    const int teams = (team > kNormWarps ? team : kNormWarps) / team;
    const long long all = (rows + teams - 1) / teams, most = 2 * kSmCount;
    return all < most ? all : most;
}
size_t rmsnorm_backward_workspace(long long rows, long long d) { return size_t(norm_back_ctas(rows, norm_team((int)d))) * size_t(d) * 4; }

template <typename DT, typename HT, typename XT, bool VEC>
static cudaError_t norm_back_v(const NormBackParams& p, cudaStream_t stream) {
    static SmemOptIn opt;
    const int team = norm_team(p.d), warps = team > kNormWarps ? team : kNormWarps, teams = warps / team;
    const size_t smem = teams > 1 && p.parts ? size_t(warps) * kNormWarpCols * 4 : 0;
    cudaError_t e = ensure_dynamic_smem(k_rmsnorm_backward<DT, HT, XT, VEC>, smem, opt);
    if (e != cudaSuccess) return e;
    const long long ctas = norm_back_ctas(p.rows, team);
    e = launch_pdl(k_rmsnorm_backward<DT, HT, XT, VEC>, dim3((unsigned)ctas), dim3(warps * 32), smem, stream, p, team);
    if (e != cudaSuccess || !p.parts) return e;
    return launch_pdl(k_norm_dweight, dim3((p.d + 31) / 32), dim3(256), 0, stream, static_cast<const float*>(p.parts), (int)ctas, p.d, p.dweight);
}
template <typename DT, typename HT>
static cudaError_t norm_back_x(const NormBackParams& p, int dx_type, bool vec, cudaStream_t stream) {
    if (dx_type == DST_F32) return vec ? norm_back_v<DT, HT, float, true>(p, stream) : norm_back_v<DT, HT, float, false>(p, stream);
    return vec ? norm_back_v<DT, HT, __nv_bfloat16, true>(p, stream) : norm_back_v<DT, HT, __nv_bfloat16, false>(p, stream);
}
cudaError_t launch_rmsnorm_backward(const NormBackParams& p, int dy_type, int h_type, int dx_type, cudaStream_t stream) {
    const bool vec = p.d % 4 == 0 && rows_aligned(p.dy, p.ldy, bytes_of(dy_type)) && rows_aligned(p.h, p.ldh, bytes_of(h_type)) &&
                     rows_aligned(p.dsum, p.ldds, bytes_of(dx_type)) && rows_aligned(p.dx, p.lddx, bytes_of(dx_type)) && rows_aligned(p.weight, 0, 4);
    if (dy_type == DST_F32) return h_type == DST_F32 ? norm_back_x<float, float>(p, dx_type, vec, stream) : norm_back_x<float, __nv_bfloat16>(p, dx_type, vec, stream);
    return h_type == DST_F32 ? norm_back_x<__nv_bfloat16, float>(p, dx_type, vec, stream) : norm_back_x<__nv_bfloat16, __nv_bfloat16>(p, dx_type, vec, stream);
}

}  // namespace dst
