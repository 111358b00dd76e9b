// Root-mean-square norm of the residual stream with the addition of a sub-layer's output, to 32, 16 or 8 bits, and its gradient.
//
// A row belongs to a team of warps, 16 elements a lane (32 above 8192 columns), one warp up to 512 columns; a CTA has several teams,
// each with every so many-th row.  A row's elements stay in registers between the sum of squares and the result, and the next row's
// are on their way meanwhile: every element crosses from memory and to it once, and memory's time is the floor.
//
// The weight's gradient: a lane adds up its columns over its rows, the CTA's teams are added in their order and the CTAs' shares in
// theirs, so the order follows from the sizes alone.
//
// Measured, with the residual: 8192 x 512 bf16 6.8 us forward, 11.9 backward (3 of them the joining of the weight's shares; 33.5 MB each way need 5.1); 12,801 x
// 1021 fp32, unaligned, 35 and 38 us (209 MB need 31.9).  To 8 bits, without and with a result in bf16: 8192 x 512 7.8 and 8.8 us (29.4 and 37.7 MB need 4.5 and
// 5.8), 8192 x 1024 13.0 and 14.7 (9.0 and 11.5), 48 x 1024 1.9 and 2.0.
//
// Above 8192 columns a lane's 32 elements and, in the gradient, as many of the weight's leave 128 registers short: the gradient spills 390 to 520 bytes a thread, the forward
// pass 136 at most.  2048 x 16,384 bf16 49 us forward, 114 backward (90 without the weight's gradient; 40.9 needed each way), fp32 89 and 138 (81.8); 2047 x 16,381 bf16,
// unaligned, 166 and 184.  2048 x 8192 bf16 25 and 45 (20.5), fp32 43 and 52 (40.9).
#include "dst_fp8.cuh"
#include "dst_step.cuh"

namespace dst {

constexpr int kNormOnSm = 2;                 // CTAs of eight warps and 128 registers that fit an SM (the forward kernel on 8192 x 512 bf16: 6.8 us, with three of 80 registers 6.5,
                                             // but 12,801 x 1021 fp32 38.6 against 35.0)
constexpr int kNormWarps = 8;                // of a CTA, at most where a team has fewer

// How a lane's elements lie in a row.  8 and 4: in vectors of so many, aligned to them; 0: a column a lane, in any place.
template <int MODE, int PER> struct Place {
    int col0, d;
    __device__ __forceinline__ Place(int warp, int columns) : col0(warp * PER * 32 + lane_id() * (MODE ? MODE : 1)), d(columns) {}
    static __device__ __forceinline__ constexpr int step(int i) { return MODE ? i / MODE * (MODE * 32) + i % MODE : i * 32; }
    __device__ __forceinline__ int col(int i) const { return col0 + step(i); }
    __device__ __forceinline__ bool here(int i) const { return col(i) < d; }
};

// A lane's elements of one row as they are stored.
template <typename T, int MODE, int PER> struct Elements {
    static constexpr int kBits = 8 * (int)sizeof(T);
    unsigned w[MODE == 0 ? PER : PER * kBits / 32];
    __device__ __forceinline__ void load(const T* row, const Place<MODE, PER>& at) {
        if constexpr (MODE == 0) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                w[i] = 0u;
                if (at.here(i)) {
                    if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(row[at.col(i)]);
                    else w[i] = (unsigned)__bfloat16_as_ushort(row[at.col(i)]) << 16;
                }
            }
        } else {
            constexpr int kWords = MODE * kBits / 32;
#pragma unroll
            for (int v = 0; v < PER / MODE; ++v) {
                const bool in = at.here(v * MODE);
                const T* const from = row + at.col(v * MODE);
#pragma unroll
                for (int j = 0; j < kWords; j += 4) {
                    unsigned* const to = w + v * kWords + j;
                    if constexpr (kWords == 2) {
                        const uint2 x = in ? *reinterpret_cast<const uint2*>(from) : make_uint2(0u, 0u);
                        to[0] = x.x; to[1] = x.y;
                    } else {
                        const uint4 x = in ? reinterpret_cast<const uint4*>(from)[j / 4] : make_uint4(0u, 0u, 0u, 0u);
                        to[0] = x.x; to[1] = x.y; to[2] = x.z; to[3] = x.w;
                    }
                }
            }
        }
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 4 || MODE == 0) return __uint_as_float(w[i]);
        else return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    }
    // rounds v and keeps it
    __device__ __forceinline__ void set(const float (&v)[PER]) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < PER; ++i) w[i] = __float_as_uint(v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < PER; i += 2) {
                const unsigned both = pack_bf16(v[i], v[i + 1]);
                if constexpr (MODE == 0) { w[i] = both << 16; w[i + 1] = both & 0xFFFF0000u; }
                else w[i / 2] = both;
            }
        }
    }
    __device__ __forceinline__ void store(T* row, const Place<MODE, PER>& at) const {
        if constexpr (MODE == 0) {
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (at.here(i)) {
                    if constexpr (sizeof(T) == 4) row[at.col(i)] = __uint_as_float(w[i]);
                    else row[at.col(i)] = __ushort_as_bfloat16((unsigned short)(w[i] >> 16));
                }
        } else {
            constexpr int kWords = MODE * kBits / 32;
#pragma unroll
            for (int v = 0; v < PER / MODE; ++v) {
                if (!at.here(v * MODE)) continue;
                T* const to = row + at.col(v * MODE);
#pragma unroll
                for (int j = 0; j < kWords; j += 4) {
                    const unsigned* const x = w + v * kWords + j;
                    if constexpr (kWords == 2) *reinterpret_cast<uint2*>(to) = make_uint2(x[0], x[1]);
                    else reinterpret_cast<uint4*>(to)[j / 4] = make_uint4(x[0], x[1], x[2], x[3]);
                }
            }
        }
    }
};
template <typename T, int MODE, int PER>
__device__ __forceinline__ void store_row(void* out, long long offset, const Place<MODE, PER>& at, const float (&v)[PER]) {
    Elements<T, MODE, PER> e;
    e.set(v);
    e.store(static_cast<T*>(out) + offset, at);
}
template <typename T, int MODE, int PER>
__device__ __forceinline__ void load_row(const void* from, long long offset, const Place<MODE, PER>& at, float (&v)[PER]) {
    Elements<T, MODE, PER> e;
    e.load(static_cast<const T*>(from) + offset, at);
#pragma unroll
    for (int i = 0; i < PER; ++i) v[i] = e.get(i);
}
template <int MODE, int PER>
__device__ __forceinline__ void load_weight(const float* weight, const Place<MODE, PER>& at, float (&w)[PER]) {
    Elements<float, MODE, PER> e;
    if (weight) e.load(weight, at);
#pragma unroll
    for (int i = 0; i < PER; ++i) w[i] = weight ? e.get(i) : 1.f;
}

// The sum over a row's warps, which meet at their own barrier.  `part` is used by turns, so that a row's sums are read before the row
// after the next one writes.
__device__ __forceinline__ float team_sum(float x, int team, float* part) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
    if (team == 1) return x;
    const int first = warp_id() / team * team;
    if (lane_id() == 0) part[warp_id()] = x;
    asm volatile("bar.sync %0, %1;" ::"r"(1 + warp_id() / team), "r"(team * 32) : "memory");
    x = 0.f;
    for (int w = 0; w < team; ++w) x += part[first + w];
    return x;
}

// a row's blocks of 128 columns in 8 bits
template <int MODE, int PER>
__device__ __forceinline__ void store_fp8(const Fp8View& q, long long row, const Place<MODE, PER>& at, const float (&y)[PER]) {
    constexpr int kOf = MODE == 8 ? 8 : 4;                                 // a lane's elements of a block, and the lanes that hold it
    constexpr int kLanes = MODE == 8 ? 16 : 32;
#pragma unroll
    for (int v = 0; v < PER; v += kOf) {
        unsigned top = 0;
#pragma unroll
        for (int i = 0; i < kOf; ++i) top = max(top, float_abs(y[v + i]));
        if constexpr (kLanes == 32) top = __reduce_max_sync(0xFFFFFFFFu, top);
        else
#pragma unroll
            for (int d = 1; d < kLanes; d *= 2) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
        const float u = block_inverse(top);
        uint8_t* const to = q.q + row * q.ld;
        if constexpr (MODE == 0) {
#pragma unroll
            for (int i = 0; i < kOf; i += 2) {
                const unsigned two = to_e4m3x4(y[v + i] * u, y[v + i + 1] * u, 0.f, 0.f);
                if (at.here(v + i)) to[at.col(v + i)] = (uint8_t)two;
                if (at.here(v + i + 1)) to[at.col(v + i + 1)] = (uint8_t)(two >> 8);
            }
        } else if (at.here(v)) {
#pragma unroll
            for (int i = 0; i < kOf; i += 4)
                reinterpret_cast<unsigned*>(to + at.col(v))[i / 4] = to_e4m3x4(y[v + i] * u, y[v + i + 1] * u, y[v + i + 2] * u, y[v + i + 3] * u);
        }
        if (lane_id() % kLanes == 0 && at.here(v)) *scale_byte(q, row, at.col(v) >> 7) = (uint8_t)block_exponent(top);
    }
}

template <typename XT, typename ST, int MODE, int PER>
__global__ void __launch_bounds__(512) k_rmsnorm(const __grid_constant__ NormParams p, int team, int out_type) {
    __shared__ float parts[2][16];
    const int teams = blockDim.x / 32 / team;
    const Place<MODE, PER> at(warp_id() % team, p.d);
    const long long step = (long long)gridDim.x * teams;
    long long row = (long long)blockIdx.x * teams + warp_id() / team;
    pdl_trigger();
    pdl_wait();
    if (row >= p.rows) return;
    Elements<XT, MODE, PER> x;
    Elements<ST, MODE, PER> r;
    constexpr bool kAhead = PER == 16;                                     // (32 elements of the next row do not fit the registers)
    auto load = [&](long long of) {
        x.load(static_cast<const XT*>(p.x) + of * p.ldx, at);
        if (p.residual) r.load(static_cast<const ST*>(p.residual) + of * p.ldr, at);
    };
    if (kAhead) load(row);
    float w[PER];
    load_weight<MODE, PER>(p.weight, at, w);
    const float each = 1.f / (float)p.d;
    for (int turn = 0; row < p.rows; row += step, turn ^= 1) {
        if (!kAhead) load(row);
        float h[PER], sum = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) h[i] = p.residual ? x.get(i) + r.get(i) : x.get(i);
        if (kAhead && row + step < p.rows) load(row + step);
        if (p.keep) {                                                      // the norm is that of the stream as it is stored
            Elements<ST, MODE, PER> s;
            s.set(h);
#pragma unroll
            for (int i = 0; i < PER; ++i) h[i] = s.get(i);
            if (p.sum_out) s.store(static_cast<ST*>(p.sum_out) + row * p.lds, at);
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) sum = fmaf(h[i], h[i], sum);
        const float inv = rsqrtf(fmaf(team_sum(sum, team, parts[turn]), each, p.eps));
        if (p.inv_rms && at.col0 == 0) p.inv_rms[row] = inv;
#pragma unroll
        for (int i = 0; i < PER; ++i) h[i] = h[i] * inv * w[i];
        if (p.out) {
            if (out_type == DST_F32) store_row<float, MODE, PER>(p.out, row * p.ldo, at, h);
            else store_row<__nv_bfloat16, MODE, PER>(p.out, row * p.ldo, at, h);
        }
        if (p.q.q) {
#pragma unroll
            for (int i = 0; i < PER; ++i) if (!at.here(i)) h[i] = 0.f;      // (an infinite inv_rms times nothing)
            store_fp8<MODE, PER>(p.q, row, at, h);
        }
    }
}

template <typename DT, typename HT, int MODE, int PER>
__global__ void __launch_bounds__(512) k_rmsnorm_backward(const __grid_constant__ NormBackParams p, int team, int dx_type) {
    extern __shared__ float shares[];                                      // [teams][team * PER * 32], with the weight's gradient and several teams
    __shared__ float parts[2][16];
    const int teams = blockDim.x / 32 / team;
    const Place<MODE, PER> at(warp_id() % team, p.d);
    const long long step = (long long)gridDim.x * teams;
    long long row = (long long)blockIdx.x * teams + warp_id() / team;
    pdl_trigger();
    pdl_wait();
    Elements<DT, MODE, PER> y;
    Elements<HT, MODE, PER> h;
    float inv = 0.f;
    auto load = [&](long long of) {
        y.load(static_cast<const DT*>(p.dy) + of * p.ldy, at);
        h.load(static_cast<const HT*>(p.h) + of * p.ldh, at);
        inv = p.inv_rms[of];
    };
    constexpr bool kAhead = PER == 16;                                     // (32 elements of the next row do not fit the registers)
    if (kAhead && row < p.rows) load(row);
    float w[PER], dw[PER];
    load_weight<MODE, PER>(p.weight, at, w);
#pragma unroll
    for (int i = 0; i < PER; ++i) dw[i] = 0.f;
    const float each = 1.f / (float)p.d;
    for (int turn = 0; row < p.rows; row += step, turn ^= 1) {
        if (!kAhead) load(row);
        float u[PER], g[PER], along = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            u[i] = h.get(i) * inv;
            g[i] = y.get(i);
            dw[i] = fmaf(g[i], u[i], dw[i]);
            g[i] *= w[i];
            along = fmaf(g[i], u[i], along);
        }
        const float scale = inv;
        float ds[PER] = {};
        if (p.dsum) {
            if (dx_type == DST_F32) load_row<float, MODE, PER>(p.dsum, row * p.ldds, at, ds);
            else load_row<__nv_bfloat16, MODE, PER>(p.dsum, row * p.ldds, at, ds);
        }
        if (kAhead && row + step < p.rows) load(row + step);
        along = team_sum(along, team, parts[turn]) * each;
#pragma unroll
        for (int i = 0; i < PER; ++i) g[i] = fmaf(scale, fmaf(-u[i], along, g[i]), ds[i]);
        if (dx_type == DST_F32) store_row<float, MODE, PER>(p.dx, row * p.lddx, at, g);
        else store_row<__nv_bfloat16, MODE, PER>(p.dx, row * p.lddx, at, g);
    }
    if (!p.parts) return;
    float* const out = p.parts + (long long)blockIdx.x * p.d;
    if (teams > 1) {
        const int pitch = team * PER * 32;
#pragma unroll
        for (int i = 0; i < PER; ++i) shares[warp_id() / team * pitch + at.col(i)] = dw[i];
        __syncthreads();
        for (int c = threadIdx.x; c < p.d; c += blockDim.x) {
            float v = 0.f;
            for (int t = 0; t < teams; ++t) v += shares[t * pitch + c];
            out[c] = v;
        }
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) if (at.here(i)) out[at.col(i)] = dw[i];
    }
}

// dweight[c] = the CTAs' shares in their order: 32 columns a CTA, each of its warps a run of the shares
constexpr int kShareWarps = 32;
__global__ void __launch_bounds__(kShareWarps * 32) k_norm_dweight(const float* parts, int n, int d, float* dweight) {
    __shared__ float sums[kShareWarps][32];
    pdl_trigger();
    pdl_wait();
    const int c = blockIdx.x * 32 + lane_id(), from = n * warp_id() / kShareWarps, to = n * (warp_id() + 1) / kShareWarps;
    float v = 0.f;
    if (c < d)
#pragma unroll 8
        for (int i = from; i < to; ++i) v += parts[(long long)i * d + c];
    sums[warp_id()][lane_id()] = v;
    __syncthreads();
    if (warp_id() == 0 && c < d) {
#pragma unroll 8
        for (int w = 1; w < kShareWarps; ++w) v += sums[w][lane_id()];
        dweight[c] = v;
    }
}

// ---- host -------------------------------------------------------------------------
struct NormShape { int per, team, warps; long long ctas; };
// CTAs: as many as rows give teams, up to `most`.  (Of a B200's SMs, not the device's: the order of the weight's sums follows from the
// sizes.)
static NormShape norm_shape(long long rows, long long d, long long most) {
    NormShape s{16, 1, 0, 0};
    if (d > 8192) s.per = 32;
    while ((long long)s.team * s.per * 32 < d) s.team *= 2;
    int teams = s.team < kNormWarps ? kNormWarps / s.team : 1;
    // few rows: spread over the SMs (forward, 48 x 512 bf16 1.5 us against 1.6, 150 x 1024 fp32 1.9 against 2.9)
    while (teams > 1 && rows <= (long long)kSmCount * teams / 2) teams /= 2;
    s.warps = teams * s.team;
    const long long all = (rows + teams - 1) / teams;
    s.ctas = all < most ? all : most;
    return s;
}
// the largest of 8, 4 and 0 that rows at p with this leading dimension are aligned to, in elements
static int rows_mode(const void* p, long long ld, int type) {
    const size_t size = type == DST_F32 ? 4 : 2;
    if (!p) return 8;
    const uintptr_t a = reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * size);
    return a % 16 == 0 ? 8 : a % (4 * size) == 0 ? 4 : 0;
}
template <typename... M> static int least(int a, M... more) {
    int m = a;
    ((m = more < m ? more : m), ...);
    return m;
}

template <typename XT, typename ST, int MODE>
static cudaError_t norm_m(const NormParams& p, int out_type, cudaStream_t stream) {
    const NormShape s = norm_shape(p.rows, p.d, kNormOnSm * kSmCount);
    const dim3 grid((unsigned)s.ctas), block(s.warps * 32);
    return s.per == 16 ? launch_pdl(k_rmsnorm<XT, ST, MODE, 16>, grid, block, 0, stream, p, s.team, out_type)
                       : launch_pdl(k_rmsnorm<XT, ST, MODE, 32>, grid, block, 0, stream, p, s.team, out_type);
}
template <typename XT, typename ST>
static cudaError_t norm_s(const NormParams& p, int mode, int out_type, cudaStream_t stream) {
    return mode == 8 ? norm_m<XT, ST, 8>(p, out_type, stream) : mode == 4 ? norm_m<XT, ST, 4>(p, out_type, stream) : norm_m<XT, ST, 0>(p, out_type, stream);
}
// All rows in fp32 take vectors of four: neighbouring lanes then hold neighbouring 16 bytes (8192 x 4096: 88 us against 97 with eight).
static int norm_mode(int mode, long long d, bool all32) {
    if (d % 8 != 0 && mode == 8) mode = 4;
    if (d % 4 != 0) mode = 0;
    return mode == 8 && all32 ? 4 : mode;
}
cudaError_t launch_rmsnorm(const NormParams& p, int x_type, int sum_type, int out_type, cudaStream_t stream) {
    const int mode = norm_mode(least(rows_mode(p.x, p.ldx, x_type), rows_mode(p.residual, p.ldr, sum_type), rows_mode(p.sum_out, p.lds, sum_type),
                                     rows_mode(p.out, p.ldo, out_type), rows_mode(p.weight, 0, DST_F32)),
                               p.d, x_type == DST_F32 && sum_type == DST_F32 && (!p.out || out_type == DST_F32));
    if (x_type == DST_F32) return sum_type == DST_F32 ? norm_s<float, float>(p, mode, out_type, stream) : norm_s<float, __nv_bfloat16>(p, mode, out_type, stream);
    return sum_type == DST_F32 ? norm_s<__nv_bfloat16, float>(p, mode, out_type, stream) : norm_s<__nv_bfloat16, __nv_bfloat16>(p, mode, out_type, stream);
}

static NormShape back_shape(long long rows, long long d) { return norm_shape(rows, d, kNormOnSm * kSmCount); }
size_t rmsnorm_backward_workspace(long long rows, long long d) { return size_t(back_shape(rows, d).ctas) * size_t(d) * 4; }

template <typename DT, typename HT, int MODE, int PER>
static cudaError_t back_run(const NormBackParams& p, const NormShape& s, int dx_type, cudaStream_t stream) {
    static SmemOptIn opt;
    const size_t smem = s.warps > s.team && p.parts ? size_t(s.warps) * PER * 32 * 4 : 0;
    cudaError_t e = ensure_dynamic_smem(k_rmsnorm_backward<DT, HT, MODE, PER>, smem, opt);
    if (e != cudaSuccess) return e;
    e = launch_pdl(k_rmsnorm_backward<DT, HT, MODE, PER>, dim3((unsigned)s.ctas), dim3(s.warps * 32), smem, stream, p, s.team, dx_type);
    if (e != cudaSuccess || !p.parts) return e;
    return launch_pdl(k_norm_dweight, dim3((p.d + 31) / 32), dim3(kShareWarps * 32), 0, stream, static_cast<const float*>(p.parts), (int)s.ctas, p.d, p.dweight);
}
template <typename DT, typename HT, int MODE>
static cudaError_t back_m(const NormBackParams& p, int dx_type, cudaStream_t stream) {
    const NormShape s = back_shape(p.rows, p.d);
    return s.per == 16 ? back_run<DT, HT, MODE, 16>(p, s, dx_type, stream) : back_run<DT, HT, MODE, 32>(p, s, dx_type, stream);
}
template <typename DT, typename HT>
static cudaError_t back_h(const NormBackParams& p, int mode, int dx_type, cudaStream_t stream) {
    return mode == 8 ? back_m<DT, HT, 8>(p, dx_type, stream) : mode == 4 ? back_m<DT, HT, 4>(p, dx_type, stream) : back_m<DT, HT, 0>(p, dx_type, stream);
}
cudaError_t launch_rmsnorm_backward(const NormBackParams& p, int dy_type, int h_type, int dx_type, cudaStream_t stream) {
    const int mode = norm_mode(least(rows_mode(p.dy, p.ldy, dy_type), rows_mode(p.h, p.ldh, h_type), rows_mode(p.dsum, p.ldds, dx_type),
                                     rows_mode(p.dx, p.lddx, dx_type), rows_mode(p.weight, 0, DST_F32)),
                               p.d, dy_type == DST_F32 && h_type == DST_F32 && dx_type == DST_F32);
    if (dy_type == DST_F32) return h_type == DST_F32 ? back_h<float, float>(p, mode, dx_type, stream) : back_h<float, __nv_bfloat16>(p, mode, dx_type, stream);
    return h_type == DST_F32 ? back_h<__nv_bfloat16, float>(p, mode, dx_type, stream) : back_h<__nv_bfloat16, __nv_bfloat16>(p, mode, dx_type, stream);
}

}  // namespace dst
