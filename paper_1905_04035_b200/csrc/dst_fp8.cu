// 8-bit floating point with a power-of-two scale for each block of 128: quantisation and the product of two such matrices.
#include <cuda.h>
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
// D[p, q] = sum over blocks b of sp[b, p] sq[b, q] (P_b Q_b^T): a block's 128 products are summed by the tensor cores
// into tensor memory, then epilogue warps take the partial tile out, scale it and add it to fp32 sums in registers,
// while the tensor cores fill the other of two tensor-memory buffers with the next block.  P is the operand whose rows
// are the 128 lanes of tensor memory, Q the one whose rows are its columns.
//
// Both sides large: two CTAs share a 256 x 256 tile (each holds 128 rows of P, half of Q's rows, and 128 x 256 of
// the result), which halves what an SM has to fetch for a block against a tile of its own: 32 KB where the tensor
// cores take 512 cycles.  One side of at most 128 rows: that side is Q, padded to 16, 32, 64 or 128 rows, and a CTA has
// 128 rows of the other one; the time is that side's bytes.
//
// Warps of a CTA: the epilogue warps (4, or 8 where a warp would otherwise hold more than 128 columns), one that issues
// the copies and one that issues the matrix instructions.  Every wait has a limit; a CTA in which one ran out leaves
// NaN in what it still had to write.
constexpr int kBlockK = 128;                              // one scale's worth of the inner dimension, in bytes too
constexpr int kTileP = 128;                               // rows of P a CTA
constexpr int kSmemMost = 232448;

template <int CG, int NT>
struct TileShape {
    static constexpr int kQRows = NT / CG;                // rows of Q a CTA holds
    static constexpr int kEpiWarps = NT > 128 ? 8 : 4;
    static constexpr int kCols = NT > 128 ? 128 : NT;     // columns of the result an epilogue warp holds
    static constexpr int kThreads = (kEpiWarps + 2) * 32;
    static constexpr int kStageBytes = (kTileP + kQRows) * kBlockK;
    static constexpr int kOutBytes = kEpiWarps * 4096;    // 32 x 32 words a warp, for turning rows into runs
    static constexpr int kHeaderBytes = 3072;
    static constexpr int kFit = (kSmemMost - kOutBytes - kHeaderBytes) / kStageBytes;
    static constexpr int kStages = kFit < 8 ? kFit : 8;
    static constexpr int kSmem = kStages * kStageBytes + kOutBytes + kHeaderBytes;
    static constexpr int kTmemCols = 2 * NT < 32 ? 32 : 2 * NT;
};

struct MatmulParams {
    const float* sp;
    const float* sq;
    long long ld_sp, ld_sq;                               // scales of a block
    int shift_p, shift_q;                                 // 7: a scale for 128 rows
    int rows_p, rows_q;
    int blocks, splits;                                   // blocks of the inner dimension, parts it is cut into
    int tiles_p, tiles_q;
    int swap;                                             // the result is [q, p]
    void* out;
    long long ldo;
    long long split_stride;                               // elements between the parts' results (splits > 1)
};

__device__ __forceinline__ unsigned smem_addr(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(unsigned bar, unsigned count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_expect(unsigned bar, unsigned bytes) { asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory"); }
// (what is handed over here is tensor memory, ordered by the tcgen05 fences around it; a release at cluster scope would
// wait for all of the thread's memory traffic: 935 -> ... )
__device__ __forceinline__ void bar_arrive_cluster(unsigned bar) { asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ bool bar_try(unsigned bar, unsigned parity) {
    unsigned done;
    asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.b32 %0, 1, 0, p; }"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
__device__ __forceinline__ bool bar_wait(unsigned bar, unsigned parity) {
    if (bar_try(bar, parity)) return true;
    const long long t0 = clock64();
    while (!bar_try(bar, parity))
        if (clock64() - t0 > kWaitCycles) return false;
    return true;
}
__device__ __forceinline__ unsigned in_cta(unsigned addr, unsigned rank) {   // the same place in another CTA of the cluster
    unsigned r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
template <int CG>
__device__ __forceinline__ void copy_tile(unsigned dst, const CUtensorMap* map, int x, int y, unsigned bar) {
    if (CG == 2)
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
template <int CG>
__device__ __forceinline__ void mma_fp8(unsigned d, uint64_t a, uint64_t b, unsigned idesc, unsigned accumulate) {
    if (CG == 2)
        asm volatile("{ .reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p; }"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile("{ .reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p; }"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// arrives at `bar` (CG == 2: at that place in both CTAs) once the matrix instructions issued so far are done
template <int CG>
__device__ __forceinline__ void mma_commit(unsigned bar) {
    if (CG == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((unsigned short)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_load16(unsigned addr, float (&v)[16]) {
    unsigned r[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
// The loads' registers are inputs and outputs here, so that nothing that reads them moves above the wait.
__device__ __forceinline__ void tmem_wait(float (&v)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]),
                   "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15])
                 :: "memory");
}
// two sums at once: the packed form has the same roundings and half the instructions
__device__ __forceinline__ void fma2(float& a0, float& a1, float x0, float x1, float s0, float s1) {
    asm("{ .reg .b64 a, x, s; mov.b64 a, {%0, %1}; mov.b64 x, {%2, %3}; mov.b64 s, {%4, %5}; fma.rn.f32x2 a, x, s, a; mov.b64 {%0, %1}, a; }"
        : "+f"(a0), "+f"(a1) : "f"(x0), "f"(x1), "f"(s0), "f"(s1));
}

// Shared-memory operand: rows of 128 bytes, 128-byte swizzle in groups of eight rows (1024 bytes apart)
__device__ __forceinline__ uint64_t operand_desc(unsigned addr) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

// The columns [c0, c0 + kCols) of a warp's 32 rows, from one row a lane to runs of consecutive columns.
template <typename OT, int COLS>
__device__ __forceinline__ void store_rows(const MatmulParams& p, OT* out, const float (&acc)[COLS], unsigned* words, int row0, int col0) {
    const int lane = lane_id();
    const int rows = min(32, p.rows_p - row0);
    constexpr int kPerWord = 4 / (int)sizeof(OT);
    constexpr int kWords = COLS / kPerWord < 32 ? COLS / kPerWord : 32;   // of a row, a round
    const bool pairs = kPerWord == 1 || ((reinterpret_cast<uintptr_t>(out) & 3u) == 0 && (p.ldo & 1) == 0);
#pragma unroll
    for (int c = 0; c < COLS; c += kWords * kPerWord) {
        if (col0 + c >= p.rows_q) break;
        __syncwarp();
#pragma unroll
        for (int w = 0; w < kWords; ++w)
            words[lane * 32 + (w ^ lane)] = kPerWord == 1 ? __float_as_uint(acc[c + w]) : pack_bf16(acc[c + w * kPerWord], acc[c + w * kPerWord + kPerWord - 1]);
        __syncwarp();
        if (pairs) {
            const int col = col0 + c + lane * kPerWord;
            for (int r = 0; r < rows; ++r) {
                const unsigned v = words[r * 32 + (lane ^ r)];
                OT* const at = out + (long long)(row0 + r) * p.ldo + col;
                if (lane < kWords && col + kPerWord <= p.rows_q) *reinterpret_cast<unsigned*>(at) = v;
                else if (lane < kWords && col < p.rows_q) *reinterpret_cast<unsigned short*>(at) = (unsigned short)v;
            }
        } else {
            for (int r = 0; r < rows; ++r)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int i = h * 32 + lane, col = col0 + c + i;
                    const unsigned v = words[r * 32 + (((i >> 1) & 31) ^ r)] >> ((i & 1) * 16);
                    if (i < kWords * kPerWord && col < p.rows_q)
                        *reinterpret_cast<unsigned short*>(out + (long long)(row0 + r) * p.ldo + col) = (unsigned short)v;
                }
        }
    }
}
// The result is [q, p]: a lane's row is its column there, neighbouring lanes write neighbouring elements.
template <typename OT, int COLS>
__device__ __forceinline__ void store_swapped(const MatmulParams& p, OT* out, const float (&acc)[COLS], int row, int col0) {
    if (row >= p.rows_p) return;
#pragma unroll
    for (int c = 0; c < COLS; ++c)
        if (col0 + c < p.rows_q) out[(long long)(col0 + c) * p.ldo + row] = from_float<OT>(acc[c]);
}

template <int CG, int NT, bool QVEC, typename OT>
__global__ void __launch_bounds__(TileShape<CG, NT>::kThreads, 1)
k_matmul_fp8(const __grid_constant__ CUtensorMap map_p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ MatmulParams p) {
    using S = TileShape<CG, NT>;
    extern __shared__ __align__(1024) unsigned char smem[];
    unsigned char* const header = smem + S::kStages * S::kStageBytes + S::kOutBytes;
    float* const scales = reinterpret_cast<float*>(header);                       // QVEC: [warps / 4][2][128]
    unsigned* const tmem_slot = reinterpret_cast<unsigned*>(header + 2048);
    const unsigned bars = smem_addr(header + 2064);
    const unsigned full = bars, empty = bars + 8 * S::kStages, tmem_full = empty + 8 * S::kStages, tmem_empty = tmem_full + 16;
    const int warp = warp_id(), lane = lane_id();
    const unsigned rank = CG == 2 ? (unsigned)(blockIdx.x & 1) : 0u;               // of the pair; 0 issues for both
    const int worker = blockIdx.x / CG, workers = gridDim.x / CG;
    pdl_trigger();

    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kStages; ++i) { bar_init(full + 8 * i, 1); bar_init(empty + 8 * i, 1); }
        for (int i = 0; i < 2; ++i) { bar_init(tmem_full + 8 * i, 1); bar_init(tmem_empty + 8 * i, CG * S::kEpiWarps); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        if (CG == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_slot)), "r"(S::kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_slot)), "r"(S::kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (CG == 2) asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const unsigned tmem = *tmem_slot;
    pdl_wait();

    const int tiles = p.tiles_p * p.tiles_q, items = tiles * p.splits;
    // an item's tile and part; the side with fewer tiles moves fastest, so that CTAs at work together share the other's rows
    auto item_of = [&](int item, int& tp, int& tq, int& k0, int& k1) {
        const int part = item / tiles, tile = item - part * tiles;
        if (p.tiles_p <= p.tiles_q) { tq = tile / p.tiles_p; tp = tile - tq * p.tiles_p; }
        else { tp = tile / p.tiles_q; tq = tile - tp * p.tiles_q; }
        k0 = (int)((long long)p.blocks * part / p.splits);
        k1 = (int)((long long)p.blocks * (part + 1) / p.splits);
        return part;
    };
    bool ok = true;

    if (warp == S::kEpiWarps) {                                                    // ---- copies ----
        if (lane == 0) {
            const unsigned stages = smem_addr(smem);
            int n = 0;
            for (int item = worker; item < items && ok; item += workers) {
                int tp, tq, k0, k1;
                item_of(item, tp, tq, k0, k1);
                for (int b = k0; b < k1; ++b, ++n) {
                    const int s = n % S::kStages;
                    ok = bar_wait(empty + 8 * s, ((n / S::kStages) & 1) ^ 1);
                    if (!ok) break;
                    const unsigned bar = CG == 2 ? in_cta(full + 8 * s, 0) : full + 8 * s;
                    if (rank == 0) bar_expect(full + 8 * s, CG * S::kStageBytes);
                    const unsigned at = stages + s * S::kStageBytes;
                    copy_tile<CG>(at, &map_p, b * kBlockK, (tp * CG + (int)rank) * kTileP, bar);
                    copy_tile<CG>(at + kTileP * kBlockK, &map_q, b * kBlockK, tq * NT + (int)rank * S::kQRows, bar);
                }
            }
            // the last arrivals at this CTA's barriers come before it ends
            for (int i = n > S::kStages ? n - S::kStages : 0; i < n && ok; ++i) ok = bar_wait(empty + 8 * (i % S::kStages), (i / S::kStages) & 1);
        }
    } else if (warp == S::kEpiWarps + 1) {                                         // ---- matrix instructions ----
        if (lane == 0 && rank == 0) {
            // fp32 results, both operands e4m3 with the inner dimension contiguous, N and M of the instruction
            constexpr unsigned idesc = 1u << 4 | (unsigned)(NT >> 3) << 17 | (unsigned)((kTileP * CG) >> 4) << 24;
            const unsigned stages = smem_addr(smem);
            int n = 0;
            for (int item = worker; item < items && ok; item += workers) {
                int tp, tq, k0, k1;
                item_of(item, tp, tq, k0, k1);
                for (int b = k0; b < k1; ++b, ++n) {
                    const int s = n % S::kStages, buf = n & 1;
                    ok = bar_wait(tmem_empty + 8 * buf, ((n >> 1) & 1) ^ 1) && bar_wait(full + 8 * s, (n / S::kStages) & 1);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t a = operand_desc(stages + s * S::kStageBytes), q = operand_desc(stages + s * S::kStageBytes + kTileP * kBlockK);
#pragma unroll
                    for (int k = 0; k < kBlockK / 32; ++k)                          // 32 bytes of the inner dimension each
                        mma_fp8<CG>(tmem + buf * NT, a + 2 * k, q + 2 * k, idesc, k > 0);
                    mma_commit<CG>(empty + 8 * s);
                    mma_commit<CG>(tmem_full + 8 * buf);
                }
            }
        }
    } else {                                                                       // ---- epilogue ----
        const int group = warp >> 2, quarter = warp & 3;                           // a warp reaches the 32 lanes of its quarter
        const unsigned mine = tmem + ((unsigned)(quarter * 32) << 16) + group * 128;
        unsigned* const words = reinterpret_cast<unsigned*>(smem + S::kStages * S::kStageBytes + warp * 4096);
        const unsigned free_bar = in_cta(tmem_empty, 0);
        int n = 0;
        for (int item = worker; item < items; item += workers) {
            int tp, tq, k0, k1;
            const int part = item_of(item, tp, tq, k0, k1);
            const int row0 = (tp * CG + (int)rank) * kTileP + quarter * 32, row = row0 + lane, col0 = tq * NT + group * 128;
            const float* sp = p.sp + (min(row, p.rows_p - 1) >> p.shift_p);
            const int my_col = QVEC ? min(col0 + (int)(threadIdx.x & 127), p.rows_q - 1) : min(col0, p.rows_q - 1);
            const float* sq = p.sq + (my_col >> p.shift_q);
            float next_p = sp[k0 * p.ld_sp], next_q = sq[k0 * p.ld_sq];
            float acc[S::kCols];
#pragma unroll
            for (int i = 0; i < S::kCols; ++i) acc[i] = 0.f;
            for (int b = k0; b < k1; ++b, ++n) {
                const int buf = n & 1;
                const float scale = QVEC ? next_p : next_p * next_q;
                float* const vec = scales + (group * 2 + buf) * 128;
                if (QVEC) {
                    vec[threadIdx.x & 127] = next_q;
                    asm volatile("bar.sync %0, 128;" ::"r"(group + 1) : "memory");
                }
                if (b + 1 < k1) { next_p = sp[(b + 1) * p.ld_sp]; next_q = sq[(b + 1) * p.ld_sq]; }
                if (ok) ok = bar_wait(tmem_full + 8 * buf, (n >> 1) & 1);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) continue;                                                 // (bar.sync above stays matched)
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                float v[2][16];
                tmem_load16(mine + buf * NT, v[0]);
#pragma unroll
                for (int c = 0; c < S::kCols; c += 16) {
                    float (&x)[16] = v[(c >> 4) & 1];
                    tmem_wait(x);
                    if (c + 16 < S::kCols) tmem_load16(mine + buf * NT + c + 16, v[((c >> 4) & 1) ^ 1]);
                    else {
                        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) bar_arrive_cluster(free_bar + 8 * buf);
                    }
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        if (QVEC) {
                            const float4 q = *reinterpret_cast<const float4*>(vec + c + i);
                            fma2(acc[c + i], acc[c + i + 1], x[i], x[i + 1], scale * q.x, scale * q.y);
                            fma2(acc[c + i + 2], acc[c + i + 3], x[i + 2], x[i + 3], scale * q.z, scale * q.w);
                        } else {
                            fma2(acc[c + i], acc[c + i + 1], x[i], x[i + 1], scale, scale);
                            fma2(acc[c + i + 2], acc[c + i + 3], x[i + 2], x[i + 3], scale, scale);
                        }
                    }
                }
            }
            if (!ok) {
#pragma unroll
                for (int i = 0; i < S::kCols; ++i) acc[i] = __uint_as_float(0x7FC00000u);
            }
            OT* const out = static_cast<OT*>(p.out) + part * p.split_stride;
            if (p.swap) store_swapped<OT, S::kCols>(p, out, acc, row, col0);
            else if (row0 < p.rows_p) store_rows<OT, S::kCols>(p, out, acc, words, row0, col0);
        }
    }
    if (!ok) {                                                                     // let copies and instructions in flight land
        const long long t0 = clock64();
        while (clock64() - t0 < (1LL << 24)) {}
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (CG == 2) asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == 0) {
        if (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kTmemCols) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kTmemCols) : "memory");
    }
}

// out = the parts' results added in their order
template <typename OT>
__global__ void __launch_bounds__(256) k_join_parts(const float* __restrict__ parts, long long stride, int splits, OT* out, long long ldo, long long rows, int cols) {
    pdl_trigger();
    pdl_wait();
    const long long total = rows * cols, step = (long long)gridDim.x * 256;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += step) {
        float v = 0.f;
        for (int s = 0; s < splits; ++s) v += __ldcs(parts + s * stride + i);
        const long long r = i / cols;
        out[r * ldo + (i - r * cols)] = from_float<OT>(v);
    }
}

// How a product is cut: which side is Q, its tile, and the parts of the inner dimension.
constexpr int kMaxParts = 32;
struct MatmulPlan { int cg, nt, swap; long long rows_p, rows_q, tiles_p, tiles_q, blocks; int splits; };
static MatmulPlan plan_matmul(long long M, long long N, long long K) {
    MatmulPlan L{};
    const long long small = M < N ? M : N;
    L.swap = small <= 128 && M < N;
    L.cg = small <= 128 ? 1 : 2;
    L.nt = small <= 16 ? 16 : small <= 32 ? 32 : small <= 64 ? 64 : small <= 128 ? 128 : 256;
    L.rows_p = L.swap ? N : M; L.rows_q = L.swap ? M : N;
    L.tiles_p = (L.rows_p + kTileP * L.cg - 1) / (kTileP * L.cg);
    L.tiles_q = (L.rows_q + L.nt - 1) / L.nt;
    L.blocks = (K + kBlockK - 1) / kBlockK;
    // Parts: the fewest microseconds by a model of 0.3 a block, 1 a tile, and for more than one part their results written
    // and read again at 4 TB/s and another launch.  SMs of a B200, not the device's, so that the order of the sums
    // follows from the sizes.
    const long long tiles = L.tiles_p * L.tiles_q, workers = kSmCount / L.cg;
    double best = 0;
    for (int s = 1; s <= kMaxParts && s <= L.blocks; ++s) {
        if (s > 1 && tiles * s > 2 * workers) break;
        const long long rounds = (tiles * s + workers - 1) / workers, len = (L.blocks + s - 1) / s;
        const double us = rounds * (len * 0.3 + 1.0) + (s > 1 ? 3.0 + double(s) * M * N * 8 / 4e6 : 0.0);
        if (s == 1 || us < best) { best = us; L.splits = s; }
    }
    return L;
}

size_t matmul_fp8_workspace(long long M, long long N, long long K) {
    const MatmulPlan L = plan_matmul(M, N, K);
    return L.splits > 1 ? size_t(L.splits) * size_t(M) * size_t(N) * 4 : 0;
}
// What no product up to these sizes exceeds: parts x tiles stay within two for each SM (or pair of them).
size_t matmul_fp8_workspace_bound(long long M, long long N, long long K) {
    const long long blocks = (K + kBlockK - 1) / kBlockK;
    if (blocks < 2) return 0;
    const size_t every = size_t(blocks < kMaxParts ? blocks : kMaxParts) * size_t(M) * size_t(N) * 4;
    const size_t pairs = size_t(kSmCount) * 256 * 256 * 4;
    return every < pairs ? every : pairs;
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static EncodeTiled encode_tiled() {
    static std::atomic<void*> known{nullptr};
    void* f = known.load();
    if (!f) {
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) return nullptr;
        known.store(f);
    }
    return reinterpret_cast<EncodeTiled>(f);
}
// Boxes of 128 bytes by `rows` rows, swizzled; outside the matrix (its inner end too) a copy reads zeros.
static bool operand_map(CUtensorMap& map, const Fp8View& m, int rows) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)m.cols, (cuuint64_t)m.rows}, strides[1] = {(cuuint64_t)m.ld};
    const cuuint32_t box[2] = {kBlockK, (cuuint32_t)rows}, step[2] = {1, 1};
    return encode(&map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, m.q, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int CG, int NT, bool QVEC, typename OT>
static cudaError_t matmul_launch(const CUtensorMap& mp, const CUtensorMap& mq, const MatmulParams& p, int sms, cudaStream_t stream) {
    using S = TileShape<CG, NT>;
    static SmemOptIn opt;
    const cudaError_t e = ensure_dynamic_smem(k_matmul_fp8<CG, NT, QVEC, OT>, S::kSmem, opt);
    if (e != cudaSuccess) return e;
    const long long items = (long long)p.tiles_p * p.tiles_q * p.splits, workers = sms / CG;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((items < workers ? items : workers) * CG)); cfg.blockDim = dim3(S::kThreads);
    cfg.dynamicSmemBytes = S::kSmem; cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CG; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, k_matmul_fp8<CG, NT, QVEC, OT>, mp, mq, p);
}
template <int CG, int NT>
static cudaError_t matmul_nt(const CUtensorMap& mp, const CUtensorMap& mq, const MatmulParams& p, int out_type, int sms, cudaStream_t stream) {
    if (p.shift_q == 0)
        return out_type == DST_F32 ? matmul_launch<CG, NT, true, float>(mp, mq, p, sms, stream) : matmul_launch<CG, NT, true, __nv_bfloat16>(mp, mq, p, sms, stream);
    return out_type == DST_F32 ? matmul_launch<CG, NT, false, float>(mp, mq, p, sms, stream) : matmul_launch<CG, NT, false, __nv_bfloat16>(mp, mq, p, sms, stream);
}

cudaError_t launch_matmul_fp8(const Fp8View& a, const Fp8View& b, void* out, long long ldo, int out_type, void* workspace, int sms, cudaStream_t stream) {
    const MatmulPlan L = plan_matmul(a.rows, b.rows, a.cols);
    const Fp8View &vp = L.swap ? b : a, &vq = L.swap ? a : b;
    CUtensorMap mp, mq;
    if (!operand_map(mp, vp, kTileP) || !operand_map(mq, vq, L.nt / L.cg)) return cudaErrorInvalidValue;
    MatmulParams p{vp.scale, vq.scale, vp.ld_scale, vq.ld_scale, vp.shift, vq.shift, (int)vp.rows, (int)vq.rows, (int)L.blocks, L.splits,
                   (int)L.tiles_p, (int)L.tiles_q, L.swap, out, ldo, 0};
    int type = out_type;
    if (L.splits > 1) { p.out = workspace; p.ldo = b.rows; p.split_stride = a.rows * b.rows; type = DST_F32; }
    cudaError_t e;
    switch (L.nt) {
        case 16: e = matmul_nt<1, 16>(mp, mq, p, type, sms, stream); break;
        case 32: e = matmul_nt<1, 32>(mp, mq, p, type, sms, stream); break;
        case 64: e = matmul_nt<1, 64>(mp, mq, p, type, sms, stream); break;
        case 128: e = matmul_nt<1, 128>(mp, mq, p, type, sms, stream); break;
        default: e = matmul_nt<2, 256>(mp, mq, p, type, sms, stream); break;
    }
    if (e != cudaSuccess || L.splits == 1) return e;
    const long long total = a.rows * b.rows, blocks = (total + 255) / 256, cap = (long long)sms * 8;
    const dim3 grid((unsigned)(blocks < cap ? blocks : cap));
    const float* parts = static_cast<const float*>(workspace);
    if (out_type == DST_F32) return launch_pdl(k_join_parts<float>, grid, dim3(256), 0, stream, parts, p.split_stride, L.splits, static_cast<float*>(out), ldo, (long long)a.rows, (int)b.rows);
    return launch_pdl(k_join_parts<__nv_bfloat16>, grid, dim3(256), 0, stream, parts, p.split_stride, L.splits, static_cast<__nv_bfloat16*>(out), ldo, (long long)a.rows, (int)b.rows);
}

}  // namespace dst
