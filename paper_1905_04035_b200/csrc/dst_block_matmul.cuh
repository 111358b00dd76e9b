// The product of two matrices in 8 or 4 bits with power-of-two scales: one kernel for both kinds of element.
#pragma once

#include <cuda.h>

#include <type_traits>

#include "dst_async.cuh"
#include "dst_fp4.cuh"
#include "dst_fp8.cuh"

namespace dst {

// D[p, q] = sum over blocks b of sp[b, p] sq[b, q] (P_b Q_b^T).  The scales are powers of two in the form the tensor
// cores multiply by themselves (one scale for 32 elements of the inner dimension; in 8 bits the four instructions of a block of
// 128 use the same byte), so whole stretches of the inner dimension are summed in tensor memory and the epilogue sees finished
// tiles.  P is the operand whose rows are the 128 lanes of tensor memory, Q the one whose rows are its columns.  The inner
// dimension goes by steps of 128 bytes of a row, whatever the elements' size.
//
// Both sides large: two CTAs share a 256 x 256 tile (each holds 128 rows of P, half of Q's rows, and 128 x 256 of
// the result), which halves what an SM has to fetch for a block against a tile of its own: 32 KB where the tensor
// cores take 512 cycles.  One side of at most 128 rows: that side is Q, padded to 16, 32, 64 or 128 rows, and a CTA has
// 128 rows of the other one; the time is that side's bytes.
//
// Measured, 8 bits: 8192 x 33,708 x 1024 to bf16 238 to 250 us (2380 to 2260 TFLOP/s; stores and the drain of a tile's sums between its
// eight blocks and the next tile's), 8192^3 392 to 407 us, 33,708 x 1024 x 8111 to fp32 280 to 290 us (the last of 7.1 rounds of
// tiles, and sums moved to registers); one row by 33,708 x 1024 7.5 us, where the weight's 34.5 MB need 5.3.
// 4 bits: 8192^3 182 us (6040 TFLOP/s), 4096 x 33,708 x 1024 to bf16 79 us (52 without its stores, which alone would take 39: both go
// through shared memory), to fp32 133 us; one row by 33,708 x 1024 4.9 us, where 18.3 MB need 2.8.
//
// Warps of a CTA: the epilogue warps (4, or 8 where a warp would otherwise hold more than 128 columns), one that issues
// the copies and one that issues the matrix instructions.  Every wait has a limit; a CTA in which one ran out leaves
// NaN in what it still had to write.
constexpr int kBlockK = 128;                              // bytes of a row that a step of the inner dimension takes
// Elements of a step; steps that one load of scales serves, and the tiles of 512 bytes that it brings for 128 rows; steps summed
// in tensor memory before an fp32 result moves to registers; bytes for rows that are quantised on the way.
struct Fp8Kind { static constexpr int kStepCols = 128, kScaleSteps = 4, kScaleTiles = 1, kChunk = 6, kResident = 32768; };
struct Fp4Kind { static constexpr int kStepCols = 256, kScaleSteps = 1, kScaleTiles = 2, kChunk = 4, kResident = 16384; };
constexpr int kTileP = 128;                               // rows of P a CTA
constexpr int kSmemMost = 232448;

// FUSED: Q is quantised by the CTA itself from the rows of x, kept whole in shared memory (kResident bytes) and used for
// every tile; its result leaves swapped.
template <typename KIND, int CG, int NT, bool FUSED = false>
struct TileShape {
    static constexpr int kQRows = NT / CG;                // rows of Q a CTA holds
    static constexpr int kEpiWarps = NT > 128 ? 8 : 4;
    static constexpr int kCols = NT > 128 ? 128 : NT;     // columns of the result an epilogue warp holds
    static constexpr int kThreads = (kEpiWarps + 2) * 32;
    static constexpr int kStageBytes = (kTileP + (FUSED ? 0 : kQRows)) * kBlockK;
    static constexpr int kQScaleTiles = (NT + 127) / 128;
    static constexpr int kScaleBytes = (1 + (FUSED ? 0 : kQScaleTiles)) * KIND::kScaleTiles * kScaleTile;   // of one load
    static constexpr int kResident = FUSED ? KIND::kResident : 0;
    static constexpr int kResidentScales = FUSED ? kResident / NT / kBlockK / KIND::kScaleSteps * KIND::kScaleTiles * kScaleTile : 0;
    // bytes of shared memory a lane stages its row in: 256 at most, and room to start anywhere in 16
    static constexpr int kOutPitch = (kCols < 64 ? kCols * 4 : 256) + 16, kOutBytes = FUSED ? 0 : kEpiWarps * 32 * kOutPitch;
    static constexpr int kHeaderBytes = 1024;
    // small tiles wait for memory, not for each other: two CTAs share an SM
    static constexpr int kCtas = NT <= 64 ? 2 : 1;
    static constexpr int kFit = (kSmemMost / kCtas - (kCtas - 1) * 1024 - kOutBytes - kResident - kResidentScales - kHeaderBytes) / (kStageBytes + kScaleBytes);
    static constexpr int kStages = kFit < 8 ? kFit : 8;
    static constexpr int kSmem = kStages * (kStageBytes + kScaleBytes) + kResident + kResidentScales + kOutBytes + kHeaderBytes;
    // tensor memory: one or two results, then a ring of scales (P's tiles, four columns each, then Q's; four loads)
    static constexpr int kBufs = NT > 128 ? 1 : 2;
    static constexpr int kScaleCols = 4 * KIND::kScaleTiles * (1 + kQScaleTiles), kScaleRing = 4;
    static constexpr int kUsedCols = kBufs * NT + kScaleRing * kScaleCols;
    static constexpr int kTmemCols = kUsedCols <= 64 ? 64 : kUsedCols <= 128 ? 128 : kUsedCols <= 256 ? 256 : 512;
};

struct MatmulParams {
    int rows_p, rows_q;
    int blocks, splits;                                   // steps of the inner dimension, parts it is cut into
    int tiles_p, tiles_q;
    int swap;                                             // the result is [q, p]
    void* out;
    long long ldo;
    long long split_stride;                               // elements between the parts' results (splits > 1)
    const void* x;                                        // FUSED: Q before its quantisation
    long long ldx;
    long long cols;
    int x_type, x_vec;                                    // rows aligned to four elements
};

// (what is handed over here is tensor memory, ordered by the tcgen05 fences around it; a release at cluster scope would
// wait for all of the thread's memory traffic)
__device__ __forceinline__ void bar_arrive_cluster(unsigned bar) { asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory"); }
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
__device__ __forceinline__ void copy_scales(unsigned dst, const CUtensorMap* map, int group, int tile, unsigned bar) {
    if (CG == 2)
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(0), "r"(group), "r"(tile), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(0), "r"(group), "r"(tile), "r"(bar) : "memory");
}
// 32 rows of 16 bytes from shared memory to four columns of tensor memory, the same in all four quarters of its lanes
template <int CG>
__device__ __forceinline__ void tmem_copy_scales(unsigned d, uint64_t desc) {
    if (CG == 2) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(d), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(d), "l"(desc) : "memory");
}
#define DST_MMA(GROUP, KIND)                                                                                                                            \
    asm volatile("{ .reg .pred p; setp.ne.b32 p, %6, 0; tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], %1, %2, %3, [%4], [%5], p; }" ::"r"(d), \
                 "l"(a), "l"(b), "r"(idesc), "r"(scale_a), "r"(scale_b), "r"(accumulate) : "memory")
template <typename KIND, int CG>
__device__ __forceinline__ void mma_scaled(unsigned d, uint64_t a, uint64_t b, unsigned idesc, unsigned scale_a, unsigned scale_b, unsigned accumulate) {
    constexpr bool k4 = std::is_same<KIND, Fp4Kind>::value;   // 64 elements with two scales a row; else 32 with one
    if (k4 && CG == 2) DST_MMA("2", "mxf4.block_scale.scale_vec::2X");
    else if (k4) DST_MMA("1", "mxf4.block_scale.scale_vec::2X");
    else if (CG == 2) DST_MMA("2", "mxf8f6f4.block_scale.scale_vec::1X");
    else DST_MMA("1", "mxf8f6f4.block_scale.scale_vec::1X");
}
#undef DST_MMA
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
// Shared-memory operand: rows of 128 bytes, 128-byte swizzle in groups of eight rows (1024 bytes apart)
__device__ __forceinline__ uint64_t operand_desc(unsigned addr) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// scales: 32 rows of 16 bytes, one after another
__device__ __forceinline__ uint64_t scale_desc(unsigned addr) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
}

// A lane's row of the tile, 256 bytes a round: into a row of shared memory that is the lane's own, at the place within 16
// bytes that it has in the output, and from there by one asynchronous bulk copy of the 16-byte pieces that lie wholly in
// the row; what is left at either end is stored plainly.  No lane waits for another one, nor for the copies until it needs its
// row of shared memory again.  (Runs of 128 bytes through registers instead: 344 us for 8192 x 33708 x 1024, whose
// rows are 8-byte aligned.)  ALIGN: bytes that rows of the output are aligned to.
template <typename OT, int COLS, int ALIGN>
__device__ __forceinline__ void store_row_aligned(const MatmulParams& p, OT* out, const float (&acc)[COLS], unsigned char* buffer, int row, int col0) {
    constexpr int kSize = (int)sizeof(OT), kRound = COLS * kSize < 256 ? COLS : 256 / kSize, kWords = kRound * kSize / 4;
    if (row >= p.rows_p) return;
#pragma unroll
    for (int c = 0; c < COLS; c += kRound) {
        if (col0 + c >= p.rows_q) break;
        unsigned char* const at = reinterpret_cast<unsigned char*>(out + (long long)row * p.ldo + col0 + c);
        const int shift = (int)(reinterpret_cast<uintptr_t>(at) & 15u), total = min(kRound, p.rows_q - col0 - c) * kSize;
        asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        unsigned v[kWords];
#pragma unroll
        for (int w = 0; w < kWords; ++w)
            v[w] = kSize == 4 ? __float_as_uint(acc[c + w]) : pack_bf16(acc[c + w * 4 / kSize], acc[c + w * 4 / kSize + 4 / kSize - 1]);
        unsigned char* const base = buffer + (ALIGN >= 4 ? shift : shift & ~3);
        if (ALIGN == 16) {
#pragma unroll
            for (int w = 0; w < kWords; w += 4) *reinterpret_cast<uint4*>(base + w * 4) = make_uint4(v[w], v[w + 1], v[w + 2], v[w + 3]);
        } else if (ALIGN == 8) {
#pragma unroll
            for (int w = 0; w < kWords; w += 2) *reinterpret_cast<uint2*>(base + w * 4) = make_uint2(v[w], v[w + 1]);
        } else if (ALIGN == 4) {
#pragma unroll
            for (int w = 0; w < kWords; ++w) *reinterpret_cast<unsigned*>(base + w * 4) = v[w];
        } else {                                             // half a word further where the row starts in the middle of one
            const unsigned pick = shift & 2 ? 0x5432u : 0x7654u;
#pragma unroll
            for (int w = 0; w <= kWords; ++w)
                *reinterpret_cast<unsigned*>(base + w * 4) = __byte_perm(w > 0 ? v[w - 1] : 0u, w < kWords ? v[w] : 0u, pick);
        }
        const int head = min((16 - shift) & 15, total), body = (total - head) & ~15;
        if (body > 0) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;\n\tcp.async.bulk.commit_group;"
                         ::"l"(at + head), "r"(smem_addr(buffer + shift + head)), "r"(body) : "memory");
        }
        auto plain = [&](int from, int n) {
            const unsigned char* const src = buffer + shift;
            if (ALIGN >= 8)
                for (; n >= 8; from += 8, n -= 8) *reinterpret_cast<uint2*>(at + from) = *reinterpret_cast<const uint2*>(src + from);
            for (; n > 0; from += kSize, n -= kSize) *reinterpret_cast<OT*>(at + from) = *reinterpret_cast<const OT*>(src + from);
        };
        if (ALIGN < 16) plain(0, head);
        plain(head + body, total - head - body);
    }
}
template <typename OT, int COLS>
__device__ __forceinline__ void store_row(const MatmulParams& p, OT* out, const float (&acc)[COLS], unsigned char* buffer, int row, int col0) {
    const unsigned at = (unsigned)reinterpret_cast<uintptr_t>(out) | (unsigned)(p.ldo * sizeof(OT));
    if ((at & 15) == 0) store_row_aligned<OT, COLS, 16>(p, out, acc, buffer, row, col0);
    else if ((at & 7) == 0) store_row_aligned<OT, COLS, 8>(p, out, acc, buffer, row, col0);
    else if (sizeof(OT) == 4 || (at & 3) == 0) store_row_aligned<OT, COLS, 4>(p, out, acc, buffer, row, col0);
    else store_row_aligned<OT, COLS, 2>(p, out, acc, buffer, row, col0);
}
// A row of 256 columns in 16 bits by the two warps that hold its halves: 512 bytes are one copy, and half as many copies are what the
// unit that makes them is busy with (4096 x 33,708 x 512 in 4 bits: 67 us against 82).  Each of the warps issues every other row's copy.
// Rows are aligned to four bytes at least, so that no word has elements of both; `buffer` is the row's place in shared memory.
template <int ALIGN>
__device__ __forceinline__ void store_row_halves(const MatmulParams& p, __nv_bfloat16* out, const float (&acc)[128], unsigned char* buffer, int row, int col0, int half, int pair) {
    const bool issues = (lane_id() & 1) == half;
    if (issues) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    asm volatile("bar.sync %0, 64;" ::"r"(pair) : "memory");
    unsigned char* const at = reinterpret_cast<unsigned char*>(out + (long long)row * p.ldo + col0);
    const int shift = (int)(reinterpret_cast<uintptr_t>(at) & 15u), total = min(256, p.rows_q - col0) * 2;
    unsigned char* const base = buffer + half * 256;
    unsigned v[64];
#pragma unroll
    for (int w = 0; w < 64; ++w) v[w] = pack_bf16(acc[2 * w], acc[2 * w + 1]);
#pragma unroll
    for (int w = 0; w < 64; w += ALIGN / 4) {
        if (ALIGN == 16) *reinterpret_cast<uint4*>(base + w * 4) = make_uint4(v[w], v[w + 1], v[w + 2], v[w + 3]);
        else if (ALIGN == 8) *reinterpret_cast<uint2*>(base + w * 4) = make_uint2(v[w], v[w + 1]);
        else *reinterpret_cast<unsigned*>(base + w * 4) = v[w];
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    asm volatile("bar.sync %0, 64;" ::"r"(pair) : "memory");
    if (!issues || row >= p.rows_p) return;
    const int head = min((16 - shift) & 15, total), body = (total - head) & ~15;
    if (body > 0)
        asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;\n\tcp.async.bulk.commit_group;"
                     ::"l"(at + head), "r"(smem_addr(buffer + head)), "r"(body) : "memory");
    auto plain = [&](int from, int n) {
        const unsigned char* const src = buffer;
        for (; n >= 4; from += 4, n -= 4) *reinterpret_cast<unsigned*>(at + from) = *reinterpret_cast<const unsigned*>(src + from);
        if (n > 0) *reinterpret_cast<unsigned short*>(at + from) = *reinterpret_cast<const unsigned short*>(src + from);
    };
    if (ALIGN < 16) plain(0, head);
    plain(head + body, total - head - body);
}
// The result is [q, p]: a lane's row is its column there, neighbouring lanes write neighbouring elements.
template <typename OT, int COLS>
__device__ __forceinline__ void store_swapped(const MatmulParams& p, OT* out, const float (&acc)[COLS], int row, int col0) {
    if (row >= p.rows_p) return;
#pragma unroll
    for (int c = 0; c < COLS; ++c)
        if (col0 + c < p.rows_q) out[(long long)(col0 + c) * p.ldo + row] = from_float<OT>(acc[c]);
}
// The same with many columns: the four warps put a tile into shared memory transposed, a row of it for each of the COLS columns that they hold, and
// each row leaves as one copy.  Rows lie there as they do in the output, within 16 bytes: by a distance that has the output's remainder.
// (As above, against this: 48 x 33,708 x 1024 10.1 and 9.7 us, in 4 bits x 512 5.9 and 5.2; 8 and 20 columns 3.7 and 4.0, 6.4 and 6.7.)
template <typename OT, int COLS>
__device__ __forceinline__ void store_transposed(const MatmulParams& p, OT* out, const float (&acc)[COLS], unsigned char* buffer, int tile0, int row, int col0) {
    static_assert(COLS <= 128, "a thread for each row");
    constexpr int kSize = (int)sizeof(OT);
    const int over = (int)(p.ldo * kSize) & 15, pitch = 128 * kSize + (over ? over : 16);
    unsigned char* const first = reinterpret_cast<unsigned char*>(out + (long long)col0 * p.ldo + tile0);
    unsigned char* const base = buffer + (reinterpret_cast<uintptr_t>(first) & 15u);
    asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    asm volatile("bar.sync 1, 128;" ::: "memory");
#pragma unroll
    for (int c = 0; c < COLS; ++c) *reinterpret_cast<OT*>(base + c * pitch + (row - tile0) * kSize) = from_float<OT>(acc[c]);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    asm volatile("bar.sync 1, 128;" ::: "memory");
    const int c = threadIdx.x;
    if (c >= COLS || col0 + c >= p.rows_q) return;
    unsigned char* const at = first + (long long)c * p.ldo * kSize;
    const unsigned char* const src = base + c * pitch;
    const int total = min(128, p.rows_p - tile0) * kSize, head = min((int)(16 - (reinterpret_cast<uintptr_t>(at) & 15u)) & 15, total), body = (total - head) & ~15;
    if (body > 0)
        asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;\n\tcp.async.bulk.commit_group;"
                     ::"l"(at + head), "r"(smem_addr(src + head)), "r"(body) : "memory");
    for (int i = 0; i < head; i += kSize) *reinterpret_cast<OT*>(at + i) = *reinterpret_cast<const OT*>(src + i);
    for (int i = head + body; i < total; i += kSize) *reinterpret_cast<OT*>(at + i) = *reinterpret_cast<const OT*>(src + i);
}

// x's rows as ROW blocks straight into the shared-memory form of an operand: the swizzle exchanges the 16-byte pieces of a
// 128-byte row by the row's number.  A unit is a block of a row and belongs to a warp, eight at a time.
template <typename KIND, typename T, int NT>
__device__ __forceinline__ void quantize_resident(const MatmulParams& p, long long cols, unsigned char* q, unsigned char* scales, int warps) {
    constexpr int kUnits = KIND::kStepCols / 128;            // of a step; in 4 bits a unit is four blocks, eight lanes each
    const int lane = lane_id(), units = p.rows_q * p.blocks * kUnits;
    using Raw = decltype(Four<T>::v);
    for (int u0 = warp_id(); u0 < units; u0 += 8 * warps) {
        Four<T> v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int unit = u0 + j * warps, row = unit % p.rows_q, block = unit / p.rows_q;
            const long long c = (long long)block * 128 + lane * 4;
            const T* const x = static_cast<const T*>(p.x) + row * p.ldx + c;
            v[j].clear();
            if (unit < units) {
                if (p.x_vec && c + 4 <= cols) v[j].v = *reinterpret_cast<const Raw*>(x);
                else
#pragma unroll
                    for (int i = 0; i < 4; ++i) if (c + i < cols) v[j].set(i, x[i]);
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int unit = u0 + j * warps, row = unit % p.rows_q, block = unit / p.rows_q;
            if (unit >= units) break;
            if constexpr (std::is_same<KIND, Fp4Kind>::value) {
                unsigned top = v[j].amax();
#pragma unroll
                for (int d = 1; d < 8; d *= 2) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
                const float u = block_inverse4(top);
                const int at = (block & 1) * 64 + lane * 2;  // byte of the step's 128
                *reinterpret_cast<unsigned short*>(q + (block >> 1) * (NT * kBlockK) + row * kBlockK + (((at >> 4) ^ (row & 7)) << 4) + (at & 15)) =
                    (unsigned short)to_e2m1x4(v[j].get(0) * u, v[j].get(1) * u, v[j].get(2) * u, v[j].get(3) * u);
                if ((lane & 7) == 0) scales[block * kScaleTile + (row & 31) * 16 + (row >> 5) * 4 + (lane >> 3)] = (uint8_t)block_exponent4(top);
                continue;
            }
            const unsigned top = __reduce_max_sync(0xFFFFFFFFu, v[j].amax());
            const float u = block_inverse(top);
            *reinterpret_cast<unsigned*>(q + block * (NT * kBlockK) + row * kBlockK + (((lane >> 2) ^ (row & 7)) << 4) + (lane & 3) * 4) =
                to_e4m3x4(v[j].get(0) * u, v[j].get(1) * u, v[j].get(2) * u, v[j].get(3) * u);
            if (lane == 0) scales[(block >> 2) * kScaleTile + (row & 31) * 16 + (row >> 5) * 4 + (block & 3)] = (uint8_t)block_exponent(top);
        }
    }
}

template <typename KIND, int CG, int NT, bool FUSED, typename OT>
__global__ void __launch_bounds__(TileShape<KIND, CG, NT, FUSED>::kThreads, TileShape<KIND, CG, NT, FUSED>::kCtas)
k_block_matmul(const __grid_constant__ CUtensorMap map_p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_sp,
             const __grid_constant__ CUtensorMap map_sq, const __grid_constant__ MatmulParams p) {
    using S = TileShape<KIND, CG, NT, FUSED>;
    constexpr int kSteps = KIND::kScaleSteps, kTiles = KIND::kScaleTiles;
    // Blocks summed in tensor memory before that sum is added to the one in registers.  Additions there do not round to
    // nearest: where one block outweighs the ones after it, each of them takes up to a unit off.  On the gradients of 8111
    // tokens by 33,708 words (fp32 dx and dweight, K 33,708 and 8111) the errors are 3.3e-5 and 4.8e-6 with no limit, 1.9e-6
    // and 1.2e-6 with 16 blocks, 9e-7 and 6e-7 with 8, 7e-7 and 4.5e-7 with 6, 4.8e-7 and 3.2e-7 with 4 (products in fp32:
    // 3.8e-6 and 1.2e-6), for 520, 542, 556, 561 and 593 us together.  A bf16 result has 2e-3 from its own rounding, and
    // no limit.
    constexpr bool kChunked = sizeof(OT) == 4;
    constexpr int kChunk = KIND::kChunk;
    extern __shared__ __align__(1024) unsigned char smem[];
    unsigned char* const resident = smem + S::kStages * S::kStageBytes;              // FUSED: Q, a block after the other
    unsigned char* const scale_ring = resident + S::kResident;
    unsigned char* const resident_scales = scale_ring + S::kStages * S::kScaleBytes;
    unsigned char* const out_rows = resident_scales + S::kResidentScales;
    unsigned char* const header = out_rows + S::kOutBytes;
    unsigned* const tmem_slot = reinterpret_cast<unsigned*>(header);
    const unsigned bars = smem_addr(header + 16);
    const unsigned full = bars, empty = bars + 8 * S::kStages, tmem_full = empty + 8 * S::kStages, tmem_empty = tmem_full + 8 * S::kBufs, q_ready = tmem_empty + 8 * S::kBufs;
    const int warp = warp_id(), lane = lane_id();
    const unsigned rank = CG == 2 ? (unsigned)(blockIdx.x & 1) : 0u;               // of the pair; 0 issues for both
    const int worker = blockIdx.x / CG, workers = gridDim.x / CG;
    pdl_trigger();

    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kStages; ++i) { bar_init(full + 8 * i, 1); bar_init(empty + 8 * i, 1); }
        for (int i = 0; i < S::kBufs; ++i) { bar_init(tmem_full + 8 * i, 1); bar_init(tmem_empty + 8 * i, CG * S::kEpiWarps); }
        if (FUSED) bar_init(q_ready, S::kEpiWarps);
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

    const int tiles = p.tiles_p * p.tiles_q, items = tiles * p.splits, groups = (p.blocks + kSteps - 1) / kSteps;
    // an item's tile and part (whole loads of scales); the side with fewer tiles moves fastest, so that CTAs at work
    // together share the other's rows
    auto item_of = [&](int item, int& tp, int& tq, int& k0, int& k1) {
        const int part = item / tiles, tile = item - part * tiles;
        if (p.tiles_p <= p.tiles_q) { tq = tile / p.tiles_p; tp = tile - tq * p.tiles_p; }
        else { tp = tile / p.tiles_q; tq = tile - tp * p.tiles_q; }
        k0 = (int)((long long)groups * part / p.splits) * kSteps;
        k1 = min((int)((long long)groups * (part + 1) / p.splits) * kSteps, p.blocks);
        return part;
    };
    bool ok = true;

    if (warp == S::kEpiWarps) {                                                    // ---- copies ----
        if (elect_one()) {
            const unsigned stages = smem_addr(smem), ring = smem_addr(scale_ring);
            const unsigned first_full = CG == 2 ? in_cta(full, 0) : full;          // the issuing CTA waits for both CTAs' copies
            int s = 0, used = 0;
            unsigned phase = 1;                                                    // every stage is free at first
            for (int item = worker; item < items && ok; item += workers) {
                int tp, tq, k0, k1;
                item_of(item, tp, tq, k0, k1);
                for (int b = k0; b < k1; ++b) {
                    ok = bar_wait(empty + 8 * s, phase);
                    if (!ok) break;
                    const unsigned bar = first_full + 8 * s;
                    const bool scales = b % kSteps == 0;
                    if (rank == 0) bar_expect(full + 8 * s, CG * (S::kStageBytes + (scales ? S::kScaleBytes : 0)));
                    const unsigned at = stages + s * S::kStageBytes, sc = ring + s * S::kScaleBytes;
                    copy_tile<CG>(at, &map_p, b * kBlockK, (tp * CG + (int)rank) * kTileP, bar);
                    if (!FUSED) copy_tile<CG>(at + kTileP * kBlockK, &map_q, b * kBlockK, tq * NT + (int)rank * S::kQRows, bar);
                    if (scales) {                                                  // all of Q's for both CTAs: each has every column
                        const int group = b / kSteps * kTiles;
#pragma unroll
                        for (int h = 0; h < kTiles; ++h) {                         // (past the matrix a copy brings zeros)
                            copy_scales<CG>(sc + h * kScaleTile, &map_sp, group + h, tp * CG + (int)rank, bar);
                            if (!FUSED)
                                for (int i = 0; i < S::kQScaleTiles; ++i) copy_scales<CG>(sc + (kTiles + h * S::kQScaleTiles + i) * kScaleTile, &map_sq, group + h, tq * S::kQScaleTiles + i, bar);
                        }
                    }
                    used = min(used + 1, S::kStages);
                    if (++s == S::kStages) { s = 0; phase ^= 1; }
                }
            }
            // the last arrivals at this CTA's barriers come before it ends: each stage in use becomes free once more
            for (int i = 0; i < used && ok; ++i) {
                ok = bar_wait(empty + 8 * (used < S::kStages ? i : s), used < S::kStages ? 0u : phase);
                if (used == S::kStages && ++s == S::kStages) { s = 0; phase ^= 1; }
            }
        }
    } else if (warp == S::kEpiWarps + 1) {                                         // ---- matrix instructions ----
        if (elect_one() && rank == 0) {
            // both operands e4m3 (0) or e2m1 (1) with the inner dimension contiguous, N and M of the instruction, scales as exponents
            constexpr unsigned kElement = std::is_same<KIND, Fp4Kind>::value ? 1u << 7 | 1u << 10 : 0u;
            constexpr unsigned idesc = kElement | (unsigned)(NT >> 3) << 17 | 1u << 23 | (unsigned)((kTileP * CG) >> 4) << 24;
            // The instruction queue is shallow: whatever this thread does between two blocks beyond two instructions' time
            // leaves the tensor cores idle, so the loop counts and never divides.
            const uint64_t operands = operand_desc(smem_addr(smem)), scales = scale_desc(smem_addr(scale_ring));
            const uint64_t own = operand_desc(smem_addr(resident)), own_scales = scale_desc(smem_addr(resident_scales));
            if (FUSED) ok = bar_wait(q_ready, 0);
            int s = 0, buf = 0, slot = 0;
            unsigned phase = 0, buf_phase = 1;
            for (int item = worker; item < items && ok; item += workers) {
                int tp, tq, k0, k1;
                item_of(item, tp, tq, k0, k1);
                unsigned sc = 0;
                for (int start = k0; start < k1 && ok; start += kChunk) {
                    ok = bar_wait(tmem_empty + 8 * buf, buf_phase);
                    const unsigned d = tmem + buf * NT;
                    const int end = kChunked ? min(start + kChunk, k1) : k1;
                    for (int b = start; b < end && ok; ++b) {
                        ok = bar_wait(full + 8 * s, phase);
                        if (!ok) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        if (b % kSteps == 0) {
                            sc = tmem + S::kBufs * NT + slot * S::kScaleCols;
                            slot = (slot + 1) & (S::kScaleRing - 1);
#pragma unroll
                            for (int i = 0; i < kTiles * (1 + S::kQScaleTiles); ++i)
                                tmem_copy_scales<CG>(sc + 4 * i, FUSED && i >= kTiles ? own_scales + (((b / kSteps * kTiles + i - kTiles) * kScaleTile) >> 4)
                                                                                     : scales + ((s * S::kScaleBytes + i * kScaleTile) >> 4));
                        }
                        const uint64_t a = operands + ((s * S::kStageBytes) >> 4), q = FUSED ? own + ((b * NT * kBlockK) >> 4) : a + ((kTileP * kBlockK) >> 4);
#pragma unroll
                        for (int k = 0; k < kBlockK / 32; ++k) {                    // 32 bytes of the inner dimension each
                            // the tile of scales, and which of its four bytes: of the step's place in the tile, or of the instruction's in the step
                            const unsigned h = k * kTiles / 4, byte = kTiles > 1 ? (unsigned)(k & 1) * 2 : (unsigned)(b & 3);
                            const unsigned id = idesc | byte << 4 | byte << 29;
                            mma_scaled<KIND, CG>(d, a + 2 * k, q + 2 * k, id, sc + 4 * h, sc + 4 * (kTiles + h * S::kQScaleTiles), b > start || k > 0);
                        }
                        mma_commit<CG>(empty + 8 * s);
                        if (++s == S::kStages) { s = 0; phase ^= 1; }
                    }
                    if (ok) mma_commit<CG>(tmem_full + 8 * buf);
                    if (++buf == S::kBufs) { buf = 0; buf_phase ^= 1; }
                    if (!kChunked) break;
                }
            }
        }
    } else {                                                                       // ---- epilogue ----
        const int group = warp >> 2, quarter = warp & 3;                           // a warp reaches the 32 lanes of its quarter
        const unsigned mine = tmem + ((unsigned)(quarter * 32) << 16) + group * 128;
        unsigned char* const buffer = out_rows + threadIdx.x * S::kOutPitch;
        const unsigned free_bar = in_cta(tmem_empty, 0);
        if (FUSED) {
            if (p.x_type == DST_F32) quantize_resident<KIND, float, NT>(p, p.cols, resident, resident_scales, S::kEpiWarps);
            else quantize_resident<KIND, __nv_bfloat16, NT>(p, p.cols, resident, resident_scales, S::kEpiWarps);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");           // the tensor cores read it
            __syncwarp();
            if (lane == 0) bar_arrive_cluster(in_cta(q_ready, 0));
        }
        int buf = 0;
        unsigned buf_phase = 0;
        for (int item = worker; item < items; item += workers) {
            int tp, tq, k0, k1;
            const int part = item_of(item, tp, tq, k0, k1);
            const int row0 = (tp * CG + (int)rank) * kTileP + quarter * 32, col0 = tq * NT + group * 128;
            float acc[S::kCols];
            auto sums_ready = [&] {
                if (ok) ok = bar_wait(tmem_full + 8 * buf, buf_phase);
                ok = __all_sync(0xFFFFFFFFu, ok);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                return ok;
            };
            auto sums_taken = [&] {                                                // the next ones may start
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) bar_arrive_cluster(free_bar + 8 * buf);
                if (++buf == S::kBufs) { buf = 0; buf_phase ^= 1; }
            };
            if (sums_ready()) {
#pragma unroll
                for (int c = 0; c < S::kCols; c += 16) tmem_load16(mine + buf * NT + c, *reinterpret_cast<float (*)[16]>(acc + c));
#pragma unroll
                for (int c = 0; c < S::kCols; c += 16) tmem_wait(*reinterpret_cast<float (*)[16]>(acc + c));
                sums_taken();
            }
#pragma unroll 1
            for (int b = k0 + kChunk; kChunked && b < k1; b += kChunk) {
                if (!sums_ready()) break;
                float v[2][16];
                tmem_load16(mine + buf * NT, v[0]);
#pragma unroll
                for (int c = 0; c < S::kCols; c += 16) {
                    float (&x)[16] = v[(c >> 4) & 1];
                    tmem_wait(x);
                    if (c + 16 < S::kCols) tmem_load16(mine + buf * NT + c + 16, v[((c >> 4) & 1) ^ 1]);
                    else sums_taken();
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[c + i] += x[i];
                }
            }
            if (!ok) {
#pragma unroll
                for (int i = 0; i < S::kCols; ++i) acc[i] = __uint_as_float(0x7FC00000u);
            }
            OT* const out = static_cast<OT*>(p.out) + part * p.split_stride;
            if (FUSED || p.swap) {
                if constexpr (NT == 64) store_transposed<OT, S::kCols>(p, out, acc, out_rows, row0 - quarter * 32, row0 + lane, col0);
                else store_swapped<OT, S::kCols>(p, out, acc, row0 + lane, col0);
            }
            else if constexpr (CG == 2 && NT == 256 && sizeof(OT) == 2) {
                const unsigned at = (unsigned)reinterpret_cast<uintptr_t>(out) | (unsigned)(p.ldo * sizeof(OT));
                // Rows lie in shared memory as they do in the output, within 16 bytes: by a distance that has the output's remainder.  It
                // also keeps the lanes' stores, of as many bytes as that remainder allows, out of each other's banks.
                const int over = (int)(p.ldo * sizeof(OT)) & 15, r = quarter * 32 + lane;
                const OT* const first = out + (long long)(row0 - quarter * 32) * p.ldo + tq * NT;
                unsigned char* const whole = out_rows + (reinterpret_cast<uintptr_t>(first) & 15u) + r * (512 + (over ? over : 16));
                if ((at & 15) == 0) store_row_halves<16>(p, out, acc, whole, row0 + lane, tq * NT, group, 1 + quarter);
                else if ((at & 7) == 0) store_row_halves<8>(p, out, acc, whole, row0 + lane, tq * NT, group, 1 + quarter);
                else if ((at & 3) == 0) store_row_halves<4>(p, out, acc, whole, row0 + lane, tq * NT, group, 1 + quarter);
                else store_row<OT, S::kCols>(p, out, acc, buffer, row0 + lane, col0);
            } else store_row<OT, S::kCols>(p, out, acc, buffer, row0 + lane, col0);
        }
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
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
__global__ void __launch_bounds__(256) k_join_parts(const float* parts, long long stride, int splits, OT* out, long long ldo, long long rows, int cols) {
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
template <typename KIND> static MatmulPlan plan_matmul(long long M, long long N, long long K) {
    MatmulPlan L{};
    const long long small = M < N ? M : N;
    // Up to 64 rows the small side is Q (and for Q = a the result leaves transposed, a column a lane).  With 65 to 128 it
    // is still b's case, but a of so few rows does better as half a pair's tile: 128 x 33708 x 1024 takes 17.5 us as
    // Q and 14.8 us so.
    const bool narrow = small <= 64 || (small <= 128 && N <= M);
    L.swap = narrow && M < N;
    L.cg = narrow ? 1 : 2;
    L.nt = !narrow ? 256 : small <= 16 ? 16 : small <= 32 ? 32 : small <= 64 ? 64 : 128;
    L.rows_p = L.swap ? N : M; L.rows_q = L.swap ? M : N;
    L.tiles_p = (L.rows_p + kTileP * L.cg - 1) / (kTileP * L.cg);
    L.tiles_q = (L.rows_q + L.nt - 1) / L.nt;
    L.blocks = (K + KIND::kStepCols - 1) / KIND::kStepCols;
    const long long groups = (L.blocks + KIND::kScaleSteps - 1) / KIND::kScaleSteps;
    // Parts, of whole loads of scales: the fewest microseconds by a model of 0.3 a step, 1 a tile, and for more than one part their results written
    // and read again at 4 TB/s and another launch.  SMs of a B200, not the device's, so that the order of the sums
    // follows from the sizes.
    const long long tiles = L.tiles_p * L.tiles_q, workers = kSmCount / L.cg;
    double best = 0;
    for (int s = 1; s <= kMaxParts && s <= groups; ++s) {
        if (s > 1 && tiles * s > 2 * workers) break;
        const long long rounds = (tiles * s + workers - 1) / workers, len = (groups + s - 1) / s * KIND::kScaleSteps;
        const double us = rounds * (len * 0.3 + 1.0) + (s > 1 ? 3.0 + double(s) * M * N * 8 / 4e6 : 0.0);
        if (s == 1 || us < best) { best = us; L.splits = s; }
    }
    return L;
}

template <typename KIND> static size_t block_matmul_workspace(long long M, long long N, long long K) {
    const MatmulPlan L = plan_matmul<KIND>(M, N, K);
    return L.splits > 1 ? size_t(L.splits) * size_t(M) * size_t(N) * 4 : 0;
}
// What no product up to these sizes exceeds: parts x tiles stay within two for each SM (or pair of them).
template <typename KIND> static size_t block_matmul_workspace_bound(long long M, long long N, long long K) {
    constexpr long long kGroup = KIND::kScaleSteps * KIND::kStepCols;
    const long long groups = (K + kGroup - 1) / kGroup;
    if (groups < 2) return 0;
    const size_t every = size_t(groups < kMaxParts ? groups : kMaxParts) * size_t(M) * size_t(N) * 4;
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
template <typename KIND> static bool operand_map(CUtensorMap& map, const Fp8View& m, int rows) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    constexpr int kPerByte = KIND::kStepCols / kBlockK;
    const cuuint64_t dims[2] = {(cuuint64_t)(m.cols + kPerByte - 1) / kPerByte, (cuuint64_t)m.rows}, strides[1] = {(cuuint64_t)m.ld};
    const cuuint32_t box[2] = {kBlockK, (cuuint32_t)rows}, step[2] = {1, 1};
    return encode(&map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, m.q, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The scales as [128 rows' tiles][groups of four scales][128 words], a tile a copy.
template <typename KIND> static bool scale_map(CUtensorMap& map, const Fp8View& m) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    constexpr int kGroup = KIND::kScaleSteps * KIND::kStepCols / KIND::kScaleTiles;   // columns of a tile
    const cuuint64_t dims[3] = {kScaleTile / 4, (cuuint64_t)((m.cols + kGroup - 1) / kGroup), (cuuint64_t)((m.rows + 127) / 128)};
    const cuuint64_t strides[2] = {kScaleTile, (cuuint64_t)m.ld_scale * kScaleTile};
    const cuuint32_t box[3] = {kScaleTile / 4, 1, 1}, step[3] = {1, 1, 1};
    return encode(&map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, m.scale, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
                  CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct MatmulMaps { CUtensorMap p, q, sp, sq; };
template <typename KIND, int CG, int NT, bool FUSED, typename OT>
static cudaError_t matmul_launch(const MatmulMaps& m, const MatmulParams& p, int sms, cudaStream_t stream) {
    using S = TileShape<KIND, CG, NT, FUSED>;
    static SmemOptIn opt;
    const cudaError_t e = ensure_dynamic_smem(k_block_matmul<KIND, CG, NT, FUSED, OT>, S::kSmem, opt);
    if (e != cudaSuccess) return e;
    const long long items = (long long)p.tiles_p * p.tiles_q * p.splits, workers = sms / CG * S::kCtas;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((items < workers ? items : workers) * CG)); cfg.blockDim = dim3(S::kThreads);
    cfg.dynamicSmemBytes = S::kSmem; cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CG; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, k_block_matmul<KIND, CG, NT, FUSED, OT>, m.p, m.q, m.sp, m.sq, p);
}
template <typename KIND, int CG, int NT, bool FUSED = false>
static cudaError_t matmul_nt(const MatmulMaps& m, const MatmulParams& p, int out_type, int sms, cudaStream_t stream) {
    return out_type == DST_F32 ? matmul_launch<KIND, CG, NT, FUSED, float>(m, p, sms, stream) : matmul_launch<KIND, CG, NT, FUSED, __nv_bfloat16>(m, p, sms, stream);
}

template <typename KIND> static cudaError_t launch_block_matmul(const Fp8View& a, const Fp8View& b, void* out, long long ldo, int out_type, void* workspace, int sms, cudaStream_t stream) {
    const MatmulPlan L = plan_matmul<KIND>(a.rows, b.rows, a.cols);
    const Fp8View &vp = L.swap ? b : a, &vq = L.swap ? a : b;
    MatmulMaps m;
    if (!operand_map<KIND>(m.p, vp, kTileP) || !operand_map<KIND>(m.q, vq, L.nt / L.cg) || !scale_map<KIND>(m.sp, vp) || !scale_map<KIND>(m.sq, vq)) return cudaErrorInvalidValue;
    MatmulParams p{(int)vp.rows, (int)vq.rows, (int)L.blocks, L.splits, (int)L.tiles_p, (int)L.tiles_q, L.swap, out, ldo, 0, nullptr, 0, 0, 0, 0};
    int type = out_type;
    if (L.splits > 1) { p.out = workspace; p.ldo = b.rows; p.split_stride = a.rows * b.rows; type = DST_F32; }
    cudaError_t e;
    switch (L.nt) {
        case 16: e = matmul_nt<KIND, 1, 16>(m, p, type, sms, stream); break;
        case 32: e = matmul_nt<KIND, 1, 32>(m, p, type, sms, stream); break;
        case 64: e = matmul_nt<KIND, 1, 64>(m, p, type, sms, stream); break;
        case 128: e = matmul_nt<KIND, 1, 128>(m, p, type, sms, stream); break;
        default: e = matmul_nt<KIND, 2, 256>(m, p, type, sms, stream); break;
    }
    if (e != cudaSuccess || L.splits == 1) return e;
    const long long total = a.rows * b.rows, blocks = (total + 255) / 256, cap = (long long)sms * 8;
    const dim3 grid((unsigned)(blocks < cap ? blocks : cap));
    const float* parts = static_cast<const float*>(workspace);
    if (out_type == DST_F32) return launch_pdl(k_join_parts<float>, grid, dim3(256), 0, stream, parts, p.split_stride, L.splits, static_cast<float*>(out), ldo, (long long)a.rows, (int)b.rows);
    return launch_pdl(k_join_parts<__nv_bfloat16>, grid, dim3(256), 0, stream, parts, p.split_stride, L.splits, static_cast<__nv_bfloat16*>(out), ldo, (long long)a.rows, (int)b.rows);
}

// x's rows quantised inside the product: what that takes of the sizes, and the call.
template <typename KIND> static bool block_linear_fits(const MatmulPlan& L) {
    return L.swap && L.nt == 16 && L.splits == 1 && L.blocks * L.nt * kBlockK <= TileShape<KIND, 1, 16, true>::kResident;
}
template <typename KIND>
static cudaError_t launch_block_linear(const void* x, long long ldx, int x_type, long long M, const Fp8View& w, void* out, long long ldo, int out_type,
                                       int sms, cudaStream_t stream) {
    const MatmulPlan L = plan_matmul<KIND>(M, w.rows, w.cols);
    MatmulMaps m;
    if (!operand_map<KIND>(m.p, w, kTileP) || !scale_map<KIND>(m.sp, w)) return cudaErrorInvalidValue;
    m.q = m.p; m.sq = m.sp;                                      // (not read)
    const size_t size = x_type == DST_F32 ? 4 : 2;
    const int vec = (reinterpret_cast<uintptr_t>(x) & (4 * size - 1)) == 0 && ldx % 4 == 0;
    const MatmulParams p{(int)w.rows, (int)M, (int)L.blocks, 1, (int)L.tiles_p, 1, 1, out, ldo, 0, x, ldx, w.cols, x_type, vec};
    return matmul_nt<KIND, 1, 16, true>(m, p, out_type, sms, stream);
}

}  // namespace dst
