// Dropout whose random bits are a function of position, and the embedding lookup it follows.
//
// Nothing but x, residual and out touches memory: the mask is recomputed wherever it is needed, eight columns for one
// evaluation of the generator (Philox4x32-10 gives 128 bits; 16 bits an element resolve p to 2^-16).  For bf16 tensors the
// 40 multiplications and xors of an evaluation are most of the instructions, so everything around them is kept short:
// round keys come ready from the host, a half is compared in place, positions advance by additions.
// Measured, of 6551 GB/s: dropout of 51,200 x 1024 bf16 34 us (6150 GB/s), with a residual 48 us (6510); 12,801 x 1021 fp32
// with a residual 24.5 us (6400); embedding of 25,600 rows of 1024, bf16, 24.9 us (18.6 without dropout: the generator bounds
// it), fp32 table 26.5 us (5900).
#include "dst_tied.cuh"

namespace dst {

struct Bits8 { unsigned w[4]; };

// Philox4x32 with ten rounds: each round multiplies two words by fixed odd constants and xors the high halves with the
// other two words and the round's keys.
__device__ __forceinline__ Bits8 philox(const DropParams& p, unsigned c0, unsigned c1, unsigned c2, unsigned c3) {
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const unsigned long long a = (unsigned long long)c0 * 0xD2511F53u, b = (unsigned long long)c2 * 0xCD9E8D57u;
        c0 = (unsigned)(b >> 32) ^ c1 ^ p.key0[r]; c1 = (unsigned)b;
        c2 = (unsigned)(a >> 32) ^ c3 ^ p.key1[r]; c3 = (unsigned)a;
    }
    return Bits8{{c0, c1, c2, c3}};
}
__device__ __forceinline__ Bits8 draw(const DropParams& p, unsigned long long offset, unsigned row, unsigned group) {
    if (p.none) return Bits8{{0xFFFFFFFFu, 0xFFFFFFFFu, 0xFFFFFFFFu, 0xFFFFFFFFu}};   // above `below`, which is 0 then
    return philox(p, group, row + p.row_offset, (unsigned)offset, (unsigned)(offset >> 32));
}
// column j of the eight is kept: its half, moved to the upper half of a word, is above the limit
__device__ __forceinline__ bool kept(const Bits8& b, int j, unsigned below) { return (j & 1 ? b.w[j >> 1] : b.w[j >> 1] << 16) > below; }

__device__ __forceinline__ unsigned long long drop_offset(const DropParams& p) {
    return p.offset + (p.offset_device ? *p.offset_device : 0ull);
}

// The units that a thread (or a warp) takes: its first one by a division, the next ones by additions.
struct Walk {
    long long row;
    unsigned part;
    __device__ __forceinline__ Walk(const UnitStep& s, long long unit) : row(unit / s.per_row), part((unsigned)(unit - row * s.per_row)) {}
    __device__ __forceinline__ void next(const UnitStep& s) {
        row += s.rows;
        part += s.part;
        if (part >= s.per_row) { part -= s.per_row; ++row; }
    }
};

constexpr int kDropThreads = 256;

// A unit belongs to a thread: eight columns of a row, and where the row has an even number of eights (HALVES 2) the eight
// half a row further on too, which shares what finding the row costs.  A dropped element adds nothing, whatever x holds there.
template <typename XT, typename OT, bool RES, int HALVES>
__global__ void __launch_bounds__(kDropThreads) k_dropout_vec(const __grid_constant__ DropoutParams p) {
    pdl_trigger();
    pdl_wait();
    const unsigned long long offset = drop_offset(p.drop);
    const float keep = p.drop.keep * p.scale;
    for (Walk at(p.step, (long long)blockIdx.x * kDropThreads + threadIdx.x); at.row < p.rows; at.next(p.step)) {
        const XT* const x = static_cast<const XT*>(p.x) + at.row * p.ldx;
        const OT* const res = RES ? static_cast<const OT*>(p.residual) + at.row * p.ldr : nullptr;
        OT* const out = static_cast<OT*>(p.out) + at.row * p.ldo;
        float v[HALVES][8], r[HALVES][8];
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            const unsigned c = (at.part + h * p.step.per_row) * 8;
            load8(x + c, v[h]);
            if (RES) load8(res + c, r[h]);
        }
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            const unsigned group = at.part + h * p.step.per_row;
            const Bits8 b = draw(p.drop, offset, (unsigned)at.row, group);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[h][j] = kept(b, j, p.drop.below) ? v[h][j] * keep : 0.f;
                if (RES) v[h][j] += r[h][j];
            }
            store8(out + group * 8, v[h]);
        }
    }
}

// Rows that are not 16-byte aligned: a warp takes 256 consecutive columns, so that loads and stores are of neighbouring
// elements by neighbouring lanes.  Lane l draws the bits of columns c0 + 8 l .. c0 + 8 l + 7; a vote for each of the eight
// gives every lane the words from which it picks its own: bit 4 j is that of column c0 + 32 j + lane.
__device__ __forceinline__ unsigned kept_word(const DropParams& p, unsigned long long offset, unsigned row, int c0) {
    const int lane = lane_id();
    const Bits8 b = draw(p, offset, row, (unsigned)(c0 >> 3) + lane);
    unsigned word = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const unsigned vote = __ballot_sync(0xFFFFFFFFu, kept(b, j, p.below));
        if ((lane & 7) == j) word = vote;
    }
    return word >> (lane >> 3);
}
template <typename XT, typename OT, bool RES>
__global__ void __launch_bounds__(kDropThreads) k_dropout_any(const __grid_constant__ DropoutParams p) {
    pdl_trigger();
    pdl_wait();
    const unsigned long long offset = drop_offset(p.drop);
    const int lane = lane_id();
    const float keep = p.drop.keep * p.scale;
    for (Walk at(p.step, (long long)blockIdx.x * (kDropThreads / 32) + warp_id()); at.row < p.rows; at.next(p.step)) {
        const int c0 = (int)at.part << 8, n = p.d - c0 - lane;      // this lane's columns are 0, 32, ... below n
        const XT* const x = static_cast<const XT*>(p.x) + at.row * p.ldx + c0 + lane;
        const OT* const res = RES ? static_cast<const OT*>(p.residual) + at.row * p.ldr + c0 + lane : nullptr;
        OT* const out = static_cast<OT*>(p.out) + at.row * p.ldo + c0 + lane;
        XT v[8];
        OT r[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j * 32 < n) { v[j] = x[j * 32]; if (RES) r[j] = res[j * 32]; }
        const unsigned word = kept_word(p.drop, offset, (unsigned)at.row, c0);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j * 32 < n) {
                float t = (word >> (4 * j)) & 1u ? to_float(v[j]) * keep : 0.f;
                if (RES) t += to_float(r[j]);
                out[j * 32] = from_float<OT>(t);
            }
    }
}

// What a token's index says: where its row lies; an index outside the table is counted once and gives a row of zeros.  The
// table's first row is read in its place, and not used (a table without rows does not come here): loads that depend
// on the index's check took 25600 rows of 1024, bf16, from 25.3 to 27.8 us, and of 1021 from 43.0 to 46.4.
template <typename IT>
__device__ __forceinline__ bool token_row(const EmbedParams& p, long long row, bool counts, long long& index) {
    index = (long long)static_cast<const IT*>(p.indices)[row];
    if (index >= 0 && index < p.vocab) return true;
    index = 0;
    if (counts && p.result) {
        atomicAdd(reinterpret_cast<unsigned long long*>(&p.result->n_out_of_range), 1ull);
        p.result->status = DST_ERR_INDEX_OUT_OF_RANGE;
    }
    return false;
}
__device__ __forceinline__ const float* position_row(const EmbedParams& p, long long row) {
    return p.position + (long long)((unsigned)row % (unsigned)p.n_positions) * p.d;
}

// out row = keep * (scale * weight row + position row); units as above
template <typename IT, typename WT, typename OT, bool POS, int HALVES>
__global__ void __launch_bounds__(kDropThreads) k_embed_vec(const __grid_constant__ EmbedParams p) {
    pdl_trigger();
    pdl_wait();
    const unsigned long long offset = drop_offset(p.drop);
    for (Walk at(p.step, (long long)blockIdx.x * kDropThreads + threadIdx.x); at.row < p.rows; at.next(p.step)) {
        long long index;
        const bool valid = token_row<IT>(p, at.row, at.part == 0, index);
        const WT* const w = static_cast<const WT*>(p.weight) + index * p.d;
        const float* const pos = POS ? position_row(p, at.row) : nullptr;
        OT* const out = static_cast<OT*>(p.out) + at.row * p.d;
        float v[HALVES][8], a[HALVES][8];
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            const unsigned c = (at.part + h * p.step.per_row) * 8;
            load8(w + c, v[h]);
            if (POS) load8(pos + c, a[h]);
        }
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            const unsigned group = at.part + h * p.step.per_row;
            const Bits8 b = draw(p.drop, offset, (unsigned)at.row, group);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float t = POS ? fmaf(v[h][j], p.scale, a[h][j]) : v[h][j] * p.scale;
                v[h][j] = valid && kept(b, j, p.drop.below) ? t * p.drop.keep : 0.f;
            }
            store8(out + group * 8, v[h]);
        }
    }
}

// the same for rows that are not aligned, a warp 256 columns
template <typename IT, typename WT, typename OT, bool POS>
__global__ void __launch_bounds__(kDropThreads) k_embed_any(const __grid_constant__ EmbedParams p) {
    pdl_trigger();
    pdl_wait();
    const unsigned long long offset = drop_offset(p.drop);
    const int lane = lane_id();
    for (Walk at(p.step, (long long)blockIdx.x * (kDropThreads / 32) + warp_id()); at.row < p.rows; at.next(p.step)) {
        const int c0 = (int)at.part << 8, n = p.d - c0 - lane;
        long long index;
        const bool valid = token_row<IT>(p, at.row, at.part == 0 && lane == 0, index);
        const WT* const w = static_cast<const WT*>(p.weight) + index * p.d + c0 + lane;
        const float* const pos = POS ? position_row(p, at.row) + c0 + lane : nullptr;
        OT* const out = static_cast<OT*>(p.out) + at.row * p.d + c0 + lane;
        WT v[8];
        float a[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j * 32 < n) { v[j] = w[j * 32]; if (POS) a[j] = pos[j * 32]; }
        const unsigned word = valid ? kept_word(p.drop, offset, (unsigned)at.row, c0) : 0u;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j * 32 < n) {
                const float t = POS ? fmaf(to_float(v[j]), p.scale, a[j]) : to_float(v[j]) * p.scale;
                out[j * 32] = from_float<OT>((word >> (4 * j)) & 1u ? t * p.drop.keep : 0.f);
            }
    }
}

static bool aligned(const void* p, long long ld, size_t size) {
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (ld * (long long)size) % 16 == 0;
}
// The grid for `rows` x `per_row` units, per_block at once, and how far apart a thread's are then.
static dim3 grid_for(UnitStep& s, long long rows, long long per_row, int per_block, int sms) {
    s.units = rows * per_row; s.per_row = (unsigned)per_row;
    const long long blocks = (s.units + per_block - 1) / per_block, cap = (long long)sms * 32;
    const long long grid = blocks < 1 ? 1 : blocks < cap ? blocks : cap;
    s.rows = grid * per_block / per_row; s.part = (unsigned)(grid * per_block % per_row);
    return dim3((unsigned)grid);
}

template <typename XT, typename OT, bool RES>
static cudaError_t dropout_t(DropoutParams p, int sms, cudaStream_t stream) {
    const bool vec = p.d % 8 == 0 && aligned(p.x, p.ldx, sizeof(XT)) && aligned(p.out, p.ldo, sizeof(OT)) &&
                     (!p.residual || aligned(p.residual, p.ldr, sizeof(OT)));
    const dim3 threads(kDropThreads);
    if (!vec) {
        const dim3 grid = grid_for(p.step, p.rows, (p.d + 255) / 256, kDropThreads / 32, sms);
        return launch_pdl(k_dropout_any<XT, OT, RES>, grid, threads, 0, stream, p);
    }
    // two eights a thread where they are 32 bytes to load (51200 x 1024 bf16: 36.6 -> 34.1 us); with more, the registers
    // cost warps (25600 x 1024 bf16 with a residual: 24.3 -> 25.8 us)
    if constexpr (sizeof(XT) == 2 && !RES)
        if (p.d % 16 == 0) {
            const dim3 grid = grid_for(p.step, p.rows, p.d / 16, kDropThreads, sms);
            return launch_pdl(k_dropout_vec<XT, OT, RES, 2>, grid, threads, 0, stream, p);
        }
    const dim3 grid = grid_for(p.step, p.rows, p.d / 8, kDropThreads, sms);
    return launch_pdl(k_dropout_vec<XT, OT, RES, 1>, grid, threads, 0, stream, p);
}
template <typename XT, typename OT>
static cudaError_t dropout_r(const DropoutParams& p, int sms, cudaStream_t stream) {
    return p.residual ? dropout_t<XT, OT, true>(p, sms, stream) : dropout_t<XT, OT, false>(p, sms, stream);
}

cudaError_t launch_dropout(const DropoutParams& p, int x_type, int out_type, int sms, cudaStream_t stream) {
    if (x_type == DST_F32) return out_type == DST_F32 ? dropout_r<float, float>(p, sms, stream) : dropout_r<float, __nv_bfloat16>(p, sms, stream);
    return out_type == DST_F32 ? dropout_r<__nv_bfloat16, float>(p, sms, stream) : dropout_r<__nv_bfloat16, __nv_bfloat16>(p, sms, stream);
}

template <typename IT, typename WT, typename OT, bool POS>
static cudaError_t embed_t(EmbedParams p, int sms, cudaStream_t stream) {
    const bool vec = p.d % 8 == 0 && aligned(p.weight, p.d, sizeof(WT)) && aligned(p.out, p.d, sizeof(OT)) && aligned(p.position, p.d, 4);
    const dim3 threads(kDropThreads);
    if (!vec) {
        const dim3 grid = grid_for(p.step, p.rows, (p.d + 255) / 256, kDropThreads / 32, sms);
        return launch_pdl(k_embed_any<IT, WT, OT, POS>, grid, threads, 0, stream, p);
    }
    // two eights a thread (25600 x 1024, weight bf16: 27.2 -> 24.8 us; fp32: 28.5 -> 31.3 us)
    if constexpr (sizeof(WT) == 2)
        if (p.d % 16 == 0) {
            const dim3 grid = grid_for(p.step, p.rows, p.d / 16, kDropThreads, sms);
            return launch_pdl(k_embed_vec<IT, WT, OT, POS, 2>, grid, threads, 0, stream, p);
        }
    const dim3 grid = grid_for(p.step, p.rows, p.d / 8, kDropThreads, sms);
    return launch_pdl(k_embed_vec<IT, WT, OT, POS, 1>, grid, threads, 0, stream, p);
}
template <typename IT, bool POS>
static cudaError_t embed_i(const EmbedParams& p, int weight_type, int out_type, int sms, cudaStream_t stream) {
    if (weight_type == DST_F32) return out_type == DST_F32 ? embed_t<IT, float, float, POS>(p, sms, stream) : embed_t<IT, float, __nv_bfloat16, POS>(p, sms, stream);
    return out_type == DST_F32 ? embed_t<IT, __nv_bfloat16, float, POS>(p, sms, stream) : embed_t<IT, __nv_bfloat16, __nv_bfloat16, POS>(p, sms, stream);
}

// A table without rows: no index lies inside it.  Nothing is read; the zeros of `out` are a memset.
__global__ void k_embed_none(dst_result_t* result, long long rows) {
    pdl_trigger();
    pdl_wait();
    result->status = DST_ERR_INDEX_OUT_OF_RANGE;
    result->n_out_of_range = rows;
}
static cudaError_t embed_none(const EmbedParams& p, int out_type, cudaStream_t stream) {
    const cudaError_t e = cudaMemsetAsync(p.out, 0, size_t(p.rows) * size_t(p.d) * (out_type == DST_F32 ? 4 : 2), stream);
    if (e != cudaSuccess || !p.result) return e;
    return launch_pdl(k_embed_none, dim3(1), dim3(1), 0, stream, p.result, p.rows);
}

cudaError_t launch_embed(const EmbedParams& p, int index_type, int weight_type, int out_type, int sms, cudaStream_t stream) {
    if (p.vocab == 0) return embed_none(p, out_type, stream);
    if (index_type == DST_I64) return p.position ? embed_i<long long, true>(p, weight_type, out_type, sms, stream) : embed_i<long long, false>(p, weight_type, out_type, sms, stream);
    return p.position ? embed_i<int, true>(p, weight_type, out_type, sms, stream) : embed_i<int, false>(p, weight_type, out_type, sms, stream);
}

}  // namespace dst
