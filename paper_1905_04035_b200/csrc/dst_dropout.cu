// Dropout whose random bits are a function of position, and the embedding lookup it follows.
//
// Nothing but x, residual and out touches memory: the mask is recomputed wherever it is needed, eight columns for one
// evaluation of the generator (Philox4x32-10 gives 128 bits; 16 bits an element resolve p to 2^-16).  For bf16 tensors the
// 40 multiplications and xors of an evaluation are most of the instructions, so everything around them is kept short:
// round keys come ready from the host, a half is compared in place, positions advance by additions.
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

// A unit is eight columns of a row and belongs to a thread; a dropped element adds nothing, whatever x holds there.
template <typename XT, typename OT, bool RES>
__global__ void __launch_bounds__(kDropThreads) k_dropout_vec(const __grid_constant__ DropoutParams p) {
    pdl_trigger();
    pdl_wait();
    const unsigned long long offset = drop_offset(p.drop);
    const float keep = p.drop.keep * p.scale;
    for (Walk at(p.step, (long long)blockIdx.x * kDropThreads + threadIdx.x); at.row < p.rows; at.next(p.step)) {
        const unsigned c = at.part * 8;
        float v[8], r[8];
        load8(static_cast<const XT*>(p.x) + at.row * p.ldx + c, v);
        if (RES) load8(static_cast<const OT*>(p.residual) + at.row * p.ldr + c, r);
        const Bits8 b = draw(p.drop, offset, (unsigned)at.row, at.part);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = kept(b, j, p.drop.below) ? v[j] * keep : 0.f;
            if (RES) v[j] += r[j];
        }
        store8(static_cast<OT*>(p.out) + at.row * p.ldo + c, v);
    }
}

// Rows that are not 16-byte aligned: a warp takes 256 consecutive columns, so that loads and stores are of neighbouring
// elements by neighbouring lanes.  Lane l draws the bits of columns 8 l .. 8 l + 7; a vote for each of the eight gives
// every lane the words from which it picks those of columns lane, lane + 32, ...
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
        const Bits8 b = draw(p.drop, offset, (unsigned)at.row, (unsigned)(c0 >> 3) + lane);
        unsigned word = 0;                                          // the vote on column lane % 8 of every lane's eight
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const unsigned vote = __ballot_sync(0xFFFFFFFFu, kept(b, j, p.drop.below));
            if ((lane & 7) == j) word = vote;
        }
        word >>= lane >> 3;                                         // bit 4 j: column j * 32 + lane
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j * 32 < n) {
                float t = (word >> (4 * j)) & 1u ? to_float(v[j]) * keep : 0.f;
                if (RES) t += to_float(r[j]);
                out[j * 32] = from_float<OT>(t);
            }
    }
}

// out row = keep * (scale * weight row + position row); a row of zeros for an index outside the table
template <typename IT, typename WT, typename OT, bool VEC>
__global__ void __launch_bounds__(kDropThreads) k_embed(const __grid_constant__ EmbedParams p) {
    pdl_trigger();
    pdl_wait();
    const unsigned long long offset = drop_offset(p.drop);
    for (Walk at(p.step, (long long)blockIdx.x * kDropThreads + threadIdx.x); at.row < p.rows; at.next(p.step)) {
        const int c = (int)at.part * 8, n = p.d - c < 8 ? p.d - c : 8;
        const long long index = (long long)static_cast<const IT*>(p.indices)[at.row];
        const bool valid = index >= 0 && index < p.vocab;
        if (!valid && at.part == 0 && p.result) {
            atomicAdd(reinterpret_cast<unsigned long long*>(&p.result->n_out_of_range), 1ull);
            p.result->status = DST_ERR_INDEX_OUT_OF_RANGE;
        }
        const float keep = valid ? p.drop.keep : 0.f;
        const WT* const w = static_cast<const WT*>(p.weight) + (valid ? index : 0) * p.d + c;
        const float* const pos = p.position ? p.position + (long long)((unsigned)at.row % (unsigned)p.n_positions) * p.d + c : nullptr;
        OT* const out = static_cast<OT*>(p.out) + at.row * p.d + c;
        float v[8], a[8];
        if (VEC) {
            load8(w, v);
            if (pos) load8(pos, a);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) { v[j] = j < n ? to_float(w[j]) : 0.f; if (pos) a[j] = j < n ? pos[j] : 0.f; }
        }
        const Bits8 b = draw(p.drop, offset, (unsigned)at.row, at.part);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float t = pos ? fmaf(v[j], p.scale, a[j]) : v[j] * p.scale;
            v[j] = valid && kept(b, j, p.drop.below) ? t * keep : 0.f;
        }
        if (VEC) store8(out, v);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j) if (j < n) out[j] = from_float<OT>(v[j]);
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
    const dim3 grid = vec ? grid_for(p.step, p.rows, p.d / 8, kDropThreads, sms) : grid_for(p.step, p.rows, (p.d + 255) / 256, kDropThreads / 32, sms);
    if (vec) return launch_pdl(k_dropout_vec<XT, OT, RES>, grid, dim3(kDropThreads), 0, stream, p);
    return launch_pdl(k_dropout_any<XT, OT, RES>, grid, dim3(kDropThreads), 0, stream, p);
}
template <typename XT, typename OT>
static cudaError_t dropout_r(const DropoutParams& p, int sms, cudaStream_t stream) {
    return p.residual ? dropout_t<XT, OT, true>(p, sms, stream) : dropout_t<XT, OT, false>(p, sms, stream);
}

cudaError_t launch_dropout(const DropoutParams& p, int x_type, int out_type, int sms, cudaStream_t stream) {
    if (x_type == DST_F32) return out_type == DST_F32 ? dropout_r<float, float>(p, sms, stream) : dropout_r<float, __nv_bfloat16>(p, sms, stream);
    return out_type == DST_F32 ? dropout_r<__nv_bfloat16, float>(p, sms, stream) : dropout_r<__nv_bfloat16, __nv_bfloat16>(p, sms, stream);
}

template <typename IT, typename WT, typename OT>
static cudaError_t embed_t(EmbedParams p, int sms, cudaStream_t stream) {
    const bool vec = p.d % 8 == 0 && aligned(p.weight, p.d, sizeof(WT)) && aligned(p.out, p.d, sizeof(OT)) && aligned(p.position, p.d, 4);
    const dim3 grid = grid_for(p.step, p.rows, (p.d + 7) / 8, kDropThreads, sms);
    if (vec) return launch_pdl(k_embed<IT, WT, OT, true>, grid, dim3(kDropThreads), 0, stream, p);
    return launch_pdl(k_embed<IT, WT, OT, false>, grid, dim3(kDropThreads), 0, stream, p);
}
template <typename IT>
static cudaError_t embed_i(const EmbedParams& p, int weight_type, int out_type, int sms, cudaStream_t stream) {
    if (weight_type == DST_F32) return out_type == DST_F32 ? embed_t<IT, float, float>(p, sms, stream) : embed_t<IT, float, __nv_bfloat16>(p, sms, stream);
    return out_type == DST_F32 ? embed_t<IT, __nv_bfloat16, float>(p, sms, stream) : embed_t<IT, __nv_bfloat16, __nv_bfloat16>(p, sms, stream);
}

cudaError_t launch_embed(const EmbedParams& p, int index_type, int weight_type, int out_type, int sms, cudaStream_t stream) {
    return index_type == DST_I64 ? embed_i<long long>(p, weight_type, out_type, sms, stream) : embed_i<int>(p, weight_type, out_type, sms, stream);
}

}  // namespace dst
