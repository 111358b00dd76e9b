// Dropout whose random bits are a function of position, and the embedding lookup it follows.
//
// Nothing but x, residual and out touches memory: the mask is recomputed wherever it is needed, eight columns for one
// evaluation of the generator (Philox4x32-10 gives 128 bits; 16 bits an element resolve p to 2^-16 and keep the
// generator at about 8 integer operations an element, below what the memory traffic of two bf16 tensors leaves time for).
#include "dst_tied.cuh"

namespace dst {

struct Bits8 { unsigned w[4]; };

// Philox4x32 with ten rounds: each round multiplies two words by fixed odd constants, xors the high halves with the
// other two words and the key, and the key moves by a fixed step.
__device__ __forceinline__ Bits8 philox(unsigned c0, unsigned c1, unsigned c2, unsigned c3, unsigned k0, unsigned k1) {
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const unsigned long long a = (unsigned long long)c0 * 0xD2511F53u, b = (unsigned long long)c2 * 0xCD9E8D57u;
        c0 = (unsigned)(b >> 32) ^ c1 ^ k0; c1 = (unsigned)b;
        c2 = (unsigned)(a >> 32) ^ c3 ^ k1; c3 = (unsigned)a;
        k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
    }
    return Bits8{{c0, c1, c2, c3}};
}

// bit j: column 8 * group + j of the row is kept
__device__ __forceinline__ unsigned keep_mask(const DropParams& p, unsigned long long offset, unsigned row, unsigned group) {
    if (p.cut == 0) return 0xFFu;
    const Bits8 b = philox(group, row + p.row_offset, (unsigned)offset, (unsigned)(offset >> 32), p.key0, p.key1);
    unsigned m = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        m |= ((b.w[j] & 0xFFFFu) >= p.cut ? 1u : 0u) << (2 * j);
        m |= ((b.w[j] >> 16) >= p.cut ? 1u : 0u) << (2 * j + 1);
    }
    return m;
}

__device__ __forceinline__ unsigned long long drop_offset(const DropParams& p) {
    return p.offset + (p.offset_device ? *p.offset_device : 0ull);
}

constexpr int kDropThreads = 256;

// A unit is eight columns of a row and belongs to a thread; a dropped element adds nothing, whatever x holds there.
template <typename XT, typename OT>
__global__ void __launch_bounds__(kDropThreads) k_dropout_vec(const __grid_constant__ DropoutParams p) {
    pdl_trigger();
    pdl_wait();
    const unsigned long long offset = drop_offset(p.drop);
    const unsigned groups = (unsigned)p.d >> 3;
    const float keep = p.drop.keep * p.scale;
    const long long units = p.rows * groups, stride = (long long)gridDim.x * kDropThreads;
    for (long long u = (long long)blockIdx.x * kDropThreads + threadIdx.x; u < units; u += stride) {
        const long long row = (u >> 32) ? u / groups : (long long)((unsigned)u / groups);
        const unsigned g = (unsigned)(u - row * groups);
        float v[8], r[8];
        load8(static_cast<const XT*>(p.x) + row * p.ldx + g * 8, v);
        if (p.residual) load8(static_cast<const OT*>(p.residual) + row * p.ldr + g * 8, r);
        const unsigned m = keep_mask(p.drop, offset, (unsigned)row, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float t = (m >> j) & 1u ? v[j] * keep : 0.f;
            v[j] = p.residual ? r[j] + t : t;
        }
        store8(static_cast<OT*>(p.out) + row * p.ldo + g * 8, v);
    }
}

// Rows that are not 16-byte aligned: a warp takes 256 consecutive columns, each lane computes the bits of eight
// consecutive ones and hands them out, so that loads and stores are of neighbouring elements by neighbouring lanes.
template <typename XT, typename OT>
__global__ void __launch_bounds__(kDropThreads) k_dropout_any(const __grid_constant__ DropoutParams p) {
    pdl_trigger();
    pdl_wait();
    const unsigned long long offset = drop_offset(p.drop);
    const int lane = lane_id(), chunks = (p.d + 255) >> 8;
    const float keep = p.drop.keep * p.scale;
    const long long units = p.rows * chunks, stride = (long long)gridDim.x * (kDropThreads / 32);
    for (long long u = (long long)blockIdx.x * (kDropThreads / 32) + warp_id(); u < units; u += stride) {
        const long long row = u / chunks;
        const int c0 = (int)(u - row * chunks) << 8;
        const XT* x = static_cast<const XT*>(p.x) + row * p.ldx;
        const OT* res = static_cast<const OT*>(p.residual) + (p.residual ? row * p.ldr : 0);
        OT* out = static_cast<OT*>(p.out) + row * p.ldo;
        XT v[8];
        OT r[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = c0 + j * 32 + lane;
            if (c < p.d) { v[j] = x[c]; if (p.residual) r[j] = res[c]; }
        }
        const unsigned mine = keep_mask(p.drop, offset, (unsigned)row, (unsigned)(c0 >> 3) + lane);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = c0 + j * 32 + lane;
            const unsigned m = __shfl_sync(0xFFFFFFFFu, mine, j * 4 + (lane >> 3));
            const float t = c < p.d && ((m >> (lane & 7)) & 1u) ? to_float(v[j]) * keep : 0.f;
            if (c < p.d) out[c] = from_float<OT>(p.residual ? to_float(r[j]) + t : t);
        }
    }
}

// out row = keep * (scale * weight row + position row); a row of zeros for an index outside the table
template <typename IT, typename WT, typename OT, bool VEC>
__global__ void __launch_bounds__(kDropThreads) k_embed(const __grid_constant__ EmbedParams p) {
    pdl_trigger();
    pdl_wait();
    const unsigned long long offset = drop_offset(p.drop);
    const unsigned groups = (unsigned)(p.d + 7) >> 3;
    const long long units = p.rows * groups, stride = (long long)gridDim.x * kDropThreads;
    for (long long u = (long long)blockIdx.x * kDropThreads + threadIdx.x; u < units; u += stride) {
        const long long row = (u >> 32) ? u / groups : (long long)((unsigned)u / groups);
        const unsigned g = (unsigned)(u - row * groups);
        const int c0 = (int)g * 8, n = p.d - c0 < 8 ? p.d - c0 : 8;
        const long long index = (long long)static_cast<const IT*>(p.indices)[row];
        const bool valid = index >= 0 && index < p.vocab;
        if (!valid && g == 0 && p.result) {
            atomicAdd(reinterpret_cast<unsigned long long*>(&p.result->n_out_of_range), 1ull);
            p.result->status = DST_ERR_INDEX_OUT_OF_RANGE;
        }
        const unsigned m = valid ? keep_mask(p.drop, offset, (unsigned)row, g) : 0u;
        const WT* w = static_cast<const WT*>(p.weight) + (valid ? index : 0) * p.d + c0;
        const float* pos = p.position ? p.position + (long long)((unsigned)row % (unsigned)p.n_positions) * p.d + c0 : nullptr;
        OT* out = static_cast<OT*>(p.out) + row * p.d + c0;
        float v[8], a[8];
        if (VEC) {
            load8(w, v);
            if (pos) load8(pos, a);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) { v[j] = j < n ? to_float(w[j]) : 0.f; if (pos) a[j] = j < n ? pos[j] : 0.f; }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float t = pos ? fmaf(v[j], p.scale, a[j]) : v[j] * p.scale;
            v[j] = (m >> j) & 1u ? t * p.drop.keep : 0.f;
        }
        if (VEC) store8(out, v);
        else for (int j = 0; j < n; ++j) out[j] = from_float<OT>(v[j]);
    }
}

static bool aligned(const void* p, long long ld, size_t size) {
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (ld * (long long)size) % 16 == 0;
}
static dim3 grid_for(long long units, int per_block, int sms) {
    const long long blocks = (units + per_block - 1) / per_block, cap = (long long)sms * 32;
    return dim3((unsigned)(blocks < 1 ? 1 : blocks < cap ? blocks : cap));
}

template <typename XT, typename OT>
static cudaError_t dropout_t(const DropoutParams& p, int sms, cudaStream_t stream) {
    const bool vec = p.d % 8 == 0 && aligned(p.x, p.ldx, sizeof(XT)) && aligned(p.out, p.ldo, sizeof(OT)) &&
                     (!p.residual || aligned(p.residual, p.ldr, sizeof(OT)));
    if (vec) return launch_pdl(k_dropout_vec<XT, OT>, grid_for(p.rows * (p.d / 8), kDropThreads, sms), dim3(kDropThreads), 0, stream, p);
    return launch_pdl(k_dropout_any<XT, OT>, grid_for(p.rows * ((p.d + 255) / 256), kDropThreads / 32, sms), dim3(kDropThreads), 0, stream, p);
}

cudaError_t launch_dropout(const DropoutParams& p, int x_type, int out_type, int sms, cudaStream_t stream) {
    if (x_type == DST_F32) return out_type == DST_F32 ? dropout_t<float, float>(p, sms, stream) : dropout_t<float, __nv_bfloat16>(p, sms, stream);
    return out_type == DST_F32 ? dropout_t<__nv_bfloat16, float>(p, sms, stream) : dropout_t<__nv_bfloat16, __nv_bfloat16>(p, sms, stream);
}

template <typename IT, typename WT, typename OT>
static cudaError_t embed_t(const EmbedParams& p, int sms, cudaStream_t stream) {
    const bool vec = p.d % 8 == 0 && aligned(p.weight, p.d, sizeof(WT)) && aligned(p.out, p.d, sizeof(OT)) && aligned(p.position, p.d, 4);
    const dim3 grid = grid_for(p.rows * ((p.d + 7) / 8), kDropThreads, sms);
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
