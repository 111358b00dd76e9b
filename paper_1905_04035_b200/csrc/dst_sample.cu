// One token per row of logits from a given uniform number, with temperature, top-k, top-p and min-p.
//
// No sort.  The filters keep the entries above some value and the first few (in index order) of those equal to it, so
// a row needs that value and that count alone: a histogram over equal steps of the scaled logit finds the step in
// which top-k's count, or top-p's mass, is reached, and finer histograms over the bits of the logit narrow the step
// down to one value.  The weights are whole numbers (2^31 * exp, rounded), so every sum is exact whatever its order.
//
// A row belongs to a cluster of 1, 2, 4 or 8 CTAs, each with a slice of it in shared memory; the histograms are
// joined through distributed shared memory, and every CTA takes the same decisions from the joined one.
#include <cooperative_groups.h>

#include "dst_tied.cuh"

namespace dst {
namespace cg = cooperative_groups;

typedef unsigned long long u64;
constexpr int kSampleThreads = 1024;
constexpr int kSampleWarps = kSampleThreads / 32;
constexpr int kSampleCtas = 8;               // of a cluster, at most
constexpr int kBins = 2048;
constexpr float kZeroWeight = -22.25f;       // below this z the weight rounds to zero (2^31 e^z < 1/2 below -22.18)
constexpr float kBinsPerZ = kBins / 22.25f;
constexpr int kSampleSlice = 65536;          // entries a CTA takes, at most: its sums of 16-bit halves stay within 32 bits
constexpr unsigned kLowestKey = 0x007FFFFFu; // key of -infinity

// order-preserving bits of a float; equal floats (the two zeros) have equal keys, NaN counts as -infinity
__device__ __forceinline__ unsigned key_of(float x) {
    x = x == x ? x + 0.f : -INFINITY;
    const unsigned b = __float_as_uint(x);
    return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float of_key(unsigned k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xFFFFFFFFu)); }

struct Row {                                 // what turns a logit into its weight
    float top, inv_t, min_p;
    __device__ __forceinline__ float z(float x) const { return x == top ? 0.f : __fmul_rn(x - top, inv_t); }
    __device__ __forceinline__ static unsigned weight(float e) { return __float2uint_rn(e * 2147483648.f); }
};

// part / 2^24 of total, rounded down
__device__ __forceinline__ u64 share(unsigned part, u64 total) {
    return (u64)part * (total >> 24) + (((u64)part * (total & 0xFFFFFFu)) >> 24);
}

struct SampleShared {
    unsigned count[kBins], low[kBins], high[kBins];              // this CTA's histogram (the mass in halves of 16 bits)
    u64 joined_mass[kBins];                                      // the cluster's
    unsigned joined_count[kBins];
    u64 seg_mass[kSampleWarps];
    unsigned seg_ties[kSampleWarps];
    unsigned top_key;
    unsigned warp_key[kSampleWarps];
    unsigned warp_count[kSampleWarps];
    u64 warp_mass[kSampleWarps];
    unsigned hit_bin, hit_count_above, hit_count;
    u64 hit_mass_above, hit_mass;
    unsigned pick_seg, pick_ties;
    u64 pick_left, pick_total;
};

// Where the running count (by_mass: mass) over the joined bins first reaches `need`: the bin, and what is above it.
// `need` is at least 1 and at most the sum.
__device__ void find_bin(SampleShared& s, u64 need, bool by_mass) {
    constexpr int kPer = kBins / kSampleThreads;
    const int first = threadIdx.x * kPer, lane = lane_id(), warp = warp_id();
    unsigned c[kPer], n = 0;
    u64 m[kPer], mass = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        c[i] = s.joined_count[first + i];
        m[i] = s.joined_mass[first + i];
        n += c[i]; mass += m[i];
    }
    unsigned n_in = n;
    u64 mass_in = mass;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const unsigned a = __shfl_up_sync(0xFFFFFFFFu, n_in, d);
        const u64 b = __shfl_up_sync(0xFFFFFFFFu, mass_in, d);
        if (lane >= d) { n_in += a; mass_in += b; }
    }
    if (lane == 31) { s.warp_count[warp] = n_in; s.warp_mass[warp] = mass_in; }
    __syncthreads();
    unsigned n_before = n_in - n;
    u64 mass_before = mass_in - mass;
    for (int w = 0; w < warp; ++w) { n_before += s.warp_count[w]; mass_before += s.warp_mass[w]; }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const u64 before = by_mass ? mass_before : n_before, here = by_mass ? m[i] : c[i];
        if (before < need && need <= before + here) {
            s.hit_bin = first + i; s.hit_count_above = n_before; s.hit_mass_above = mass_before;
            s.hit_count = c[i]; s.hit_mass = m[i];
        }
        n_before += c[i]; mass_before += m[i];
    }
    __syncthreads();
}

template <typename T>
__global__ void __launch_bounds__(kSampleThreads) k_sample(const __grid_constant__ SampleParams p) {
    extern __shared__ __align__(16) unsigned char dyn[];
    SampleShared& s = *reinterpret_cast<SampleShared*>(dyn);
    cg::cluster_group cluster = cg::this_cluster();
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const long long row = blockIdx.x / ctas;
    const int tid = threadIdx.x, lane = lane_id(), warp = warp_id();
    pdl_trigger();
    pdl_wait();

    // ---- the slice, into shared memory at its own offset within 16 bytes ----
    const int slice = ((p.vocab + ctas - 1) / ctas + 7) / 8 * 8;
    const int begin = min(rank * slice, p.vocab), n = min(slice, p.vocab - begin);
    const T* src = static_cast<const T*>(p.logits) + row * p.ld + begin;
    const int skew = (int)((reinterpret_cast<uintptr_t>(src) & 15u) / sizeof(T));
    T* const x = reinterpret_cast<T*>(dyn + (sizeof(SampleShared) + 15) / 16 * 16) + skew;
    {
        constexpr int kVec = 16 / sizeof(T);
        const int head = min(n, (kVec - skew) % kVec), body = (n - head) / kVec;
        for (int i = tid; i < head; i += kSampleThreads) x[i] = src[i];
        for (int i = tid; i < body; i += kSampleThreads)
            reinterpret_cast<uint4*>(x + head)[i] = reinterpret_cast<const uint4*>(src + head)[i];
        for (int i = head + body * kVec + tid; i < n; i += kSampleThreads) x[i] = src[i];
    }
    __syncthreads();

    // ---- the largest logit ----
    unsigned top_key = 0;
    for (int i = tid; i < n; i += kSampleThreads) top_key = max(top_key, key_of(to_float(x[i])));
    top_key = __reduce_max_sync(0xFFFFFFFFu, top_key);
    if (lane == 0) s.warp_key[warp] = top_key;
    __syncthreads();
    if (warp == 0) {
        top_key = __reduce_max_sync(0xFFFFFFFFu, s.warp_key[lane]);
        if (lane == 0) s.top_key = top_key;
    }
    cluster.sync();
    top_key = 0;
    for (int c = 0; c < ctas; ++c) top_key = max(top_key, *cluster.map_shared_rank(&s.top_key, c));

    Row r;
    r.top = of_key(top_key);
    const float t = p.temperature ? p.temperature[row] : 1.f;
    r.inv_t = 1.f / t;
    r.min_p = p.min_p ? fminf(p.min_p[row], 1.f) : 0.f;
    int k = p.top_k ? p.top_k[row] : 0;
    if (k <= 0 || k >= p.vocab) k = 0;
    const float top_p = p.top_p ? p.top_p[row] : 1.f;
    const bool by_mass = top_p < 1.f;
    const bool nothing = top_key <= kLowestKey;
    const bool greedy = !(t > 0.f) || k == 1;

    // ---- the value the filters keep down to, and how many of the entries equal to it ----
    unsigned cut_key = 0, cut_ties = 0xFFFFFFFFu;
    if (greedy) { cut_key = top_key; cut_ties = 1; r.inv_t = __int_as_float(0x7F800000); }
    else if (!nothing && (k || by_mass)) {
        constexpr int kShift = sizeof(T) == 2 ? 16 : 0;          // bf16 logits differ in the upper half of the key only
        const float step = 1.f / (kBinsPerZ * r.inv_t);          // width of a bin in logits
        auto histogram = [&](bool coarse, unsigned bin, unsigned hi, int shift) {
            for (int i = tid; i < kBins; i += kSampleThreads) { s.count[i] = 0; s.low[i] = 0; s.high[i] = 0; }
            __syncthreads();
            for (int i = tid; i < n; i += kSampleThreads) {
                const unsigned key = key_of(to_float(x[i]));
                const float v = of_key(key), z = r.z(v);
                if (!(z > kZeroWeight) || key <= kLowestKey) continue;
                unsigned b = min((unsigned)(-z * kBinsPerZ), (unsigned)kBins - 1);
                if (!coarse) {
                    if (b != bin || (key >> kShift) > hi) continue;
                    b = (hi - (key >> kShift)) >> shift;
                    if (b >= kBins) continue;
                }
                const unsigned w = Row::weight(expf(z));
                if (w == 0) continue;
                atomicAdd(&s.count[b], 1u);
                atomicAdd(&s.low[b], w & 0xFFFFu);
                atomicAdd(&s.high[b], w >> 16);
            }
            cluster.sync();
            const int share_bins = kBins / ctas;
            for (int i = tid; i < share_bins; i += kSampleThreads) {
                const int at = rank * share_bins + i;
                unsigned a = 0;
                u64 m = 0;
                for (int c = 0; c < ctas; ++c) {
                    a += *cluster.map_shared_rank(&s.count[at], c);
                    m += *cluster.map_shared_rank(&s.low[at], c) + ((u64)*cluster.map_shared_rank(&s.high[at], c) << 16);
                }
                for (int c = 0; c < ctas; ++c) {
                    *cluster.map_shared_rank(&s.joined_count[at], c) = a;
                    *cluster.map_shared_rank(&s.joined_mass[at], c) = m;
                }
            }
            cluster.sync();
        };
        // narrows the coarse bin in s.hit_* down to one key; `need` counts from the top of the row.  Leaves the sums
        // above that key and at it.
        auto refine = [&](u64 need, bool mass, u64& mass_above, unsigned& count_above, unsigned& key) {
            const unsigned bin = s.hit_bin;
            mass_above = s.hit_mass_above; count_above = s.hit_count_above;
            // bounds of the bin's logits, a little wider than the roundings of z and of the bin number can move them
            const float near = bin ? (float)bin * step * (1.f - 0x1p-20f) : 0.f, far = (float)(bin + 1) * step * (1.f + 0x1p-20f);
            unsigned hi = min(top_key, key_of(__fsub_ru(r.top, near))) >> kShift;
            unsigned lo = key_of(bin == kBins - 1 ? -INFINITY : __fsub_rd(r.top, far)) >> kShift;
            for (;;) {
                int shift = 0;
                while ((hi - lo) >> shift >= kBins) ++shift;
                __syncthreads();                                  // everybody has read s.hit_*
                histogram(false, bin, hi, shift);
                find_bin(s, need - (mass ? mass_above : (u64)count_above), mass);
                mass_above += s.hit_mass_above; count_above += s.hit_count_above;
                hi -= s.hit_bin << shift;
                const unsigned low = hi - ((1u << shift) - 1u);
                lo = low > hi || low < lo ? lo : low;
                if (shift == 0) break;
            }
            key = kShift == 0 ? hi : hi << kShift | (hi >> 15 ? 0u : 0xFFFFu);   // a negative number's bits are inverted
        };
        histogram(true, 0, 0, 0);
        unsigned total = 0;
        u64 total_mass = 0;
        {   // sums over all bins: the last thread's running sums in find_bin would do, but the filters may not ask for it
            find_bin(s, 1, false);
            for (int w = 0; w < kSampleWarps; ++w) { total += s.warp_count[w]; total_mass += s.warp_mass[w]; }
            __syncthreads();
        }
        u64 kept_mass = total_mass;
        u64 mass_above;
        unsigned count_above;
        if (k && (unsigned)k < total) {                           // fewer weights above zero than k: k keeps them all
            find_bin(s, k, false);
            refine(k, false, mass_above, count_above, cut_key);
            cut_ties = k - count_above;
            const unsigned w = Row::weight(expf(r.z(of_key(cut_key))));
            kept_mass = mass_above + (u64)cut_ties * w;
        }
        if (by_mass) {
            const unsigned part = top_p > 0.f ? (unsigned)(top_p * 16777216.f) : 0u;
            const u64 upto = max(share(part, kept_mass), (u64)1);
            if (cut_key) { __syncthreads(); histogram(true, 0, 0, 0); }
            find_bin(s, upto, true);
            unsigned key;
            refine(upto, true, mass_above, count_above, key);
            const unsigned w = Row::weight(expf(r.z(of_key(key))));
            const u64 ties = (upto - mass_above + w - 1) / w;
            if (key > cut_key) { cut_key = key; cut_ties = (unsigned)min(ties, (u64)0xFFFFFFFFu); }
            else cut_ties = (unsigned)min(ties, (u64)cut_ties);
        }
    }

    // ---- kept mass of every warp's segment (consecutive entries), in index order ----
    const int seg_len = ((slice + kSampleWarps - 1) / kSampleWarps + 31) / 32 * 32;
    const int seg_begin = min(warp * seg_len, n), seg_end = min(seg_begin + seg_len, n);
    const float cut_e = expf(r.z(of_key(cut_key)));
    const unsigned cut_w = cut_key && cut_e >= r.min_p ? Row::weight(cut_e) : 0u;
    auto kept = [&](int i, unsigned& key) {                       // weight of an entry above the cut
        key = key_of(to_float(x[i]));
        if (key <= max(cut_key, kLowestKey)) return 0u;
        const float e = expf(r.z(of_key(key)));
        return e >= r.min_p ? Row::weight(e) : 0u;
    };
    {
        u64 mass = 0;
        unsigned ties = 0;
        for (int i = seg_begin + lane; i < seg_end; i += 32) {
            unsigned key;
            mass += kept(i, key);
            ties += key == cut_key;
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) { mass += __shfl_xor_sync(0xFFFFFFFFu, mass, d); ties += __shfl_xor_sync(0xFFFFFFFFu, ties, d); }
        if (lane == 0) { s.seg_mass[warp] = mass; s.seg_ties[warp] = ties; }
    }
    cluster.sync();
    // ---- the segment the drawn number falls into ----
    {
        const int segs = ctas * kSampleWarps;
        u64 mass = 0, upto;
        unsigned ties = 0, ties_upto;
        if (tid < segs) {
            mass = *cluster.map_shared_rank(&s.seg_mass[tid % kSampleWarps], tid / kSampleWarps);
            ties = *cluster.map_shared_rank(&s.seg_ties[tid % kSampleWarps], tid / kSampleWarps);
        }
        ties_upto = ties;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) { const unsigned a = __shfl_up_sync(0xFFFFFFFFu, ties_upto, d); if (lane >= d) ties_upto += a; }
        if (lane == 31) s.warp_count[warp] = ties_upto;
        __syncthreads();
        for (int w = 0; w < warp; ++w) ties_upto += s.warp_count[w];
        const unsigned ties_before = ties_upto - ties;
        const unsigned ties_kept = ties_before >= cut_ties ? 0u : min(ties, cut_ties - ties_before);
        mass += (u64)ties_kept * cut_w;
        upto = mass;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) { const u64 a = __shfl_up_sync(0xFFFFFFFFu, upto, d); if (lane >= d) upto += a; }
        if (lane == 31) s.warp_mass[warp] = upto;
        __syncthreads();
        u64 total = 0;
        for (int w = 0; w < kSampleWarps; ++w) { if (w == warp) upto += total; total += s.warp_mass[w]; }
        const float u = p.uniform[row];
        const unsigned part = u > 0.f ? min((unsigned)(u * 16777216.f), 0xFFFFFFu) : 0u;
        const u64 at = share(part, total);
        if (mass && upto - mass <= at && at < upto) {
            s.pick_seg = tid; s.pick_left = at - (upto - mass); s.pick_ties = ties_before; s.pick_total = total;
        }
        __syncthreads();
    }
    // ---- and the entry in it ----
    if (nothing) {
        if (rank == 0 && tid == 0) {
            if (p.wide) static_cast<long long*>(p.tokens)[row] = -1; else static_cast<int*>(p.tokens)[row] = -1;
            if (p.prob) p.prob[row] = 0.f;
        }
    } else if (s.pick_seg == (unsigned)(rank * kSampleWarps + warp)) {
        u64 left = s.pick_left;
        unsigned ties = s.pick_ties;
        for (int i0 = seg_begin; i0 < seg_end; i0 += 32) {
            const int i = i0 + lane;
            unsigned key = 0, w = 0;
            if (i < seg_end) w = kept(i, key);
            const unsigned same = __ballot_sync(0xFFFFFFFFu, i < seg_end && key == cut_key);
            if (i < seg_end && key == cut_key && ties + __popc(same & ((1u << lane) - 1u)) < cut_ties) w = cut_w;
            ties += __popc(same);
            u64 upto = w;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) { const u64 a = __shfl_up_sync(0xFFFFFFFFu, upto, d); if (lane >= d) upto += a; }
            const unsigned over = __ballot_sync(0xFFFFFFFFu, upto > left);
            if (over) {
                if (lane == __ffs(over) - 1) {
                    const long long token = begin + i;
                    if (p.wide) static_cast<long long*>(p.tokens)[row] = token; else static_cast<int*>(p.tokens)[row] = (int)token;
                    if (p.prob) p.prob[row] = (float)w / (float)s.pick_total;
                }
                break;
            }
            left -= __shfl_sync(0xFFFFFFFFu, upto, 31);
        }
    }
    cluster.sync();                                               // nobody leaves while its shared memory is read
}

template <typename T>
static cudaError_t sample_t(const SampleParams& p, int sms, cudaStream_t stream) {
    static SmemOptIn opt;
    // CTAs a row: as many as the machine has SMs for, and enough for a slice to fit the shared memory
    int ctas = 1;
    const size_t fixed = (sizeof(SampleShared) + 15) / 16 * 16 + 32, most = 227 * 1024;
    auto bytes = [&](int c) { return fixed + size_t(((p.vocab + c - 1) / c + 7) / 8 * 8) * sizeof(T); };
    while (ctas < kSampleCtas && (bytes(ctas) > most || p.vocab > kSampleSlice * ctas || (p.rows * ctas * 2 <= sms && p.vocab > 2048 * ctas))) ctas *= 2;
    const size_t smem = bytes(ctas);
    const cudaError_t e = ensure_dynamic_smem(k_sample<T>, smem, opt);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.rows * ctas)); cfg.blockDim = dim3(kSampleThreads); cfg.dynamicSmemBytes = smem; cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)ctas; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, k_sample<T>, p);
}

cudaError_t launch_sample(const SampleParams& p, int type, int sms, cudaStream_t stream) {
    return type == DST_F32 ? sample_t<float>(p, sms, stream) : sample_t<__nv_bfloat16>(p, sms, stream);
}

}  // namespace dst
