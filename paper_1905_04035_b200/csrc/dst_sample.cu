// One token per row of logits from a given uniform number, with temperature, top-k, top-p and min-p.
//
// The filters keep the entries above some value and the first few (in index order) of those equal to it, so a row needs
// that value and that count alone.  The weights are whole numbers (2^31 * exp, rounded), so every sum is exact whatever
// its order, and a row may be split in any way.
//
// Few candidates (top-k up to some hundred, or a short row): every thread's largest logit gives a bound that at least
// k logits reach; the few that do are collected, their values and their indices sorted, and all that follows is on that
// list: the row is read twice, with a few instructions an entry.
// Otherwise: a histogram over equal steps of the scaled logit finds the step in which top-k's count, or top-p's mass, is
// reached, finer histograms over the bits of the logit narrow the step down to one value, and a last pass sums what is
// kept in index order.
//
// A row belongs to a cluster of 1, 2, 4 or 8 CTAs with a slice of it each, joined through distributed shared memory.
//
// Bound by: the list's short dependent phases (one row of 33,708 fp32 logits: 9.2 us, of 327,680: 13; 512 rows of 65,536 in bf16:
// 39 us, of which their 67 MB need 10); without top-k by the instructions and shared-memory additions an entry costs in every pass
// over the row (512 x 65,536 bf16: top-p alone 182 to 195 us, as the logits fall, min-p alone 49 to 53, no filter 78; 64 x 327,680
// bf16: top-p alone 149, no filter 63).
#include <cooperative_groups.h>

#include "dst_tied.cuh"

namespace dst {
namespace cg = cooperative_groups;

typedef unsigned long long u64;
constexpr int kSampleThreads = 512;
constexpr int kSampleWarps = kSampleThreads / 32;
constexpr int kSampleCtas = 8;               // of a cluster, at most
constexpr int kBins = 2048;
constexpr int kListMost = 1024;              // candidates that are worked on as a list (twice the threads; a place in it has 10 bits)
constexpr int kListRank = 384;               // top-k for each CTA of a row up to which the threads' maxima bound it well
constexpr float kBinsPerZ = kBins / 22.25f;  // below z = -22.18 the weight rounds to zero (2^31 e^z < 1/2)
constexpr int kSampleSlice = 65536;          // entries a CTA takes, at most: its sums of 16-bit halves stay within 32 bits
constexpr unsigned kLowestKey = 0x007FFFFFu; // key of -infinity

// order-preserving bits of a float; equal floats (the two zeros) have equal keys, NaN counts as -infinity
__device__ __forceinline__ unsigned key_of(float x) {
    x = x == x ? x + 0.f : -INFINITY;
    const unsigned b = __float_as_uint(x);
    return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float of_key(unsigned k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xFFFFFFFFu)); }

// What turns a logit into its weight, where the largest logit is finite and 1 / temperature too (z is then 0 at the largest).
struct Weigh {
    float top, inv_t, min_p;
    __device__ __forceinline__ float z(float x) const { return __fmul_rn(x - top, inv_t); }
    __device__ __forceinline__ float e(unsigned key) const { return expf(z(of_key(key))); }
    // 2^31 e, rounded.  Below 2^23 by the bits of a sum with 2^23, which saves the conversion (a quarter-rate instruction,
    // as the exponential is); a NaN gives 0
    __device__ __forceinline__ static unsigned weight(float e) {
        const float v = e * 2147483648.f;
        return v < 8388608.f ? __float_as_uint(v + 8388608.f) & 0x7FFFFFu : __float2uint_rn(v);
    }
};

// part / 2^24 of total, rounded down
__device__ __forceinline__ u64 share(unsigned part, u64 total) {
    return (u64)part * (total >> 24) + (((u64)part * (total & 0xFFFFFFu)) >> 24);
}

// The slice's vectors of 16 bytes; the first and the last may lie partly outside the row and are read entry by entry.
template <typename T> struct Vec {
    static constexpr int kN = 16 / sizeof(T);
    uint4 v;
    __device__ __forceinline__ float get(int i) const;
    __device__ __forceinline__ float largest() const;                // (the maximum of a NaN and a number is the number)
    __device__ __forceinline__ void raise(const Vec& o);            // to the larger, entry by entry
    static __device__ __forceinline__ Vec nothing();
};
template <> __device__ __forceinline__ float Vec<float>::get(int i) const { return __uint_as_float(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w); }
template <> __device__ __forceinline__ float Vec<__nv_bfloat16>::get(int i) const {
    const unsigned w = i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w;
    return __uint_as_float(i & 1 ? w & 0xFFFF0000u : w << 16);
}
template <> __device__ __forceinline__ Vec<float> Vec<float>::nothing() { return Vec{make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u)}; }
template <> __device__ __forceinline__ Vec<__nv_bfloat16> Vec<__nv_bfloat16>::nothing() { return Vec{make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u)}; }
template <> __device__ __forceinline__ void Vec<float>::raise(const Vec& o) {
    v.x = __float_as_uint(fmaxf(get(0), o.get(0))); v.y = __float_as_uint(fmaxf(get(1), o.get(1)));
    v.z = __float_as_uint(fmaxf(get(2), o.get(2))); v.w = __float_as_uint(fmaxf(get(3), o.get(3)));
}
template <> __device__ __forceinline__ void Vec<__nv_bfloat16>::raise(const Vec& o) {
    __nv_bfloat162* a = reinterpret_cast<__nv_bfloat162*>(&v);
    const __nv_bfloat162* b = reinterpret_cast<const __nv_bfloat162*>(&o.v);
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = __hmax2(a[i], b[i]);
}
template <> __device__ __forceinline__ float Vec<float>::largest() const { return fmaxf(fmaxf(get(0), get(1)), fmaxf(get(2), get(3))); }
template <> __device__ __forceinline__ float Vec<__nv_bfloat16>::largest() const {
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
    const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    return fmaxf(__low2float(m), __high2float(m));
}
template <typename T> __device__ __forceinline__ T lowest();
template <> __device__ __forceinline__ float lowest<float>() { return -INFINITY; }
template <> __device__ __forceinline__ __nv_bfloat16 lowest<__nv_bfloat16>() { return __ushort_as_bfloat16(0xFF80); }

template <typename T> struct Slice {
    const T* base;                           // 16-byte aligned, at or before the row's first entry
    int skew, vocab;                         // entries between base and the row; vector v holds entries v * kN - skew ...
    int begin, end;                          // this warp's vectors
    __device__ __forceinline__ Vec<T> load(int v) const {
        constexpr int kN = Vec<T>::kN;
        Vec<T> r;
        const int first = v * kN - skew;
        if (first >= 0 && first + kN <= vocab && v < end) r.v = *reinterpret_cast<const uint4*>(base + (long long)v * kN);
        else {
            T x[kN];
#pragma unroll
            for (int i = 0; i < kN; ++i) x[i] = first + i >= 0 && first + i < vocab && v < end ? base[(long long)v * kN + i] : lowest<T>();
            r.v = *reinterpret_cast<const uint4*>(x);
        }
        return r;
    }
    // f(four vectors, 32 apart, the first one's number) for the lane's vectors; what lies outside is -infinity, and f may
    // use the whole warp
    template <typename F> __device__ __forceinline__ void groups(F f) const {
        constexpr int kN = Vec<T>::kN;
        for (int v0 = begin; v0 < end; v0 += 128) {
            const int v = v0 + lane_id();
            Vec<T> x[4];
            if (v0 * kN >= skew && v0 + 128 <= end && (v0 + 128) * kN - skew <= vocab) {
                const T* const from = base + (long long)v * kN;
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i].v = *reinterpret_cast<const uint4*>(from + i * 32 * kN);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = load(v + i * 32);
            }
            f(x, v);
        }
    }
    // f(vector, its number), one at a time
    template <typename F> __device__ __forceinline__ void each(F f) const {
        groups([&](const Vec<T> (&x)[4], int v) {
#pragma unroll
            for (int i = 0; i < 4; ++i) f(x[i], v + i * 32);
        });
    }
};

struct SampleShared {
    union {
        struct { unsigned count[kBins], low[kBins], high[kBins], joined_count[kBins]; u64 joined_mass[kBins]; };   // the mass in halves of 16 bits
        struct { unsigned key[kListMost], order[kListMost], bins[kSampleThreads]; uint2 sorted[kListMost], spare[kListMost]; };
    };
    u64 warp_mass[kSampleWarps], seg_mass[kSampleWarps];
    unsigned warp_count[kSampleWarps], seg_ties[kSampleWarps], warp_key[kSampleWarps], warp_low[kSampleWarps];
    unsigned top_key, bound, candidates;
    unsigned hit_bin, hit_count_above, pick_seg, pick_ties, cut_key;
    u64 hit_mass_above, pick_left, pick_total;
};

__device__ __forceinline__ void warp_scan(unsigned& x) {
#pragma unroll
    for (int d = 1; d < 32; d *= 2) { const unsigned a = __shfl_up_sync(0xFFFFFFFFu, x, d); if (lane_id() >= d) x += a; }
}
__device__ __forceinline__ void warp_scan(u64& x) {
#pragma unroll
    for (int d = 1; d < 32; d *= 2) { const u64 a = __shfl_up_sync(0xFFFFFFFFu, x, d); if (lane_id() >= d) x += a; }
}
// inclusive sums over the CTA's threads, and the total; `part` is a word a warp of shared memory that is free
template <typename N> __device__ __forceinline__ N cta_scan(N& x, N* part) {
    warp_scan(x);
    if (lane_id() == 31) part[warp_id()] = x;
    __syncthreads();
    N before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kSampleWarps; ++w) { const N p = part[w]; if (w < warp_id()) before += p; total += p; }
    x += before;
    __syncthreads();
    return total;
}

// Where the running count (by_mass: mass) over the joined bins first reaches `need`: the bin, and what is above it.
// `need` is at most the sum (0: no bin is looked for).
__device__ void find_bin(SampleShared& s, u64 need, bool by_mass, unsigned* total = nullptr, u64* total_mass = nullptr) {
    constexpr int kPer = kBins / kSampleThreads;
    const int first = threadIdx.x * kPer;
    unsigned c[kPer], n = 0;
    u64 m[kPer], mass = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) { c[i] = s.joined_count[first + i]; m[i] = s.joined_mass[first + i]; n += c[i]; mass += m[i]; }
    unsigned n_before = n;
    u64 mass_before = mass;
    const unsigned all = cta_scan(n_before, s.warp_count);
    const u64 all_mass = cta_scan(mass_before, s.warp_mass);
    if (total) { *total = all; *total_mass = all_mass; }
    n_before -= n; mass_before -= mass;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const u64 before = by_mass ? mass_before : n_before, here = by_mass ? m[i] : c[i];
        if (before < need && need <= before + here) { s.hit_bin = first + i; s.hit_count_above = n_before; s.hit_mass_above = mass_before; }
        n_before += c[i]; mass_before += m[i];
    }
    __syncthreads();
}

template <typename T>
__global__ void __launch_bounds__(kSampleThreads, 2) k_sample(const __grid_constant__ SampleParams p) {
    extern __shared__ __align__(16) unsigned char dyn[];
    SampleShared& s = *reinterpret_cast<SampleShared*>(dyn);
    cg::cluster_group cluster = cg::this_cluster();
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const long long row = blockIdx.x / ctas;
    const int tid = threadIdx.x, lane = lane_id(), warp = warp_id();
    constexpr int kN = Vec<T>::kN;
    pdl_trigger();
    pdl_wait();

    const T* const logits = static_cast<const T*>(p.logits) + row * p.ld;
    Slice<T> x;
    x.skew = (int)((reinterpret_cast<uintptr_t>(logits) & 15u) / sizeof(T));
    x.base = logits - x.skew;
    x.vocab = p.vocab;
    {   // consecutive vectors for a CTA, and for a warp in it
        const int all = (x.skew + p.vocab + kN - 1) / kN, share = (all + ctas * kSampleWarps - 1) / (ctas * kSampleWarps);
        x.begin = min((rank * kSampleWarps + warp) * share, all);
        x.end = min(x.begin + share, all);
    }
    const float t = p.temperature ? p.temperature[row] : 1.f;
    int k = p.top_k ? p.top_k[row] : 0;
    if (k <= 0 || k >= p.vocab) k = 0;
    const float top_p = p.top_p ? p.top_p[row] : 1.f;
    const bool by_mass = top_p < 1.f;
    const unsigned top_part = top_p > 0.f ? (unsigned)(fminf(top_p, 1.f) * 16777216.f) : 0u;
    const float u = p.uniform[row];
    const unsigned part = u > 0.f ? min((unsigned)(fminf(u, 1.f) * 16777216.f), 0xFFFFFFu) : 0u;
    auto sync = [&] { if (ctas == 1) __syncthreads(); else cluster.sync(); };
    auto answer = [&](long long token, float prob) {
        if (p.wide) static_cast<long long*>(p.tokens)[row] = token; else static_cast<int*>(p.tokens)[row] = (int)token;
        if (p.prob) p.prob[row] = prob;
    };

    // ---- the largest logit; every thread's own, for the bound below ----
    Vec<T> most = Vec<T>::nothing();
    x.each([&](const Vec<T>& v, int) { most.raise(v); });
    const float mine = fmaxf(most.largest(), -INFINITY);
    const unsigned my_key = key_of(mine);
    const unsigned wide_top = __reduce_max_sync(0xFFFFFFFFu, my_key);
    const unsigned wide_low = __reduce_min_sync(0xFFFFFFFFu, my_key > kLowestKey ? my_key : 0xFFFFFFFFu);
    if (lane == 0) { s.warp_key[warp] = wide_top; s.warp_low[warp] = wide_low; }
    s.bins[tid] = 0;
    __syncthreads();
    unsigned top_key = 0, low_key = 0xFFFFFFFFu;
#pragma unroll
    for (int w = 0; w < kSampleWarps; ++w) { top_key = max(top_key, s.warp_key[w]); low_key = min(low_key, s.warp_low[w]); }
    // ---- few candidates: a bound that at least ceil(k / ctas) of this CTA's threads reach; the least of the CTAs' bounds
    //      is reached by k logits of the row.  It is the lower edge of a bin of the threads' maxima: every warp finds it
    //      for itself ----
    const bool short_row = p.vocab <= kListMost;
    bool list = short_row ? k || by_mass : k > 0 && k <= kListRank * ctas;
    unsigned edge = kLowestKey + 1;
    if (list && !short_row) {
        const unsigned want = (unsigned)((k + ctas - 1) / ctas);
        const float hi = of_key(top_key), lo = of_key(low_key);
        float per = hi > lo && hi - lo < INFINITY ? (kSampleThreads - 1) / (hi - lo) : 0.f;
        if (!(per < INFINITY)) per = 0.f;                       // maxima so close together that the bins have no width: one bin
        if (my_key > kLowestKey) atomicAdd(&s.bins[per > 0.f ? min((unsigned)((hi - mine) * per), (unsigned)kSampleThreads - 1) : 0u], 1u);
        __syncthreads();
        constexpr int kPer = kSampleThreads / 32;
        unsigned c[kPer], sum = 0, upto;
#pragma unroll
        for (int i = 0; i < kPer; i += 4) {
            const uint4 four = *reinterpret_cast<const uint4*>(&s.bins[lane * kPer + i]);
            c[i] = four.x; c[i + 1] = four.y; c[i + 2] = four.z; c[i + 3] = four.w;
            sum += four.x + four.y + four.z + four.w;
        }
        upto = sum;
        warp_scan(upto);
        const unsigned reached = __ballot_sync(0xFFFFFFFFu, upto >= want);
        if (reached) {                                          // (otherwise fewer threads than that have anything: no bound)
            int bin = lane * kPer;
            unsigned before = upto - sum;
#pragma unroll
            for (int i = 0; i < kPer; ++i) { before += c[i]; bin += before < want; }
            bin = __shfl_sync(0xFFFFFFFFu, bin, __ffs(reached) - 1);
            // a little lower than the roundings of the bin number can move the edge; with one bin: the least of the maxima
            edge = per > 0.f ? max(key_of(__fsub_rd(hi, (float)(bin + 1) / per * (1.f + 0x1p-20f))), kLowestKey + 1) : low_key;
        }
    }
    if (tid == 0) { s.candidates = 0; s.top_key = top_key; s.bound = edge; }
    sync();
    unsigned bound = edge;
    if (ctas > 1) {                                             // every warp asks all CTAs at once
        bound = 0xFFFFFFFFu;
        if (lane < ctas) { top_key = *cluster.map_shared_rank(&s.top_key, lane); bound = *cluster.map_shared_rank(&s.bound, lane); }
        top_key = __reduce_max_sync(0xFFFFFFFFu, top_key);
        bound = __reduce_min_sync(0xFFFFFFFFu, bound);
    }

    Weigh g;
    g.top = of_key(top_key);
    g.inv_t = 1.f / t;
    g.min_p = p.min_p ? fminf(p.min_p[row], 1.f) : 0.f;
    if (top_key <= kLowestKey) {                                // nothing left (everybody sees the same)
        if (rank == 0 && tid == 0) answer(-1, 0.f);
        sync();
        return;
    }
    // All weight on the entries equal to the largest: only the first of them for a temperature of 0; all of them where the
    // largest is infinite or the temperature next to nothing (their differences have no finite z)
    const bool greedy = !(t > 0.f) || k == 1, equal_only = greedy || !(g.top < INFINITY) || !(g.inv_t < INFINITY);
    if (equal_only) list = false;

    // ---- the candidates, in the first CTA's list: their keys, and their indices with their places in it ----
    if (list) {
        const float least = of_key(bound);
        SampleShared* const first = cluster.map_shared_rank(&s, 0);
        x.groups([&](const Vec<T> (&v)[4], int number) {
            unsigned hits = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (v[j].largest() >= least)
#pragma unroll
                    for (int i = 0; i < kN; ++i) hits |= (v[j].get(i) >= least ? 1u : 0u) << (j * kN + i);
            if (!hits) return;
            unsigned to = atomicAdd(&first->candidates, (unsigned)__popc(hits));
            for (; hits; hits &= hits - 1, ++to) {
                const int bit = __ffs(hits) - 1, index = (number + bit / kN * 32) * kN + bit % kN - x.skew;
                if (to < kListMost) { first->key[to] = key_of(to_float(logits[index])); first->order[to] = (unsigned)index << 10 | to; }
            }
        });
        sync();
        const unsigned total = first->candidates;
        list = total <= kListMost;
        if (list) {
            if (rank != 0) return;                              // the rest is the first CTA's, with nobody else's memory
            const int count = (int)total;
            // Keys in descending order, indices (with places) in ascending order, entry i of both in register i / 512 of
            // thread i % 512: a bitonic network for both at once.  Stretches of 32 are put in order by shuffles alone;
            // only wider steps pass through shared memory, and warps without entries have no part in it.
            const int halves = count > kSampleThreads ? 2 : 1;
            int size = 32;
            while (size < count) size *= 2;
            unsigned key[2], order[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int i = r * kSampleThreads + tid;
                key[r] = i < count ? s.key[i] : 0u;
                order[r] = i < count ? s.order[i] : 0xFFFFFFFFu;
            }
            // the larger key and the smaller index stay where `larger` says
            auto exchange = [](unsigned& k0, unsigned& o0, unsigned k1, unsigned o1, bool larger) {
                k0 = larger ? max(k0, k1) : min(k0, k1);
                o0 = larger ? min(o0, o1) : max(o0, o1);
            };
            if (warp * 32 < size) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    if (r >= halves) break;
                    const int i = r * kSampleThreads + tid;
#pragma unroll
                    for (int width = 2; width <= 32; width *= 2)
#pragma unroll
                        for (int step = width / 2; step > 0; step /= 2)
                            exchange(key[r], order[r], __shfl_xor_sync(0xFFFFFFFFu, key[r], step), __shfl_xor_sync(0xFFFFFFFFu, order[r], step),
                                     ((i & step) == 0) == ((i & width) == 0));
                }
                int buffer = 0;
                const int threads = min(size, kSampleThreads);
#pragma unroll 1
                for (int width = 64; width <= size; width *= 2) {
#pragma unroll 1
                    for (int step = width / 2; step >= 32; step /= 2) {
                        if (step == kSampleThreads) {               // the two registers of a thread
                            const unsigned k1 = key[1], o1 = order[1];
                            exchange(key[1], order[1], key[0], order[0], false);
                            exchange(key[0], order[0], k1, o1, true);
                            continue;
                        }
                        uint2* const at = buffer ? s.spare : s.sorted;
                        buffer ^= 1;                                // the next exchange writes elsewhere: no second wait
#pragma unroll
                        for (int r = 0; r < 2; ++r) if (r < halves) at[r * kSampleThreads + tid] = make_uint2(key[r], order[r]);
                        asm volatile("bar.sync 1, %0;" ::"r"(threads) : "memory");
#pragma unroll
                        for (int r = 0; r < 2; ++r)
                            if (r < halves) {
                                const int i = r * kSampleThreads + tid;
                                const uint2 other = at[i ^ step];
                                exchange(key[r], order[r], other.x, other.y, ((i & step) == 0) == ((i & width) == 0));
                            }
                    }
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        if (r >= halves) break;
                        const bool descending = ((r * kSampleThreads + tid) & width) == 0;
#pragma unroll
                        for (int step = 16; step > 0; step /= 2)
                            exchange(key[r], order[r], __shfl_xor_sync(0xFFFFFFFFu, key[r], step), __shfl_xor_sync(0xFFFFFFFFu, order[r], step),
                                     ((tid & step) == 0) == descending);
                    }
                }
            }
            // how many of them the filters keep, and from that the value they keep down to and the count at it
            const int limit = k ? min(k, count) : count;
            int kept = limit;
            if (by_mass) {
                u64 w[2] = {0, 0}, upto[2], mass = 0;
#pragma unroll
                for (int r = 0; r < 2; ++r)
                    if (r < halves) {
                        if (r * kSampleThreads + tid < limit) w[r] = Weigh::weight(g.e(key[r]));
                        upto[r] = w[r];
                        const u64 all = cta_scan(upto[r], s.warp_mass);
                        upto[r] += mass - w[r];
                        mass += all;
                    }
                const u64 most = max(share(top_part, mass), (u64)1);
                kept = 0;
#pragma unroll
                for (int r = 0; r < 2; ++r) if (r < halves) kept += __syncthreads_count(r * kSampleThreads + tid < limit && upto[r] < most);
            }
#pragma unroll
            for (int r = 0; r < 2; ++r) if (r * kSampleThreads + tid == kept - 1) s.cut_key = key[r];
            __syncthreads();
            const unsigned cut = s.cut_key;
            unsigned ties = 0, same_all = 0;
#pragma unroll
            for (int r = 0; r < 2; ++r)
                if (r < halves) {
                    ties += __syncthreads_count(r * kSampleThreads + tid < kept && key[r] == cut);
                    same_all += __syncthreads_count(key[r] == cut);
                }
            // the draw, in index order
            u64 w[2] = {0, 0}, upto[2] = {0, 0}, sum = 0;
            unsigned same_before = 0;
#pragma unroll
            for (int r = 0; r < 2; ++r)
                if (r < halves) {
                    const unsigned mine_key = r * kSampleThreads + tid < count ? s.key[order[r] & 1023u] : 0u;
                    bool take = mine_key >= cut;
                    if (ties < same_all) {                          // only the first ones of those equal to the cut
                        unsigned same = mine_key == cut;
                        const unsigned here = same;
                        const unsigned all = cta_scan(same, s.warp_count);
                        if (here && same_before + same > ties) take = false;
                        same_before += all;
                    }
                    const float e = g.e(mine_key);
                    if (take && e >= g.min_p) w[r] = Weigh::weight(e);
                    upto[r] = w[r];
                    const u64 all = cta_scan(upto[r], s.warp_mass);
                    upto[r] += sum;
                    sum += all;
                }
            const u64 drawn = share(part, sum);
#pragma unroll
            for (int r = 0; r < 2; ++r)
                if (upto[r] - w[r] <= drawn && drawn < upto[r]) answer(order[r] >> 10, (float)w[r] / (float)sum);
            if (ctas > 1) cluster.sync();                       // others may still be reading the number of candidates; those that left count as arrived
            return;
        }
    }

    // ---- the value the filters keep down to, and how many of the entries equal to it ----
    unsigned cut_key = 0, cut_ties = 0xFFFFFFFFu;
    if (equal_only) {
        cut_key = top_key;
        cut_ties = greedy ? 1u : k ? (unsigned)k : 0xFFFFFFFFu;
        if (!greedy && by_mass) {
            unsigned same = 0;
            x.each([&](const Vec<T>& v, int) {
#pragma unroll
                for (int i = 0; i < kN; ++i) same += v.get(i) == g.top;
            });
            same = __reduce_add_sync(0xFFFFFFFFu, same);
            if (lane == 0) s.seg_ties[warp] = same;
            sync();
            u64 all = 0;
            for (int c = 0; c < ctas * kSampleWarps; ++c) all += *cluster.map_shared_rank(&s.seg_ties[c % kSampleWarps], c / kSampleWarps);
            sync();
            const u64 one = 1ull << 31, upto = max(share(top_part, min(all, (u64)cut_ties) * one), (u64)1);
            cut_ties = (unsigned)min((u64)cut_ties, (upto + one - 1) / one);
        }
    } else if (k || by_mass) {
        constexpr int kShift = sizeof(T) == 2 ? 16 : 0;          // bf16 logits differ in the upper half of the key only
        // One round: a histogram of the whole row over the steps of z (coarse), or of one such bin's entries over the bits
        // of their keys below `hi`; joined; and the bin in which the sum reaches what is still wanted.  First top-k's
        // count is narrowed down to one key, then top-p's mass.
        bool for_k = k > 0, coarse = true, first = true;
        unsigned bin = 0, hi = 0, lo = 0, count_above = 0;
        int shift = 0;
        u64 mass_above = 0, need = 0, kept_mass = 0;
        float floor_of = -INFINITY;                               // no entry of the bin lies below it
        for (;;) {
            for (int i = tid; i < kBins; i += kSampleThreads) { s.count[i] = 0; s.low[i] = 0; s.high[i] = 0; }
            __syncthreads();
            x.each([&](const Vec<T>& v, int) {
                if (!(v.largest() >= floor_of)) return;
#pragma unroll
                for (int i = 0; i < kN; ++i) {
                    const float f = v.get(i), z = g.z(f);
                    // to the nearest whole number of steps, by the bits of a sum with 2^23 (anything where the weight is 0)
                    unsigned b = min(__float_as_uint(__fmaf_rn(z, -kBinsPerZ, 8388608.f)) & 0x7FFFFFu, kBins - 1u);
                    if (!coarse) {                                // few are in the bin: no exponential for the others
                        const unsigned key = key_of(f) >> kShift;
                        if (b != bin || key > hi || (hi - key) >> shift >= kBins) continue;
                        b = (hi - key) >> shift;
                    }
                    const unsigned w = Weigh::weight(expf(z));
                    if (w) {
                        if (k) atomicAdd(&s.count[b], 1u);
                        atomicAdd(&s.low[b], w & 0xFFFFu);
                        if (w >> 16) atomicAdd(&s.high[b], w >> 16);
                    }
                }
            });
            sync();
            const int share_bins = kBins / ctas;
            for (int i = tid; i < share_bins; i += kSampleThreads) {
                const int at = rank * share_bins + i;
                unsigned n = 0;
                u64 m = 0;
                for (int c = 0; c < ctas; ++c) {
                    n += *cluster.map_shared_rank(&s.count[at], c);
                    m += *cluster.map_shared_rank(&s.low[at], c) + ((u64)*cluster.map_shared_rank(&s.high[at], c) << 16);
                }
                for (int c = 0; c < ctas; ++c) {
                    *cluster.map_shared_rank(&s.joined_count[at], c) = n;
                    *cluster.map_shared_rank(&s.joined_mass[at], c) = m;
                }
            }
            sync();
            if (first) {
                first = false;
                unsigned all;
                find_bin(s, 0, false, &all, &kept_mass);          // the sums alone
                if ((unsigned)k >= all) for_k = false;            // fewer weights above zero than k: k keeps them all
                if (!for_k && !by_mass) break;
                need = for_k ? (u64)k : max(share(top_part, kept_mass), (u64)1);
            }
            find_bin(s, need - (for_k ? (u64)count_above : mass_above), !for_k);
            if (coarse) {
                bin = s.hit_bin; count_above = s.hit_count_above; mass_above = s.hit_mass_above;
                // bounds of the bin's logits, a little wider than the roundings of z and of the bin number can move them; in 64
                // bits, as the width of a bin in logits is no fp32 number for temperatures below 3e-37
                const double step = 1. / ((double)kBinsPerZ * g.inv_t), near = bin ? (bin - 0.5) * step * (1. - 0x1p-19) : 0.,
                             far = (bin + 0.5) * step * (1. + 0x1p-19);
                floor_of = bin == kBins - 1 ? -INFINITY : __double2float_rd(__dsub_rd(g.top, far));
                hi = min(top_key, key_of(__double2float_ru(__dsub_ru(g.top, near)))) >> kShift;
                lo = key_of(floor_of) >> kShift;
                coarse = false;
            } else {
                count_above += s.hit_count_above; mass_above += s.hit_mass_above;
                hi -= s.hit_bin << shift;
                const unsigned low = hi - ((1u << shift) - 1u);
                lo = low > hi || low < lo ? lo : low;
                if (shift == 0) {                                 // one key
                    const unsigned key = kShift == 0 ? hi : hi << kShift | (hi >> 15 ? 0u : 0xFFFFu);   // a negative number's bits are inverted
                    const unsigned w = Weigh::weight(g.e(key));
                    if (for_k) {
                        cut_key = key; cut_ties = k - count_above;
                        kept_mass = mass_above + (u64)cut_ties * w;
                        if (!by_mass) break;
                        for_k = false; coarse = true;
                        count_above = 0; mass_above = 0; floor_of = -INFINITY;
                        need = max(share(top_part, kept_mass), (u64)1);
                        __syncthreads();
                        continue;
                    }
                    const u64 ties = (need - mass_above + w - 1) / w;
                    if (key > cut_key) { cut_key = key; cut_ties = (unsigned)min(ties, (u64)0xFFFFFFFFu); }
                    else cut_ties = (unsigned)min(ties, (u64)cut_ties);
                    break;
                }
            }
            shift = 0;
            while ((hi - lo) >> shift >= kBins) ++shift;
            __syncthreads();                                      // everybody has read s.hit_*
        }
    }

    // ---- kept mass of every warp's vectors (consecutive entries), in index order ----
    const float cut_e = equal_only ? 1.f : g.e(cut_key), least = cut_key > kLowestKey ? of_key(cut_key) : -INFINITY;
    const unsigned cut_w = cut_key && cut_e >= g.min_p ? Weigh::weight(cut_e) : 0u;
    // nothing below `skip` is kept: the cut, or what min-p leaves at most, taken a little lower than its logarithm can be off
    // (where only the largest count, the cut is the largest, which min-p never takes, and inv_t may be anything)
    const float skip = equal_only || !(g.min_p > 0.f) ? least : fmaxf(least, g.top + (logf(g.min_p) - 1e-3f) / g.inv_t * 1.0001f - fabsf(g.top) * 1e-6f);
    auto kept = [&](float f) {                                    // weight of an entry above the cut
        const float e = expf(g.z(f));
        return f > least && e >= g.min_p ? Weigh::weight(e) : 0u;
    };
    {
        u64 mass = 0;
        unsigned ties = 0;
        x.each([&](const Vec<T>& v, int) {
            if (v.largest() < skip) return;
            unsigned small = 0;                                   // eight weights below 2^23 stay within 32 bits
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                const unsigned w = kept(v.get(i));
                if (w < 8388608u) small += w; else mass += w;
                ties += v.get(i) == least;
            }
            mass += small;
        });
#pragma unroll
        for (int d = 16; d; d >>= 1) { mass += __shfl_xor_sync(0xFFFFFFFFu, mass, d); ties += __shfl_xor_sync(0xFFFFFFFFu, ties, d); }
        if (lane == 0) { s.seg_mass[warp] = mass; s.seg_ties[warp] = cut_key ? ties : 0u; }
    }
    sync();
    // ---- the warp whose entries the drawn number falls into ----
    {
        u64 mass = 0, upto;
        unsigned ties = 0, ties_before;
        if (tid < ctas * kSampleWarps) {
            mass = *cluster.map_shared_rank(&s.seg_mass[tid % kSampleWarps], tid / kSampleWarps);
            ties = *cluster.map_shared_rank(&s.seg_ties[tid % kSampleWarps], tid / kSampleWarps);
        }
        ties_before = ties;
        cta_scan(ties_before, s.warp_count);
        ties_before -= ties;
        mass += (u64)(ties_before >= cut_ties ? 0u : min(ties, cut_ties - ties_before)) * cut_w;
        upto = mass;
        const u64 total = cta_scan(upto, s.warp_mass), at = share(part, total);
        if (upto - mass <= at && at < upto) { s.pick_seg = tid; s.pick_left = at - (upto - mass); s.pick_ties = ties_before; s.pick_total = total; }
        __syncthreads();
    }
    // ---- and the entry among them ----
    if (s.pick_seg == (unsigned)(rank * kSampleWarps + warp)) {
        u64 left = s.pick_left;
        unsigned ties = s.pick_ties;
        bool found = false;
        x.each([&](const Vec<T>& v, int number) {
            if (found || __all_sync(0xFFFFFFFFu, v.largest() < skip)) return;
            unsigned same = 0, w[kN];
            if (cut_key)
#pragma unroll
                for (int i = 0; i < kN; ++i) same += v.get(i) == least;
            unsigned same_upto = same;
            warp_scan(same_upto);
            unsigned rank_of = ties + same_upto - same;
            u64 mass = 0;
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                w[i] = kept(v.get(i));
                if (cut_key && v.get(i) == least && rank_of++ < cut_ties) w[i] = cut_w;
                mass += w[i];
            }
            ties += __shfl_sync(0xFFFFFFFFu, same_upto, 31);
            u64 upto = mass;
            warp_scan(upto);
            const unsigned over = __ballot_sync(0xFFFFFFFFu, upto > left);
            if (over) {
                found = true;
                if (lane == __ffs(over) - 1) {
                    u64 run = upto - mass;
                    bool open = true;
#pragma unroll
                    for (int i = 0; i < kN; ++i) {
                        run += w[i];
                        if (open && run > left) { open = false; answer((long long)number * kN - x.skew + i, (float)w[i] / (float)s.pick_total); }
                    }
                }
                return;
            }
            left -= __shfl_sync(0xFFFFFFFFu, upto, 31);
        });
    }
    sync();                                               // nobody leaves while its shared memory is read
}

template <typename T>
static cudaError_t sample_t(const SampleParams& p, int sms, cudaStream_t stream) {
    static SmemOptIn opt;
    // CTAs a row: as many as fill the machine without a second round of CTAs (two share an SM), each with 2048 entries at least
    int ctas = 1;
    while (ctas < kSampleCtas && p.rows * ctas * 2 <= sms && p.vocab > 2048 * ctas) ctas *= 2;
    auto slice = [&](int c) {                                    // the most entries of a CTA
        const int n = Vec<T>::kN, vectors = (p.vocab + 2 * n - 2) / n;
        return c == 1 ? p.vocab : (vectors + c * kSampleWarps - 1) / (c * kSampleWarps) * kSampleWarps * n;
    };
    while (slice(ctas) > kSampleSlice) ctas *= 2;
    const cudaError_t e = ensure_dynamic_smem(k_sample<T>, sizeof(SampleShared), opt);
    if (e != cudaSuccess) return e;
    static std::atomic<bool> carved[64];                         // two CTAs share an SM's shared memory only if it is told to be that large
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64 || !carved[dev].load()) {
        const cudaError_t c = cudaFuncSetAttribute(k_sample<T>, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
        if (c != cudaSuccess) return c;
        if (dev >= 0 && dev < 64) carved[dev].store(true);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.rows * ctas)); cfg.blockDim = dim3(kSampleThreads); cfg.dynamicSmemBytes = sizeof(SampleShared); cfg.stream = stream;
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
