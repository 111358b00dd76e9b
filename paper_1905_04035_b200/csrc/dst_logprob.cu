// Log probabilities of given tokens, entropy and the most likely tokens of rows of logits, and the gradient through them.
//
// With m the largest logit of some part of a row, a part is described by three numbers: m, r = sum exp(z) - 1 (the largest
// logit's own 1 apart, so that what the others add is not rounded against it) and t = sum exp(z) z, z = scale (x - m) <= 0.
// Two parts join by multiplying the one with the smaller m by exp(scale (m - M)) and moving its z's by the same
// difference; a thread's logits, the lanes of a warp, the warps of a CTA and the CTAs of a row join in that way, and each
// is read once.  Then log p = z - log1p(r) and the entropy is log1p(r) - t / (1 + r): a sum of two terms of one sign.
//
// A row belongs to a cluster of 1, 2, 4 or 8 CTAs, joined through distributed shared memory, that stream their parts or, where a part is four vectors of
// 16 bytes a thread, keep it in registers for the gradient and the alternatives (k_logprob); for the gradient of many long rows a CTA keeps a whole
// row in shared memory (k_logprob_ring).
//
// Alternatives: the n-th largest of the maxima of 32 or 64 groups of logits is a bound that n logits reach at least and few more than n
// do; those are collected and ranked by counting, and the CTAs of a row place their own n among all.  Where too many reach it (equal
// logits), n rounds look for the next largest instead, each of which reads the row again (all logits equal: 512 x 65,536 bf16 with five alternatives
// 251 us, with twenty 787, where others take 19 and 24; 4096 x 33,708 bf16 with five 1230 and 84; one row of 33,708 fp32 with twenty 31 and 6.6).
//
// Measured: forward 8111 x 33,708 fp32 162 us (6750 GB/s: the rate of reading), 4096 x 33,708 bf16 52 us (5270 GB/s; the exponential unit
// and the issue slots are 67 % busy), 512 x 65,536 bf16 16 us and 19.4 with five alternatives, one row of 33,708 fp32 3.7 us and 6.6 with
// twenty; loss and gradient of 4096 x 33,708 bf16 120 us (4600 GB/s; two exponentials a logit), of 8111 x 33,708 fp32 400 us (5470 GB/s);
// the gradient alone 99 us (5580) and 348 (6290).
#include <cooperative_groups.h>

#include <type_traits>

#include "dst_async.cuh"
#include "dst_step.cuh"

namespace dst {
namespace cg = cooperative_groups;

typedef unsigned long long u64;
constexpr int kLpThreads = 512;              // of a CTA, at most
constexpr int kLpStream = 256;               // ... where it streams its part
constexpr int kLpWarps = kLpThreads / 32;
constexpr int kLpVecs = 4;                   // vectors a thread takes at a time
constexpr int kLpCtas = 8;                   // of a row, at most
constexpr int kLpList = 512;                 // candidates that are ranked
constexpr unsigned kKeyLowest = 0x007FFFFFu; // key of -infinity
constexpr float kLn2 = 0.693147180559945309f, kLog2e = 1.44269504088896341f;
constexpr float kLeastZ = -1000.f;           // in place of z = -infinity (and of anything below): its exponential is zero, and zero times it too

__device__ __forceinline__ float exp2_fast(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float max_nan(float a, float b) { float y; asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b)); return y; }
__device__ __forceinline__ float warp_max(float x) { float y; asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x)); return y; }

// two floats at a time
typedef unsigned long long Two;
__device__ __forceinline__ Two two(float x, float y) { Two r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y)); return r; }
__device__ __forceinline__ void apart(Two a, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(a)); }
__device__ __forceinline__ Two add2(Two a, Two b) { Two r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ Two mul2(Two a, Two b) { Two r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) { Two r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }

// order-preserving bits of a float; the two zeros have the same, NaN counts as -infinity
__device__ __forceinline__ unsigned order_key(float x) {
    x = x == x ? x + 0.f : -INFINITY;
    const unsigned b = __float_as_uint(x);
    return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float of_order_key(unsigned k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xFFFFFFFFu)); }

template <typename T> struct Logits8;        // a vector of 16 bytes
template <> struct Logits8<float> {
    static constexpr int kN = 4;
    uint4 v;
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w); }
    __device__ __forceinline__ float largest() const { return fmaxf(fmaxf(get(0), get(1)), fmaxf(get(2), get(3))); }
    static __device__ __forceinline__ float largest(const Logits8 (&x)[kLpVecs]) {
        float m = x[0].largest();
#pragma unroll
        for (int i = 1; i < kLpVecs; ++i) m = fmaxf(m, x[i].largest());
        return m;
    }
    static __device__ __forceinline__ Logits8 nothing() { return Logits8{make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u)}; }
};
template <> struct Logits8<__nv_bfloat16> {
    static constexpr int kN = 8;
    uint4 v;
    __device__ __forceinline__ float get(int i) const {
        const unsigned w = i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w;
        return __uint_as_float(i & 1 ? w & 0xFFFF0000u : w << 16);
    }
    __device__ __forceinline__ float largest() const {
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
        const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
        return fmaxf(__low2float(m), __high2float(m));
    }
    static __device__ __forceinline__ float largest(const Logits8 (&x)[kLpVecs]) {
        __nv_bfloat162 m = reinterpret_cast<const __nv_bfloat162*>(&x[0].v)[0];
#pragma unroll
        for (int i = 0; i < kLpVecs; ++i)
#pragma unroll
            for (int j = i ? 0 : 1; j < 4; ++j) m = __hmax2(m, reinterpret_cast<const __nv_bfloat162*>(&x[i].v)[j]);
        return fmaxf(__low2float(m), __high2float(m));
    }
    static __device__ __forceinline__ Logits8 nothing() { return Logits8{make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u)}; }
};

// A row in vectors that start at multiples of 16 bytes: vector v holds entries v kN - skew and on.  The first and the last may
// lie partly outside the row and are read entry by entry.
template <typename T> struct RowView {
    static constexpr int kN = Logits8<T>::kN;
    const T* row;
    int skew, vocab;
    __device__ __forceinline__ RowView(const T* r, int n) : row(r), skew((int)((reinterpret_cast<uintptr_t>(r) & 15u) / sizeof(T))), vocab(n) {}
    __device__ __forceinline__ int first(int v) const { return v * kN - skew; }
    __device__ __forceinline__ Logits8<T> load(int v) const {
        const int at = first(v);
        Logits8<T> x;
        if (at >= 0 && at + kN <= vocab) { x.v = *reinterpret_cast<const uint4*>(row + at); return x; }
        T e[kN];
#pragma unroll
        for (int i = 0; i < kN; ++i) e[i] = at + i >= 0 && at + i < vocab ? row[at + i] : from_float<T>(-INFINITY);
        x.v = *reinterpret_cast<const uint4*>(e);
        return x;
    }
};

template <typename OT, int N>
__device__ __forceinline__ void store_whole(OT* to, const float (&g)[N]) {
    if (sizeof(OT) == 4) {
#pragma unroll
        for (int i = 0; i < N; i += 4) __stcs(reinterpret_cast<float4*>(to + i), make_float4(g[i], g[i + 1], g[i + 2], g[i + 3]));
    } else if (N == 4) {
        __stcs(reinterpret_cast<uint2*>(to), make_uint2(pack_bf16(g[0], g[1]), pack_bf16(g[2], g[3])));
    } else {
        __stcs(reinterpret_cast<uint4*>(to), make_uint4(pack_bf16(g[0], g[1]), pack_bf16(g[2], g[3]), pack_bf16(g[N - 4], g[N - 3]), pack_bf16(g[N - 2], g[N - 1])));
    }
}
// eight or four results to entries `at` and on of a row of the output; ALIGNED: the vector's place is aligned to its size or 16
template <typename OT, int N>
__device__ __forceinline__ void store_vec(OT* row, int at, int vocab, const float (&g)[N], bool aligned) {
    if (aligned && at >= 0 && at + N <= vocab) {
        store_whole<OT, N>(row + at, g);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) if (at + i >= 0 && at + i < vocab) row[at + i] = from_float<OT>(g[i]);
}
template <typename OT, int N>
__device__ __forceinline__ bool vec_aligned(const OT* row, int skew) {
    constexpr unsigned kTo = N * sizeof(OT) < 16 ? N * sizeof(OT) : 16;
    return ((reinterpret_cast<uintptr_t>(row) - (uintptr_t)skew * sizeof(OT)) & (kTo - 1)) == 0;
}

struct Part { float m, r, t; };              // t with z in units of log 2
__device__ __forceinline__ Part no_part() { return Part{-INFINITY, -1.f, 0.f}; }

// The parts of a warp's lanes as one; `owner` is the first lane with the largest logit, whose 1 stays apart.
__device__ __forceinline__ Part join_lanes(Part p, float scale2, int& owner) {
    const float top = warp_max(p.m);
    owner = __ffs(__ballot_sync(0xFFFFFFFFu, p.m == top)) - 1;
    float r = 0.f, t = 0.f;
    if (p.m != -INFINITY) {
        const float d = max_nan((p.m - top) * scale2, kLeastZ), f = exp2_fast(d), s = 1.f + p.r;
        r = s * f; t = f * fmaf(d, s, p.t);
        if (lane_id() == owner) { r = p.r; t = p.t; }
        if (top == INFINITY) r = t = NAN;
    } else if (lane_id() == owner) r = -1.f;     // (all are -infinity)
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) { r += __shfl_xor_sync(0xFFFFFFFFu, r, d); t += __shfl_xor_sync(0xFFFFFFFFu, t, d); }
    return Part{top, r, t};
}

struct LpSums {
    Part warp[kLpWarps], cta;                // `cta`: read by the other CTAs of the row
};
struct LpTop {                               // for the alternatives
    uint2 group[32];
    unsigned threads[kLpThreads];            // their maxima
    unsigned bound, count;
    u64 round[kLpWarps];
    u64 list[kLpList];
    u64 top[DST_LOGPROB_MAX_TOP];            // the CTA's alternatives: key, then the index' complement (a larger number comes first)
};
struct LpNoTop {};

// The gradient by a row's logits: scale (dlogprob ([here the target] - p) - dentropy p (log p + H)).
struct RowGrad {
    float top, scale, scale2, log_total, entropy, dlogprob, dentropy;
    float base, slope;                       // p's factor is base + slope z2, z2 = log2(p sum); 1 / sum is in both
    bool zero;                               // nothing reaches the row, or it has no probabilities
    long long target;
    __device__ __forceinline__ RowGrad(const LogprobParams& p, long long row, long long given, float largest, float log_sum, float h)
        : top(largest), scale(p.scale), scale2(p.scale2), log_total(log_sum), entropy(h), target(given) {
        dlogprob = target >= 0 && p.dlogprob ? p.dlogprob[row] : 0.f;
        dentropy = p.dentropy ? p.dentropy[row] : 0.f;
        zero = (dlogprob == 0.f && dentropy == 0.f) || top == -INFINITY;
        const float unit = -scale * exp2_fast(-log_total * kLog2e);
        base = unit * (dentropy == 0.f ? dlogprob : fmaf(dentropy, entropy - log_total, dlogprob));
        slope = unit * dentropy * kLn2;
    }
    // of a vector without the target; SLOPE: the entropy counts, and its factor grows where the exponential goes to zero
    template <typename T, bool SLOPE> __device__ __forceinline__ void plain(const Logits8<T>& v, float (&g)[Logits8<T>::kN]) const {
        const Two minus = two(-top, -top), factor = two(scale2, scale2), b2 = two(base, base), s2 = two(slope, slope);
#pragma unroll
        for (int j = 0; j < Logits8<T>::kN; j += 2) {
            float z0, z1;
            apart(mul2(add2(two(v.get(j), v.get(j + 1)), minus), factor), z0, z1);
            if (SLOPE) {
                z0 = max_nan(z0, kLeastZ);
                z1 = max_nan(z1, kLeastZ);
                apart(mul2(two(exp2_fast(z0), exp2_fast(z1)), fma2(s2, two(z0, z1), b2)), g[j], g[j + 1]);
            } else apart(mul2(two(exp2_fast(z0), exp2_fast(z1)), b2), g[j], g[j + 1]);
        }
    }
    // of one logit: any, and the target's, with 1 - p not as a difference
    __device__ __forceinline__ float at(float x) const {
        const float z = max_nan((x - top) * scale2, kLeastZ);
        return exp2_fast(z) * fmaf(slope, z, base);
    }
    __device__ __forceinline__ float target_at(float x) const {
        const float log_p = fmaf(x - top, scale, -log_total), p = exp2_fast(max_nan(log_p * kLog2e, kLeastZ));
        return scale * fmaf(dlogprob, -expm1f(log_p), dentropy == 0.f ? 0.f : -dentropy * p * (max_nan(log_p, kLeastZ) + entropy));
    }
    // of a vector whose first entry is number `at`
    template <typename T> __device__ __forceinline__ void of(const Logits8<T>& v, int at, float (&g)[Logits8<T>::kN]) const {
#pragma unroll
        for (int j = 0; j < Logits8<T>::kN; ++j) g[j] = 0.f;
        if (zero) return;
        if (slope == 0.f) plain<T, false>(v, g); else plain<T, true>(v, g);
        if (target >= at && target < at + Logits8<T>::kN)
#pragma unroll
            for (int j = 0; j < Logits8<T>::kN; ++j) if (at + j == target) g[j] = target_at(v.get(j));
    }
};

// A CTA's part of a row.  KEEP: four vectors a thread, that stay in registers.
template <typename T, bool KEEP, bool GRAD> struct RowPart {
    static constexpr int kN = Logits8<T>::kN;
    RowView<T> row;
    int begin, end;                          // the CTA's vectors
    Logits8<T> kept[KEEP ? kLpVecs : 1];
    __device__ __forceinline__ RowPart(const T* r, int vocab, int b, int e) : row(r, vocab), begin(b), end(e) {}
    __device__ __forceinline__ void fetch(Logits8<T> (&x)[kLpVecs], int v0) const {
        const int step = blockDim.x;
        if (v0 >= (row.skew != 0) && v0 + (kLpVecs - 1) * step < min(end, (row.vocab + row.skew) / kN)) {   // all wholly in the row
            const uint4* const from = reinterpret_cast<const uint4*>(row.row - row.skew) + v0;
#pragma unroll
            for (int i = 0; i < kLpVecs; ++i) {
                if constexpr (GRAD) x[i].v = from[i * step];
                else x[i].v = read_once(from + i * step);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kLpVecs; ++i) if (v0 + i * step < end) x[i] = row.load(v0 + i * step); else x[i] = Logits8<T>::nothing();
        }
    }
    // f(four vectors, the first one's number) for all of the thread's; the others are blockDim.x on, and past the end they hold
    // -infinity.  The next four are on their way meanwhile.
    template <typename F> __device__ __forceinline__ void tiles(F f) {
        if constexpr (KEEP) f(kept, begin + (int)threadIdx.x);
        else {
            const int step = kLpVecs * blockDim.x;
            Logits8<T> x[kLpVecs], y[kLpVecs];
            fetch(x, begin + threadIdx.x);
            if constexpr (GRAD) {                            // (one copy of f: two of them do not fit the registers)
#pragma unroll 1
                for (int v0 = begin + threadIdx.x; v0 < end; v0 += step) {
                    if (v0 + step < end) fetch(y, v0 + step);
                    f(x, v0);
#pragma unroll
                    for (int i = 0; i < kLpVecs; ++i) x[i] = y[i];
                }
            } else {
#pragma unroll 1
                for (int v0 = begin + threadIdx.x; v0 < end; v0 += 2 * step) {
                    if (v0 + step < end) fetch(y, v0 + step);
                    f(x, v0);
                    if (v0 + step >= end) break;
                    if (v0 + 2 * step < end) fetch(x, v0 + 2 * step);
                    f(y, v0 + step);
                }
            }
        }
    }
};

// four more vectors of a thread's
template <typename T>
__device__ __forceinline__ void add_logits(Part& p, const Logits8<T> (&x)[kLpVecs], float scale2) {
    constexpr int kN = Logits8<T>::kN;
    const float top = fmaxf(p.m, Logits8<T>::largest(x));
    float s = 1.f + p.r, t = p.t;
    if (top != p.m) {                                    // what was summed before, seen from the larger maximum
        const float d = max_nan((p.m - top) * scale2, kLeastZ), f = exp2_fast(d);
        t = f * fmaf(d, s, t); s *= f;
        p.m = top;
    }
    const float from = top == -INFINITY ? 0.f : top;     // (nothing but -infinity: z is -infinity all the same; a NaN stays)
    const Two minus = two(-from, -from), factor = two(scale2, scale2);
    Two s2 = two(s, 0.f), t2 = two(t, 0.f);
#pragma unroll
    for (int i = 0; i < kLpVecs; ++i)
#pragma unroll
        for (int j = 0; j < kN; j += 2) {
            float z0, z1;
            apart(mul2(add2(two(x[i].get(j), x[i].get(j + 1)), minus), factor), z0, z1);
            z0 = max_nan(z0, kLeastZ);
            z1 = max_nan(z1, kLeastZ);
            const Two e = two(exp2_fast(z0), exp2_fast(z1));
            s2 = add2(s2, e);
            t2 = fma2(e, two(z0, z1), t2);
        }
    float s1, t1;
    apart(s2, s, s1);
    apart(t2, t, t1);
    p.r = (s + s1) - 1.f;
    p.t = t + t1;
}
template <typename T, bool KEEP, bool GRAD>
__device__ __forceinline__ Part thread_part(RowPart<T, KEEP, GRAD>& mine, float scale2) {
    Part p = no_part();
    mine.tiles([&](const Logits8<T> (&x)[kLpVecs], int) { add_logits<T>(p, x, scale2); });
    return p;
}

// The sum of a thread's exponentials without the first of those that equal `top`, by its warp: vector(i) are the thread's n.
template <typename T, typename F>
__device__ __forceinline__ float others_of(int n, float top, float scale2, F vector) {
    float s = 0.f;
    int ties = 0;
    for (int i = lane_id(); i < n; i += 32) {
        const Logits8<T> x = vector(i);
#pragma unroll
        for (int j = 0; j < Logits8<T>::kN; ++j) {
            const float v = x.get(j);
            if (v == top) ++ties; else s += exp2_fast(max_nan((v - top) * scale2, kLeastZ));
        }
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    return s + (float)((int)__reduce_add_sync(0xFFFFFFFFu, (unsigned)ties) - 1);
}

__device__ __forceinline__ void rank_into(const u64* list, int count, u64* out, int n, int threads) {
    for (int i = threadIdx.x; i < count; i += threads) {
        const u64 k = list[i];
        int before = 0;
#pragma unroll 8
        for (int j = 0; j < count; ++j) before += list[j] > k;
        if (before < n) out[before] = k;
    }
}

// What comes before find_top, around the barrier that the row's sums need too: a bound that n logits reach at least, and few more than n.  It
// is the n-th largest of the maxima of 32 groups (64 for more than eight): the threads with one lane number, since frequent
// tokens often lie together and would all be one group's otherwise.  By the second warp: the first joins the row's sums meanwhile.
__device__ __forceinline__ void post_maximum(float thread_max, LpTop& s) {
    s.threads[threadIdx.x] = order_key(thread_max);
    if (threadIdx.x < DST_LOGPROB_MAX_TOP) s.top[threadIdx.x] = 0;
    if (threadIdx.x == 0) s.count = 0;
}
__device__ __forceinline__ void find_bound(int n, LpTop& s) {
    const int warps = blockDim.x / 32, halves = n > 8 && warps > 1 ? 2 : 1;
    if (warp_id() != (warps > 1 ? 1 : 0)) return;
    uint2 k = make_uint2(0u, 0u);                                       // (below every key)
    for (int w = 0; w < warps; w += halves) {
        k.x = max(k.x, s.threads[w * 32 + lane_id()]);
        if (halves == 2 && w + 1 < warps) k.y = max(k.y, s.threads[w * 32 + 32 + lane_id()]);
    }
    s.group[lane_id()] = k;
    __syncwarp();
    int above_x = 0, from_x = 0, above_y = 0, from_y = 0;               // groups above, and not below, this lane's two
#pragma unroll 8
    for (int j = 0; j < 32; ++j) {
        const uint2 o = s.group[j];
        above_x += (o.x > k.x) + (o.y > k.x); from_x += (o.x >= k.x) + (o.y >= k.x);
        above_y += (o.x > k.y) + (o.y > k.y); from_y += (o.x >= k.y) + (o.y >= k.y);
    }
    if (above_x < n && from_x >= n) s.bound = k.x;
    if (halves == 2 && above_y < n && from_y >= n) s.bound = k.y;
}

// The CTA's n largest logits into s.top (0: none left), for the first warp to see.
template <typename T, bool KEEP, bool GRAD>
__device__ __forceinline__ void find_top(RowPart<T, KEEP, GRAD>& mine, float thread_max, int n, LpTop& s) {
    constexpr int kN = Logits8<T>::kN;
    const int threads = blockDim.x;
    const unsigned key = order_key(thread_max);
    __syncthreads();
    const unsigned bound = max(s.bound, kKeyLowest + 1);                // (-infinity is never listed)
    auto collect = [&](const Logits8<T>& x, int v) {
        if (order_key(x.largest()) < bound) return;
#pragma unroll
        for (int j = 0; j < kN; ++j) {
            const unsigned k = order_key(x.get(j));
            if (k < bound) continue;
            const unsigned at = atomicAdd(&s.count, 1u);
            if (at < kLpList) s.list[at] = (u64)k << 32 | (unsigned)~(mine.row.first(v) + j);
        }
    };
    if constexpr (KEEP) {
        if (key >= bound)
            mine.tiles([&](const Logits8<T> (&x)[kLpVecs], int v0) {
#pragma unroll
                for (int i = 0; i < kLpVecs; ++i) collect(x[i], v0 + i * threads);
            });
    } else {
        // a thread's vectors again, by a whole warp, those of four threads at a time; neighbouring threads by different warps
        const int warps = threads / 32;
        for (unsigned left = __ballot_sync(0xFFFFFFFFu, s.threads[lane_id() * warps + warp_id()] >= bound); left;) {
            int first[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                first[i] = left ? mine.begin + (__ffs(left) - 1) * warps + warp_id() + lane_id() * threads : mine.end;
                left &= left - 1;
            }
            for (int at = 0; at < mine.end - mine.begin; at += 32 * threads) {
                Logits8<T> x[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) if (first[i] + at < mine.end) x[i] = mine.row.load(first[i] + at); else x[i] = Logits8<T>::nothing();
#pragma unroll
                for (int i = 0; i < 4; ++i) collect(x[i], first[i] + at);
            }
        }
    }
    __syncthreads();
    const int count = (int)s.count;
    if (count <= 64) {                                                  // as nearly always: by one warp
        if (warp_id() == 0) {
            rank_into(s.list, count, s.top, n, 32);
            __syncwarp();
        }
        return;
    }
    if (count <= kLpList) {
        rank_into(s.list, count, s.top, n, threads);
        __syncthreads();
        return;
    }
    u64 last = ~0ull;
    for (int place = 0; place < n; ++place) {
        u64 best = 0;
        if (key >= bound)
            mine.tiles([&](const Logits8<T> (&x)[kLpVecs], int v0) {
#pragma unroll
                for (int i = 0; i < kLpVecs; ++i)
#pragma unroll
                    for (int j = 0; j < kN; ++j) {
                        const unsigned k = order_key(x[i].get(j));
                        const u64 full = (u64)k << 32 | (unsigned)~(mine.row.first(v0 + i * threads) + j);
                        if (k >= bound && full < last && full > best) best = full;
                    }
            });
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) { const u64 o = __shfl_xor_sync(0xFFFFFFFFu, best, d); if (o > best) best = o; }
        if (lane_id() == 0) s.round[warp_id()] = best;
        __syncthreads();
        for (int w = 0; w < threads / 32; ++w) if (s.round[w] > best) best = s.round[w];
        if (threadIdx.x == 0) s.top[place] = best;
        __syncthreads();
        if (best == 0) break;
        last = best;
    }
}

__device__ __forceinline__ long long target_of(const LogprobParams& p, long long row) {
    if (!p.targets) return -1;
    return p.wide ? static_cast<const long long*>(p.targets)[row] : static_cast<const int*>(p.targets)[row];
}

// the given token of a row, -1 for none; one that is out of range is counted by one thread
__device__ __forceinline__ long long checked_target(const LogprobParams& p, long long row, bool counts) {
    const long long target = target_of(p, row);
    if (target < p.vocab) return target;
    if (p.result && counts) {
        atomicAdd(reinterpret_cast<u64*>(&p.result->n_out_of_range), 1ull);
        p.result->status = DST_ERR_INDEX_OUT_OF_RANGE;
    }
    return -1;
}

// A whole row's numbers.
struct RowSums {
    float top, log_total, entropy;
    __device__ __forceinline__ RowSums(Part all) : top(all.m) {
        if (all.m == INFINITY) all.r = all.t = NAN;
        log_total = log1pf(all.r);                            // (log1p(-1) is -infinity, for a row of nothing but that)
        entropy = all.m == -INFINITY ? 0.f : log_total - all.t * kLn2 / (1.f + all.r);
    }
    __device__ __forceinline__ void write(const LogprobParams& p, long long row, long long target, float given) const {
        const bool empty = top == -INFINITY;
        if (p.logprob) p.logprob[row] = target < 0 ? 0.f : empty ? -INFINITY : fmaf(given - top, p.scale, -log_total);
        if (p.lse) p.lse[row] = empty ? -INFINITY : fmaf(top, p.scale, log_total);
        if (p.entropy) p.entropy[row] = entropy;
        if (p.stats) { p.stats[2 * row] = top; p.stats[2 * row + 1] = log_total; }
    }
};

// GRAD: with the gradient; LIST: with the alternatives
template <typename T, typename OT, bool KEEP, bool GRAD, bool LIST>
__global__ void __launch_bounds__(KEEP ? kLpThreads : kLpStream, !KEEP ? 4 : GRAD ? 2 : 1) k_logprob(const __grid_constant__ LogprobParams p) {
    constexpr int kN = Logits8<T>::kN;
    __shared__ LpSums s;
    __shared__ std::conditional_t<LIST, LpTop, LpNoTop> tops;   // (what no call needs would be taken from the first-level cache)
    cg::cluster_group cluster = cg::this_cluster();
    const int ctas = 1 << p.cut, rank = blockIdx.x & (ctas - 1);
    const long long row = blockIdx.x >> p.cut;
    pdl_trigger();
    pdl_wait();
    const T* const x = static_cast<const T*>(p.logits) + row * p.ld;
    RowPart<T, KEEP, GRAD> mine(x, p.vocab, rank * p.vectors, 0);
    mine.end = min(mine.begin + p.vectors, (p.vocab + mine.row.skew + kN - 1) / kN);
    if constexpr (KEEP) mine.fetch(mine.kept, mine.begin + threadIdx.x);

    const Part thread = thread_part(mine, p.scale2);
    // (thread 0 of the first CTA alone uses the given token's logit; it is read before anything is written, and registers are few while the row is)
    const long long target = checked_target(p, row, rank == 0 && threadIdx.x == 0);
    const float given = target >= 0 && threadIdx.x == 0 ? to_float<T>(x[target]) : 0.f;
    // (a thread with nothing but NaN and -infinity has no largest logit, but its NaN counts)
    int owner;
    Part all = join_lanes(thread.m == -INFINITY && thread.r != thread.r ? Part{0.f, thread.r, thread.r} : thread, p.scale2, owner);
    if (all.r < 0.25f && all.m != -INFINITY) {               // nearly all on one token: what the thread that holds it rounded against 1, anew
        const int first = mine.begin + warp_id() * 32 + owner, step = blockDim.x;
        const float exact = others_of<T>((mine.end - first + step - 1) / step, all.m, p.scale2, [&](int i) { return mine.row.load(first + i * step); });
        all.r += exact - __shfl_sync(0xFFFFFFFFu, thread.r, owner);
    }
    if (lane_id() == 0) s.warp[warp_id()] = all;
    if constexpr (LIST) post_maximum(thread.m, tops);
    __syncthreads();
    if constexpr (LIST) find_bound(p.top_n, tops);
    if (GRAD || ctas > 1 || warp_id() == 0) all = join_lanes(lane_id() < (int)blockDim.x / 32 ? s.warp[lane_id()] : no_part(), p.scale2, owner);
    else if (!LIST) return;
    if constexpr (LIST) find_top(mine, thread.m, p.top_n, tops);
    if (ctas > 1) {
        if (threadIdx.x == 0) s.cta = all;
        cluster.sync();
        int first;
        all = join_lanes(lane_id() < ctas ? *cluster.map_shared_rank(&s.cta, lane_id()) : no_part(), p.scale2, first);
    }
    const RowSums sums(all);
    if (rank == 0 && threadIdx.x == 0) sums.write(p, row, target, given);
    if constexpr (GRAD) {
        const RowGrad grad(p, row, target, all.m, sums.log_total, sums.entropy);
        OT* const d = static_cast<OT*>(p.dlogits) + row * p.ldd;
        const bool aligned = vec_aligned<OT, kN>(d, mine.row.skew);
        mine.tiles([&](const Logits8<T> (&v)[kLpVecs], int v0) {
#pragma unroll
            for (int i = 0; i < kLpVecs; ++i) {
                if (v0 + i * (int)blockDim.x >= mine.end) break;
                const int at = mine.row.first(v0 + i * blockDim.x);
                float g[kN];
                grad.of(v[i], at, g);
                store_vec<OT, kN>(d, at, p.vocab, g, aligned);
            }
        });
    } else if constexpr (LIST) {
        const int n = p.top_n;
        auto put = [&](int place, u64 k) {
            if (p.top_tokens) {
                const int token = k == 0 ? -1 : (int)~(unsigned)k;
                if (p.wide) static_cast<long long*>(p.top_tokens)[row * n + place] = token;
                else static_cast<int*>(p.top_tokens)[row * n + place] = token;
            }
            if (p.top_logprob) p.top_logprob[row * n + place] = k == 0 ? -INFINITY : fmaf(of_order_key((unsigned)(k >> 32)) - all.m, p.scale, -sums.log_total);
        };
        if (ctas == 1) {
            if ((int)threadIdx.x < n) put(threadIdx.x, tops.top[threadIdx.x]);
        } else {
            // every CTA finds the places of its own n among all: a lane for each of them and each CTA's n (empty places, which all come last, by their own place)
            for (int i = threadIdx.x; i < ctas * n; i += blockDim.x) tops.list[i] = cluster.map_shared_rank(tops.top, i / n)[i % n];
            __syncthreads();
            for (int u0 = warp_id() * 32; u0 < ctas * n; u0 += blockDim.x) {
                const int i = min((u0 + lane_id()) >> p.cut, n - 1), of = (lane_id() & (ctas - 1)) * n, me = rank * n + i;
                const u64 k = tops.list[me];
                int before = 0;
#pragma unroll 4
                for (int j = of; j < of + n; ++j) { const u64 o = tops.list[j]; before += o > k || (o == k && j < me); }
                for (int d = 1; d < ctas; d *= 2) before += __shfl_xor_sync(0xFFFFFFFFu, before, d);
                if (u0 + lane_id() < ctas * n && (lane_id() & (ctas - 1)) == 0 && before < n) put(before, k);
            }
        }
    }
    if (ctas > 1) cluster.sync();                            // (what others read of this CTA stays until then)
}

// The gradient from what the forward call gave: the same arithmetic.
template <typename T, typename OT>
__global__ void __launch_bounds__(256) k_logprob_backward(const __grid_constant__ LogprobParams p) {
    constexpr int kN = Logits8<T>::kN;
    const int parts = ((p.vocab + 2 * kN - 2) / kN + p.vectors - 1) / p.vectors;
    const unsigned block = gridDim.x - 1 - blockIdx.x;       // last rows first: what the forward call read last is still in L2 (both calls, in turn with the first row first, three times: 8111 x 33,708 fp32 497 us against 501, 700 x 33,708 54.0 against 55.3, 4096 x 33,708 bf16 159.9 against 161.0)
    const long long row = block / parts;
    const int part = (int)(block - row * parts);
    pdl_trigger();
    pdl_wait();
    const RowView<T> x(static_cast<const T*>(p.logits) + row * p.ld, p.vocab);
    const int begin = part * p.vectors + threadIdx.x, end = min((part + 1) * p.vectors, (p.vocab + x.skew + kN - 1) / kN);
    Logits8<T> v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) if (begin + i * 256 < end) v[i] = x.load(begin + i * 256);
    const long long target = target_of(p, row);
    const RowGrad grad(p, row, target < p.vocab ? target : -1, p.saved_stats[2 * row], p.saved_stats[2 * row + 1], p.saved_entropy ? p.saved_entropy[row] : 0.f);
    OT* const d = static_cast<OT*>(p.dlogits) + row * p.ldd;
    const bool aligned = vec_aligned<OT, kN>(d, x.skew);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (begin + i * 256 >= end) break;
        const int at = x.first(begin + i * 256);
        float g[kN];
        grad.of(v[i], at, g);
        store_vec<OT, kN>(d, at, p.vocab, g, aligned);
    }
}

// The loss and its gradient of many rows that fit into shared memory: a CTA takes every gridDim.x-th row.  One warp brings the rows in by
// bulk copies, chunk after chunk into a ring; the others read a row twice there, for its sums and for the gradient, and give the
// chunks back on the second time.  Every logit crosses from memory once, and what is free of the ring holds the next row's first
// chunks while a row's sums are joined.  The pieces of a row before and after its whole vectors come by the copying warp's own loads.
template <int N> struct Ring {                              // N threads that work; one more warp copies
    static constexpr int kCtas = N <= 384 ? 2 : 1;          // on an SM
    static constexpr int kChunk = 2 * N;                    // vectors
    static constexpr int kSlots = (kCtas == 2 ? 112 : 224) * 1024 / (kChunk * 16);
    static constexpr int kSmem = kSlots * kChunk * 16;
};
template <typename T, typename OT, int N>
__global__ void __launch_bounds__(N + 32, Ring<N>::kCtas) k_logprob_ring(const __grid_constant__ LogprobParams p) {
    using S = Ring<N>;
    constexpr int kN = Logits8<T>::kN, kWarps = N / 32;
    static_assert(kLpVecs == 4, "two chunks of two vectors");
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ Part parts[2][kWarps];
    __shared__ __align__(8) unsigned long long bars[2 * S::kSlots];
    const unsigned full = smem_addr(bars), empty = full + 8 * S::kSlots;
    pdl_trigger();
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kSlots; ++i) { bar_init(full + 8 * i, 1); bar_init(empty + 8 * i, kWarps); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    pdl_wait();
    bool ok = true;
    if (warp_id() == kWarps) {                               // ---- copies ----
        int slot = 0;
        unsigned phase = 1;                                  // every slot is free at first
        for (long long row = blockIdx.x; row < p.rows && ok; row += gridDim.x) {
            const RowView<T> x(static_cast<const T*>(p.logits) + row * p.ld, p.vocab);
            const int whole0 = x.skew ? 1 : 0, whole1 = (p.vocab + x.skew) / kN, end = (p.vocab + x.skew + kN - 1) / kN;
            // an entry of the first or the last vector, where they lie partly outside the row
            const int piece = lane_id() / kN == 0 && whole0 ? 0 : lane_id() / kN == 1 && whole1 < end ? whole1 : -1, entry = x.first(piece) + lane_id() % kN;
            T value = from_float<T>(-INFINITY);
            if (piece >= 0 && entry >= 0 && entry < p.vocab) value = x.row[entry];
            for (int v = 0; v < end; v += S::kChunk) {
                ok = bar_wait(empty + 8 * slot, phase);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                unsigned char* const at = ring + slot * S::kChunk * 16;
                const int from = max(v, whole0), to = min(v + S::kChunk, whole1);
                if (piece >= v && piece < v + S::kChunk) reinterpret_cast<T*>(at)[(piece - v) * kN + lane_id() % kN] = value;
                __syncwarp();
                if (lane_id() == 0) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // (the pieces' places belong to a copy again next time)
                    if (from < to) {
                        bar_expect(full + 8 * slot, (to - from) * 16);
                        copy_bytes(smem_addr(at) + (from - v) * 16, x.row + x.first(from), (to - from) * 16, full + 8 * slot);
                    } else bar_arrive(full + 8 * slot);
                }
                if (++slot == S::kSlots) { slot = 0; phase ^= 1; }
            }
        }
    } else {
        const uint4* const slots = reinterpret_cast<const uint4*>(ring);
        int slot = 0, turn = 0;
        unsigned phase = 0;
        for (long long row = blockIdx.x; row < p.rows; row += gridDim.x, turn ^= 1) {
            const RowView<T> x(static_cast<const T*>(p.logits) + row * p.ld, p.vocab);
            const int end = (p.vocab + x.skew + kN - 1) / kN, chunks = (end + S::kChunk - 1) / S::kChunk;
            const long long target = checked_target(p, row, threadIdx.x == 0);
            const float given = target >= 0 ? to_float<T>(x.row[target]) : 0.f;   // (read before anything is written, which may be in place)
            Part mine = no_part();
            const int slot0 = slot;
            auto next_chunk = [&] {
                ok = ok && bar_wait(full + 8 * slot, phase);
                const uint4* const at = slots + slot * S::kChunk + threadIdx.x;
                if (++slot == S::kSlots) { slot = 0; phase ^= 1; }
                return at;
            };
#pragma unroll 1
            for (int c = 0; c < chunks; c += 2) {
                Logits8<T> v[kLpVecs];
                const uint4* from = next_chunk();
                if ((c + 2) * S::kChunk <= end) {
                    v[0].v = from[0]; v[1].v = from[N];
                    from = next_chunk();
                    v[2].v = from[0]; v[3].v = from[N];
                } else {
                    const uint4* const more = c + 1 < chunks ? next_chunk() : from;
#pragma unroll
                    for (int i = 0; i < kLpVecs; ++i) {
                        v[i] = Logits8<T>::nothing();
                        if (c * S::kChunk + i * N + (int)threadIdx.x < end) v[i].v = (i < 2 ? from : more)[(i & 1) * N];
                    }
                }
                add_logits<T>(mine, v, p.scale2);
            }
            if (!ok) mine.r = NAN;                           // a copy that never came
            int owner;
            Part all = join_lanes(mine.m == -INFINITY && mine.r != mine.r ? Part{0.f, mine.r, mine.r} : mine, p.scale2, owner);
            if (all.r < 0.25f && all.m != -INFINITY) {       // (as in k_logprob; the lane's vectors by memory)
                const int first = warp_id() * 32 + owner;
                const float exact = others_of<T>((end - first + N - 1) / N, all.m, p.scale2, [&](int i) {
                    Logits8<T> v;
                    v.v = slots[(slot0 + i / 2) % S::kSlots * S::kChunk + (i & 1) * N + first];
                    return v;
                });
                all.r += exact - __shfl_sync(0xFFFFFFFFu, mine.r, owner);
            }
            if (lane_id() == 0) parts[turn][warp_id()] = all;
            asm volatile("bar.sync 1, %0;" ::"n"(N) : "memory");
            all = join_lanes(lane_id() < kWarps ? parts[turn][lane_id()] : no_part(), p.scale2, owner);
            const RowSums sums(all);
            if (threadIdx.x == 0) sums.write(p, row, target, given);
            const RowGrad grad(p, row, target, all.m, sums.log_total, sums.entropy);
            OT* const d = static_cast<OT*>(p.dlogits) + row * p.ldd;
            const int whole0 = x.skew != 0, whole1 = (p.vocab + x.skew) / kN;
            const bool aligned = vec_aligned<OT, kN>(d, x.skew);
            // f(chunk, the thread's two vectors of it) for the row's chunks, which go back once every lane has worked with what it read: a
            // read that was only issued may still be on its way when the next copy lands
            auto each_chunk = [&](auto f) {
                int k = slot0;
#pragma unroll 1
                for (int c = 0; c < chunks; ++c) {
                    f(c, slots + k * S::kChunk + threadIdx.x);
                    __syncwarp();
                    if (lane_id() == 0) bar_arrive(empty + 8 * k);
                    if (++k == S::kSlots) k = 0;
                }
            };
            auto gradients = [&](auto slope) {
                OT* const mine_out = d + x.first(threadIdx.x);
                each_chunk([&](int c, const uint4* from) {
                    OT* const to = mine_out + c * (S::kChunk * kN);
                    const int at = c * S::kChunk + threadIdx.x;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        Logits8<T> v;
                        v.v = from[h * N];
                        float g[kN];
                        grad.template plain<T, decltype(slope)::value>(v, g);
                        if (at + h * N >= whole0 && at + h * N < whole1) store_whole<OT, kN>(to + h * N * kN, g);
                    }
                });
            };
            if (grad.zero || !aligned)
                each_chunk([&](int c, const uint4* from) {
#pragma unroll 1
                    for (int at = c * S::kChunk + threadIdx.x, h = 0; h < 2 && at < end; at += N, ++h) {
                        Logits8<T> v;
                        v.v = from[h * N];
                        float g[kN];
                        grad.of(v, x.first(at), g);
                        store_vec<OT, kN>(d, x.first(at), p.vocab, g, aligned);
                    }
                });
            else if (grad.slope == 0.f) gradients(std::false_type{});
            else gradients(std::true_type{});
            if (grad.zero || !aligned) continue;
            // the target, by the thread that wrote its vector, and the pieces before and after the whole vectors, an entry a lane
            const int of = target >= 0 ? (int)((target + x.skew) / kN) : -1;
            if (of >= whole0 && of < whole1 && of % N == (int)threadIdx.x) d[target] = from_float<OT>(grad.target_at(given));
            const int pieces = p.vocab - (whole1 - whole0) * kN, entry = lane_id() < x.first(whole0) ? lane_id() : lane_id() + (whole1 - whole0) * kN;
            if (warp_id() == kWarps - 1 && lane_id() < pieces) {
                const float v = to_float<T>(x.row[entry]);
                d[entry] = from_float<OT>(entry == target ? grad.target_at(v) : grad.at(v));
            }
        }
    }
    if (!ok) {                                               // let copies in flight land
        const long long t0 = clock64();
        while (clock64() - t0 < (1LL << 24)) {}
    }
}

// How a row is cut.  Many rows: a CTA of 256 threads each (fewer for short rows: eight vectors a thread at least, 2000 x 5000 bf16 9.4 us against 12.8 with
// two), four on an SM, which read them four vectors a thread at a time.  Where two CTAs a row still do not pass the SMs, two to eight, each with
// as many threads as hold its part at two to four vectors (48 x 33,708 bf16 4.9 us with two, 8.2 with eight; 150 rows 6.6 with one, 10.2 with two, 20 with four: clusters
// of CTAs that fill the device wait for one another's places).
struct LogprobShape { int ctas, threads, vectors, keep; };
static LogprobShape logprob_shape(long long rows, long long vocab, int per_vector, bool grad, int sms) {
    const long long all = (vocab + 2 * per_vector - 2) / per_vector;     // whatever the row's place within 16 bytes
    LogprobShape L{1, 0, 0, 1};
    auto per = [&] { return (all + L.ctas - 1) / L.ctas; };
    while (L.ctas < kLpCtas && rows * L.ctas * 2 <= sms && per() > 256) L.ctas *= 2;
    const long long most = rows * L.ctas < 2 * sms && per() <= kLpVecs * kLpThreads ? kLpThreads : kLpStream;
    const long long each = rows * L.ctas < 2 * sms ? 2 : grad ? kLpVecs : 2 * kLpVecs;   // vectors a thread, at least
    long long t = (per() + each - 1) / each;
    t = (t + 31) / 32 * 32;
    L.threads = int(t < most ? t : most);
    L.vectors = int(per());
    // (kept in registers: for the gradient, or where rows are few; many rows without one do better with half the registers a thread)
    L.keep = per() <= (long long)kLpVecs * L.threads && (grad || rows * L.ctas < 2 * sms);
    return L;
}

template <typename T, typename OT, bool KEEP, bool GRAD, bool LIST>
static cudaError_t logprob_run(const LogprobParams& p, const LogprobShape& L, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.rows * L.ctas)); cfg.blockDim = dim3(L.threads); cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = L.ctas; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, k_logprob<T, OT, KEEP, GRAD, LIST>, p);
}
template <typename T, typename OT, bool GRAD, bool LIST>
static cudaError_t logprob_t(LogprobParams p, int sms, cudaStream_t stream) {
    const LogprobShape L = logprob_shape(p.rows, p.vocab, Logits8<T>::kN, GRAD, sms);
    p.vectors = L.vectors;
    p.cut = L.ctas == 1 ? 0 : L.ctas == 2 ? 1 : L.ctas == 4 ? 2 : 3;
    return L.keep ? logprob_run<T, OT, true, GRAD, LIST>(p, L, stream) : logprob_run<T, OT, false, GRAD, LIST>(p, L, stream);
}
cudaError_t launch_logprob(const LogprobParams& p, int type, int sms, cudaStream_t stream) {
    if (p.top_n > 0) return type == DST_F32 ? logprob_t<float, float, false, true>(p, sms, stream) : logprob_t<__nv_bfloat16, float, false, true>(p, sms, stream);
    return type == DST_F32 ? logprob_t<float, float, false, false>(p, sms, stream) : logprob_t<__nv_bfloat16, float, false, false>(p, sms, stream);
}

template <typename T, typename OT, int N>
static cudaError_t ring_run(const LogprobParams& p, int sms, cudaStream_t stream) {
    using S = Ring<N>;
    static SmemOptIn opt;
    const cudaError_t e = ensure_dynamic_smem(k_logprob_ring<T, OT, N>, S::kSmem, opt);
    if (e != cudaSuccess) return e;
    const long long ctas = (long long)sms * S::kCtas;
    return launch_pdl(k_logprob_ring<T, OT, N>, dim3((unsigned)(p.rows < ctas ? p.rows : ctas)), dim3(N + 32), S::kSmem, stream, p);
}
template <typename T, typename OT>
static cudaError_t loss_t(const LogprobParams& p, int sms, cudaStream_t stream) {
    // Threads: two CTAs an SM while a row fits half of its shared memory, as many as their registers allow (4096 x 33,708 bf16 122 us with 384, 136 with 320,
    // 128 with 288, 130 with 256; shorter rows 2400 x 9000 35.2, 34.7, 32.9, 36.6); else one CTA of 480, whose slots
    // hold rows of up to 12 chunks of 960 vectors, where 736 threads have room for 7 of 1472 (8111 x 33,708 fp32 372 us with 480, 392 with 416, 374 with 640,
    // 363 with 736; 4096 x 65,536 bf16 249, 249, 250, 238).
    constexpr int kTwo = 384, kOne = 480;
    const long long vectors = (p.vocab + 2 * Logits8<T>::kN - 2) / Logits8<T>::kN;
    // More than half as many rows as SMs, fewer of which are cut, and rows longer than four vectors for each of 256 threads, which keep them in
    // registers (ring and not, bf16: 100 x 33,708 9.7 and 13.8 us, 600 x 33,708 23.5 and 31.6, 2400 x 33,708 74 and 92, 2400 x 65,536 149 and 153, 2400 x 9000 35.3 and
    // 36.4, 1200 x 5000 16.3 and 11.0; fp32: 100 x 33,708 9.3 and 19.8, 2400 x 33,708 119 and 154, 1200 x 5000 15.7 and 17.3).  Rows that leave the ring no room for two
    // chunks more are streamed and read again from L2.
    if (2 * p.rows > sms && vectors > 1024) {
        if (vectors <= (Ring<kTwo>::kSlots - 2) * Ring<kTwo>::kChunk) return ring_run<T, OT, kTwo>(p, sms, stream);
        if (vectors <= (Ring<kOne>::kSlots - 2) * Ring<kOne>::kChunk) return ring_run<T, OT, kOne>(p, sms, stream);
    }
    return logprob_t<T, OT, true, false>(p, sms, stream);
}
cudaError_t launch_logprob_loss(const LogprobParams& p, int type, int d_type, int sms, cudaStream_t stream) {
    if (type == DST_F32) return d_type == DST_F32 ? loss_t<float, float>(p, sms, stream) : loss_t<float, __nv_bfloat16>(p, sms, stream);
    return d_type == DST_F32 ? loss_t<__nv_bfloat16, float>(p, sms, stream) : loss_t<__nv_bfloat16, __nv_bfloat16>(p, sms, stream);
}

template <typename T, typename OT>
static cudaError_t logprob_backward_t(LogprobParams p, cudaStream_t stream) {
    constexpr int kN = Logits8<T>::kN;
    p.vectors = 4 * 256;
    const long long parts = ((p.vocab + 2 * kN - 2) / kN + p.vectors - 1) / p.vectors;
    return launch_pdl(k_logprob_backward<T, OT>, dim3((unsigned)(p.rows * parts)), dim3(256), 0, stream, p);
}
cudaError_t launch_logprob_backward(const LogprobParams& p, int type, int d_type, cudaStream_t stream) {
    if (type == DST_F32) return d_type == DST_F32 ? logprob_backward_t<float, float>(p, stream) : logprob_backward_t<float, __nv_bfloat16>(p, stream);
    return d_type == DST_F32 ? logprob_backward_t<__nv_bfloat16, float>(p, stream) : logprob_backward_t<__nv_bfloat16, __nv_bfloat16>(p, stream);
}

}  // namespace dst
