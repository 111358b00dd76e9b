// The norm over a list of tensors and their scaling by one factor.
//
// The tensors are cut into chunks, numbered through the list; a CTA takes every gridDim.x-th and finds the tensor by bisection
// in the table, which travels as a kernel parameter (longer lists take several launches).  Squares are summed in 64 bits:
// exact to 2^-52, and neither a large gradient overflows nor a small one vanishes.  The CTAs' sums are added in their order by one
// CTA, so the norm depends on the values, the sizes and types, and on which tensors are aligned to 16 bytes (the others are read an element
// a thread, and their squares are added up in other lanes).  Bound by memory: the list is read once for the norm, read and written
// once for the scaling.
// Measured: 186 million gradients, 34.5 million in fp32 and 151 in bf16: norm 70 us (6280 GB/s; 74 by way of the first-level cache), scaling 144 us (6110 GB/s); 163,840 in fp32: 3.9
// and 3.3 us, launches and one round of loads.
#include "dst_step.cuh"

namespace dst {

constexpr int kClipEntries = 96;             // tensors of a launch
constexpr int kClipThreads = 256;
constexpr int kClipBatch = 4;                // pieces of 16 bytes that a thread has in flight
constexpr int kClipChunk = kClipThreads * 64;    // elements
constexpr int kClipOnSm = 6;                 // CTAs that fit an SM, and
constexpr int kClipCtas = kClipOnSm * kSmCount;   // most CTAs of a launch (of a B200's SMs, not the device's: they fix the order of sums)

struct ClipEntry {
    const void* in;
    void* out;
    long long n;
    int first;                               // number of the tensor's first chunk in this launch
    short in_type, out_type;
};
struct ClipTable {
    ClipEntry e[kClipEntries];
    int count, chunks;
};

// the chunk's tensor, and the chunk's place in it
__device__ __forceinline__ const ClipEntry& tensor_of(const ClipTable& t, int chunk, long long& start, int& n) {
    int low = 0, high = t.count - 1;
    while (low < high) {
        const int mid = (low + high + 1) / 2;
        if (t.e[mid].first <= chunk) low = mid; else high = mid - 1;
    }
    const ClipEntry& e = t.e[low];
    start = (long long)(chunk - e.first) * kClipChunk;
    n = (int)min(e.n - start, (long long)kClipChunk);
    return e;
}
__device__ __forceinline__ bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

template <typename T>
__device__ __forceinline__ double chunk_squares(const T* x, int n) {
    double s[2] = {0., 0.};
    int done = 0;
    if (aligned16(x)) {
        constexpr int kPer = 16 / (int)sizeof(T), kBatch = kClipBatch;
        const int pieces = n / kPer;
        done = pieces * kPer;
        const uint4* const from = reinterpret_cast<const uint4*>(x);
#pragma unroll 1
        for (int i = threadIdx.x; i < pieces; i += kBatch * kClipThreads) {
            uint4 w[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) w[j] = i + j * kClipThreads < pieces ? read_once(from + i + j * kClipThreads) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const unsigned u[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (sizeof(T) == 4) { const double v = (double)__uint_as_float(u[k]); s[k & 1] = fma(v, v, s[k & 1]); }
                    else {
                        const double a = (double)__uint_as_float(u[k] << 16), b = (double)__uint_as_float(u[k] & 0xFFFF0000u);
                        s[0] = fma(a, a, s[0]); s[1] = fma(b, b, s[1]);
                    }
                }
            }
        }
    }
    for (int i = done + threadIdx.x; i < n; i += kClipThreads) {
        const double v = (double)to_float<T>(x[i]);
        s[0] = fma(v, v, s[0]);
    }
    return s[0] + s[1];
}

__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
    return x;
}

__global__ void __launch_bounds__(kClipThreads, kClipOnSm) k_grad_squares(const __grid_constant__ ClipTable t, double* parts) {
    __shared__ double sums[kClipThreads / 32];
    pdl_trigger();
    pdl_wait();
    double s = 0.;
    for (int c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        long long start;
        int n;
        const ClipEntry& e = tensor_of(t, c, start, n);
        s += e.in_type == DST_F32 ? chunk_squares(static_cast<const float*>(e.in) + start, n) : chunk_squares(static_cast<const __nv_bfloat16*>(e.in) + start, n);
    }
    s = warp_sum(s);
    if (lane_id() == 0) sums[warp_id()] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kClipThreads / 32; ++w) s += sums[w];
        parts[blockIdx.x] = s;
    }
}

__global__ void __launch_bounds__(kClipThreads) k_grad_norm(const double* parts, int n, double max_norm, float* clip) {
    __shared__ double sums[kClipThreads / 32];
    pdl_trigger();
    pdl_wait();
    double s = 0.;
    for (int i = threadIdx.x; i < n; i += kClipThreads) s += parts[i];
    s = warp_sum(s);
    if (lane_id() == 0) sums[warp_id()] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kClipThreads / 32; ++w) s += sums[w];
        const double norm = sqrt(s), factor = max_norm / (norm + 1e-6);
        clip[0] = (float)norm;
        clip[1] = !isfinite(s) ? 0.f : factor < 1. ? (float)factor : 1.f;
    }
}

__device__ __forceinline__ float scaled(float x, float f) { return f == 0.f ? 0.f : x * f; }
__device__ __forceinline__ unsigned scaled_two(unsigned w, float f) {      // two bf16
    return pack_bf16(scaled(__uint_as_float(w << 16), f), scaled(__uint_as_float(w & 0xFFFF0000u), f));
}
// 16 bytes of a tensor whose output has its type
__device__ __forceinline__ uint4 scaled_piece(uint4 v, float f, const float*) {
    return make_uint4(__float_as_uint(scaled(__uint_as_float(v.x), f)), __float_as_uint(scaled(__uint_as_float(v.y), f)),
                      __float_as_uint(scaled(__uint_as_float(v.z), f)), __float_as_uint(scaled(__uint_as_float(v.w), f)));
}
__device__ __forceinline__ uint4 scaled_piece(uint4 v, float f, const __nv_bfloat16*) {
    return make_uint4(scaled_two(v.x, f), scaled_two(v.y, f), scaled_two(v.z, f), scaled_two(v.w, f));
}
template <typename T>
__device__ __forceinline__ void scale_chunk(const T* x, T* out, int n, float f) {
    constexpr int kPer = 16 / (int)sizeof(T), kBatch = kClipBatch;
    int done = 0;
    if (aligned16(x) && aligned16(out)) {
        const int pieces = n / kPer;
        done = pieces * kPer;
        const uint4* const from = reinterpret_cast<const uint4*>(x);
        uint4* const to = reinterpret_cast<uint4*>(out);
#pragma unroll 1
        for (int i = threadIdx.x; i < pieces; i += kBatch * kClipThreads) {
            uint4 v[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) if (i + j * kClipThreads < pieces) v[j] = from[i + j * kClipThreads];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) if (i + j * kClipThreads < pieces) to[i + j * kClipThreads] = scaled_piece(v[j], f, x);
        }
    }
    for (int i = done + threadIdx.x; i < n; i += kClipThreads) out[i] = from_float<T>(scaled(to_float<T>(x[i]), f));
}
template <typename T, typename OT>
__device__ __forceinline__ void scale_convert(const T* x, OT* out, int n, float f) {
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += kClipThreads) out[i] = from_float<OT>(scaled(to_float<T>(x[i]), f));
}

__global__ void __launch_bounds__(kClipThreads, 4) k_clip(const __grid_constant__ ClipTable t, const float* clip) {
    pdl_trigger();
    pdl_wait();
    const float f = clip[1];
    for (int c = t.chunks - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) {   // last first: what the norm read last is still in L2
        long long start;
        int n;
        const ClipEntry& e = tensor_of(t, c, start, n);
        if (f == 1.f && e.in == e.out) continue;             // (in place: nothing to do)
        const float* const x = static_cast<const float*>(e.in) + start;
        const __nv_bfloat16* const h = static_cast<const __nv_bfloat16*>(e.in) + start;
        float* const out = static_cast<float*>(e.out) + start;
        __nv_bfloat16* const half = static_cast<__nv_bfloat16*>(e.out) + start;
        if (e.in_type == DST_F32 && e.out_type == DST_F32) scale_chunk(x, out, n, f);
        else if (e.in_type == DST_BF16 && e.out_type == DST_BF16) scale_chunk(h, half, n, f);
        else if (e.in_type == DST_F32) scale_convert(x, half, n, f);
        else scale_convert(h, out, n, f);
    }
}

// f(table) for every launch that the list takes; tensors without elements are left out
template <typename F>
static cudaError_t tables(const dst_tensor_t* in, const dst_tensor_t* out, long long count, F f) {
    ClipTable t;
    t.count = 0; t.chunks = 0;
    for (long long i = 0; i < count; ++i) {
        if (in[i].n == 0) continue;
        const long long chunks = (in[i].n + kClipChunk - 1) / kClipChunk;
        if (t.count == kClipEntries || t.chunks + chunks > 0x7FFFFFFFll) {
            const cudaError_t e = f(t);
            if (e != cudaSuccess) return e;
            t.count = 0; t.chunks = 0;
        }
        t.e[t.count++] = ClipEntry{in[i].data, out ? out[i].data : nullptr, (long long)in[i].n, t.chunks, (short)in[i].type, (short)(out ? out[i].type : in[i].type)};
        t.chunks += (int)chunks;
    }
    return t.count > 0 ? f(t) : cudaSuccess;
}
static int clip_ctas(const ClipTable& t) { return t.chunks < kClipCtas ? t.chunks : kClipCtas; }

size_t grad_norm_workspace(const dst_tensor_t* tensors, long long count) {
    size_t ctas = 0;
    tables(tensors, nullptr, count, [&](const ClipTable& t) { ctas += clip_ctas(t); return cudaSuccess; });
    return ctas * sizeof(double);
}
cudaError_t launch_grad_norm(const dst_tensor_t* tensors, long long count, double max_norm, float* clip, void* workspace, int* launches, cudaStream_t stream) {
    double* const parts = static_cast<double*>(workspace);
    int done = 0;
    const cudaError_t e = tables(tensors, nullptr, count, [&](const ClipTable& t) {
        const int ctas = clip_ctas(t);
        done += ctas; ++*launches;
        return launch_pdl(k_grad_squares, dim3(ctas), dim3(kClipThreads), 0, stream, t, parts + done - ctas);
    });
    if (e != cudaSuccess) return e;
    ++*launches;
    return launch_pdl(k_grad_norm, dim3(1), dim3(kClipThreads), 0, stream, static_cast<const double*>(parts), done, max_norm, clip);
}
cudaError_t launch_clip(const dst_tensor_t* tensors, const dst_tensor_t* outs, long long count, const float* clip, int* launches, cudaStream_t stream) {
    return tables(tensors, outs, count, [&](const ClipTable& t) {
        ++*launches;
        return launch_pdl(k_clip, dim3(clip_ctas(t)), dim3(kClipThreads), 0, stream, t, clip);
    });
}

}  // namespace dst
