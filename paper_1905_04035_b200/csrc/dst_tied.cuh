// Shared definitions of the kernels around the tied weight: dropout, embedding, 8-bit products, sampling.
#pragma once

#include "dst_common.cuh"
#include "dst_tied.h"

namespace dst {

// ---- shared host state (dst_api.cu) ----------------------------------------------
int device_sm_count();                      // of the current device, asked of the runtime once
void count_launches(int n);                 // what dst_kernel_launches reports

// ---- dropout and embedding (dst_dropout.cu) ---------------------------------------
struct DropParams {                         // the generator's keys of every round and counter, and the factor of a kept element
    unsigned key0[10], key1[10];
    unsigned below;                         // 16-bit halves, in the upper half of a word, up to this are dropped
    int none;                               // nothing is dropped, no bits are drawn
    float keep;                             // 65536 / (65536 - cut), 0 when everything is dropped
    unsigned long long offset;
    const unsigned long long* offset_device;
    unsigned row_offset;
};
// Units (parts of a row) that a thread takes are a fixed number apart; where the next one lies follows by additions.
struct UnitStep { long long units, rows; unsigned per_row, part; };   // in all, rows on, parts of a row, parts on
struct DropoutParams {
    DropParams drop;
    UnitStep step;
    const void* x;
    const void* residual;
    void* out;
    long long ldx, ldr, ldo;
    long long rows;
    int d;
    float scale;
};
struct EmbedParams {
    DropParams drop;
    UnitStep step;
    const void* indices;
    const void* weight;
    const float* position;
    void* out;
    dst_result_t* result;
    long long rows, vocab, n_positions;
    int d;
    float scale;
};
cudaError_t launch_dropout(const DropoutParams& p, int x_type, int out_type, int sms, cudaStream_t stream);
cudaError_t launch_embed(const EmbedParams& p, int index_type, int weight_type, int out_type, int sms, cudaStream_t stream);

// ---- 8-bit floating point (dst_fp8.cu) --------------------------------------------
struct Fp8View {                            // dst_fp8_t
    uint8_t* q;
    uint8_t* scale;
    long long rows, cols, ld, ld_scale;
    int square;
};
constexpr int kScaleTile = 512;             // bytes of scales for 128 rows by 4 column blocks
struct QuantParams {
    const void* x;
    long long ldx, rows, cols;
    Fp8View q, qt;                          // q.q / qt.q null: not wanted
};
cudaError_t launch_quantize(const QuantParams& p, int x_type, cudaStream_t stream);
size_t matmul_fp8_workspace(long long M, long long N, long long K);        // of this product
size_t matmul_fp8_workspace_bound(long long M, long long N, long long K);  // of this one and every smaller one
cudaError_t launch_matmul_fp8(const Fp8View& a, const Fp8View& b, void* out, long long ldo, int out_type, void* workspace,
                              int sms, cudaStream_t stream);

bool linear_fp8_fused(long long M, long long N, long long K);               // x can be quantised inside the product
cudaError_t launch_linear_fp8_fused(const void* x, long long ldx, int x_type, long long M, const Fp8View& w, void* out, long long ldo,
                                    int out_type, int sms, cudaStream_t stream);

// ---- sampling (dst_sample.cu) -----------------------------------------------------
struct SampleParams {
    const void* logits;
    const float* uniform;
    const float* temperature;
    const int* top_k;
    const float* top_p;
    const float* min_p;
    void* tokens;
    float* prob;
    long long ld, rows;
    int vocab;
    int wide;                               // tokens are 64-bit
};
cudaError_t launch_sample(const SampleParams& p, int type, int sms, cudaStream_t stream);

// ---- device helpers ---------------------------------------------------------------
#ifdef __CUDACC__
template <typename T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// eight consecutive elements, 16-byte aligned (fp32: 32 bytes in two loads); plain loads, never the read-only path: an
// input may be the output, and no load may move above the wait for the kernel before
template <typename T> __device__ __forceinline__ void load8(const T* p, float (&v)[8]);
template <> __device__ __forceinline__ void load8<float>(const float* p, float (&v)[8]) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void widen8(const uint4& t, float (&v)[8]) {      // eight bf16
    v[0] = __uint_as_float(t.x << 16); v[1] = __uint_as_float(t.x & 0xFFFF0000u);
    v[2] = __uint_as_float(t.y << 16); v[3] = __uint_as_float(t.y & 0xFFFF0000u);
    v[4] = __uint_as_float(t.z << 16); v[5] = __uint_as_float(t.z & 0xFFFF0000u);
    v[6] = __uint_as_float(t.w << 16); v[7] = __uint_as_float(t.w & 0xFFFF0000u);
}
template <> __device__ __forceinline__ void load8<__nv_bfloat16>(const __nv_bfloat16* p, float (&v)[8]) {
    widen8(*reinterpret_cast<const uint4*>(p), v);
}
__device__ __forceinline__ unsigned pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const unsigned*>(&v);
}
template <typename T> __device__ __forceinline__ void store8(T* p, const float (&v)[8]);
template <> __device__ __forceinline__ void store8<float>(float* p, const float (&v)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
template <> __device__ __forceinline__ void store8<__nv_bfloat16>(__nv_bfloat16* p, const float (&v)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}
#endif

}  // namespace dst
