// Shared definitions of the kernels of a step: log probabilities, root-mean-square norm, gradient norm and clipping.
#pragma once

#include "dst_step.h"
#include "dst_tied.cuh"

namespace dst {

// ---- log probabilities (dst_logprob.cu) -------------------------------------------
struct LogprobParams {
    const void* logits;
    const void* targets;                    // or null
    const float* dlogprob;                  // gradient: or null, as dentropy
    const float* dentropy;
    const float* saved_stats;               // backward alone: what the forward call gave
    const float* saved_entropy;
    float* logprob;                         // outputs, or null
    float* lse;
    float* entropy;
    float* stats;
    void* top_tokens;
    float* top_logprob;
    void* dlogits;
    dst_result_t* result;
    long long ld, ldd, rows;
    int vocab, wide;                        // indices are 64-bit
    int top_n;
    float scale, scale2;                    // scale2 = scale * log2(e)
    int vectors;                            // of 16 bytes that a CTA of the row's cluster takes
    int cut;                                // a row has 2^cut CTAs
};
cudaError_t launch_logprob(const LogprobParams& p, int type, int sms, cudaStream_t stream);
cudaError_t launch_logprob_loss(const LogprobParams& p, int type, int d_type, int sms, cudaStream_t stream);
cudaError_t launch_logprob_backward(const LogprobParams& p, int type, int d_type, cudaStream_t stream);

// ---- root-mean-square norm (dst_norm.cu) ------------------------------------------
struct NormParams {
    const void* x;
    const void* residual;
    void* sum_out;
    const float* weight;
    void* out;
    Fp8View q;                              // q.q null: not wanted
    float* inv_rms;
    long long ldx, ldr, lds, ldo, rows;
    int d;
    float eps;
    int keep;                               // h is rounded to the stream's type before the norm
};
cudaError_t launch_rmsnorm(const NormParams& p, int x_type, int sum_type, int out_type, cudaStream_t stream);
struct NormBackParams {
    const void* dy;
    const void* h;
    const float* weight;
    const float* inv_rms;
    const void* dsum;
    void* dx;
    float* dweight;
    float* parts;                           // [CTAs, d]
    long long ldy, ldh, ldds, lddx, rows;
    int d;
};
size_t rmsnorm_backward_workspace(long long rows, long long d);
cudaError_t launch_rmsnorm_backward(const NormBackParams& p, int dy_type, int h_type, int dx_type, cudaStream_t stream);

// ---- gradient norm and clipping (dst_clip.cu) -------------------------------------
size_t grad_norm_workspace(const dst_tensor_t* tensors, long long count);
cudaError_t launch_grad_norm(const dst_tensor_t* tensors, long long count, double max_norm, float* clip, void* workspace, int* launches, cudaStream_t stream);
cudaError_t launch_clip(const dst_tensor_t* tensors, const dst_tensor_t* outs, long long count, const float* clip, int* launches, cudaStream_t stream);

// ---- device helpers ---------------------------------------------------------------
#ifdef __CUDACC__
// 16 bytes that are read once and that nothing writes meanwhile, not kept in the first-level cache (volatile: it stays behind the wait for
// the kernel before)
__device__ __forceinline__ uint4 read_once(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
#endif

}  // namespace dst
