/*
 * What a training step, or an answer, around the tied weight needs next to dst.h and dst_tied.h:
 *
 *   dst_rmsnorm, dst_rmsnorm_backward   the norm before the projection, with the residual's addition, to 8 bits where
 *                                       dst_matmul_fp8 takes it
 *   dst_logprob                         log probabilities of given tokens, entropy, the most likely tokens
 *   dst_logprob_loss,
 *   dst_logprob_backward                the gradient of the logits, which the projection's backward takes
 *   dst_grad_norm, dst_clip             the norm over all gradients and their scaling, before dst_densify_apply
 *
 * Conventions are those of dst.h and dst_tied.h: device pointers, caller-owned buffers, nothing allocated or
 * synchronised, all work on `stream`, bad arguments refused on the host before anything is enqueued.  A matrix argument
 * has a leading dimension in elements; its rows are contiguous.  Sizes of zero are valid and do nothing unless a comment
 * says otherwise.  Calls that share a workspace or an output must be ordered, captured ones too.  Two calls with the same arguments give the same bits; the order of sums follows from the sizes and types, and
 * from how rows are aligned.
 */
#ifndef DST_STEP_H_
#define DST_STEP_H_

#include "dst_tied.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Log probabilities under softmax(scale * x), x the logits of a row as fp32 and scale (1 / temperature) above 0 and at most 2e38:
 *     z_i = scale * (x_i - max x),  S = sum exp(z_i),  log p_i = z_i - log S
 *   logprob [rows]        log p of the row's target; 0 for a row without one
 *   lse [rows]            scale * max x + log S (an infinity where that passes fp32's range)
 *   stats [rows, 2]       max x and log S, for the gradient: with them z is a difference of logits, whatever their size
 *   entropy [rows]        -sum p_i log p_i
 *   top_tokens, top_logprob [rows, top_n]   the top_n <= DST_LOGPROB_MAX_TOP largest logits in descending order, equal
 *                         ones by index, and their log p; logits of -infinity and NaN are not listed, places left over
 *                         hold token -1 and -infinity.  A row in which hundreds of logits equal the last of these (all logits
 *                         equal; a mask of the type's lowest value that leaves fewer than top_n) is read once more for each
 * targets [rows] and top_tokens have index_type.  A negative target marks a row without one (padding); one of vocab or
 * more counts as none too, and is counted in `result` (optional, cleared by this call).  Every output may be NULL;
 * targets may be NULL where logprob is.
 * Logits of -infinity have probability zero and add nothing to the entropy.  A row of nothing but -infinity has lse and
 * logprob -infinity and entropy 0.  A row with a NaN or +infinity has NaN for all three and in top_logprob.
 * A log probability near zero is accurate relative to itself, not to one: what the largest logit leaves is summed apart
 * (probabilities below 2^-126 count as zero).
 * rows > 0 with vocab = 0 is refused.
 */
#define DST_LOGPROB_MAX_TOP 32
int dst_logprob(const void* logits, int64_t ld, int32_t type, int64_t rows, int64_t vocab, const void* targets,
                int32_t index_type, float scale, float* logprob, float* lse, float* entropy, float* stats,
                int64_t top_n, void* top_tokens, float* top_logprob, dst_result_t* result, dst_stream_t stream);

/*
 * The gradient of a loss that reaches a row through logprob and entropy, with dlogprob and dentropy [rows] its
 * derivatives by them (NULL: zero):
 *     dlogits_i = scale * (dlogprob * ([i = target] - p_i) - dentropy * p_i * (log p_i + entropy))
 * in d_type (fp32 or bf16, rounded once).  dlogits may be the logits themselves where type and leading dimension agree;
 * it must not overlap them otherwise.  A row without a target has dlogprob = 0.  A row whose two derivatives are zero,
 * and one whose logits are all -infinity, gets zeros whatever its logits.
 *
 * dst_logprob_loss is dst_logprob (without alternatives) and the gradient in one pass, for derivatives that are known
 * before (cross entropy: dlogprob = -1 / tokens).  dst_logprob_backward takes what dst_logprob gave: stats, and entropy with
 * dentropy.  (The calls may split a row's sums in other ways, which the number of rows decides too; they agree to rounding.)
 */
int dst_logprob_loss(const void* logits, int64_t ld, int32_t type, int64_t rows, int64_t vocab, const void* targets,
                     int32_t index_type, float scale, const float* dlogprob, const float* dentropy, float* logprob,
                     float* lse, float* entropy, void* dlogits, int64_t ldd, int32_t d_type, dst_result_t* result,
                     dst_stream_t stream);
int dst_logprob_backward(const void* logits, int64_t ld, int32_t type, int64_t rows, int64_t vocab, const void* targets,
                         int32_t index_type, float scale, const float* stats, const float* entropy, const float* dlogprob,
                         const float* dentropy, void* dlogits, int64_t ldd, int32_t d_type, dst_stream_t stream);

/*
 * Root-mean-square norm of the residual stream, d <= DST_RMSNORM_MAX_D:
 *     h = x + residual, rounded to sum_type (h = x where residual and sum_out are NULL)
 *     inv_rms = 1 / sqrt(mean(h^2) + eps),  y = h * inv_rms * weight        (sums in fp32: a row whose squares pass its range has
 *     inv_rms 0)
 *   x [rows, d] in x_type; residual (optional) and sum_out (optional, receives h; may be residual, or x where types
 *   agree) in sum_type; weight [d] fp32 or NULL (ones); inv_rms [rows] fp32, optional, for the backward pass
 *   out [rows, d] in out_type and / or q, its 8-bit form (DST_FP8_ROW blocks, rounded once from fp32, as
 *   dst_quantize_fp8 would from an fp32 y); one of them at least.  out may be x's or residual's buffer where that one is not
 *   needed afterwards and type and leading dimension agree; sum_out's holds h, and out in its place is refused.
 */
#define DST_RMSNORM_MAX_D 16384
int dst_rmsnorm(const void* x, int64_t ldx, int32_t x_type, const void* residual, int64_t ldr, void* sum_out,
                int64_t lds, int32_t sum_type, const float* weight, float eps, void* out, int64_t ldo, int32_t out_type,
                const dst_fp8_t* q, float* inv_rms, int64_t rows, int64_t d, dst_stream_t stream);

/*
 * Its gradient, with dy [rows, d] in dy_type that of y, h in h_type and inv_rms as the forward call left them, and u = h * inv_rms:
 *     dx = dsum + inv_rms * (dy * weight - u * mean(dy * weight * u))       (the gradient of x and of residual alike)
 *     dweight = sum over rows of dy * u
 * dsum (optional: what reaches h by the residual stream) and dx in dx_type; dx may be dsum, dy or h where type and leading
 * dimension agree.  dweight [d] fp32, optional: overwritten, in an order of sums that the sizes fix; zeros where rows = 0.
 * workspace: dst_rmsnorm_backward_workspace_bytes(rows, d) bytes, 256-byte aligned, needed with dweight alone.
 */
size_t dst_rmsnorm_backward_workspace_bytes(int64_t rows, int64_t d);
int dst_rmsnorm_backward(const void* dy, int64_t ldy, int32_t dy_type, const void* h, int64_t ldh, int32_t h_type,
                         const float* weight, const float* inv_rms, const void* dsum, int64_t ldds, void* dx, int64_t lddx,
                         int32_t dx_type, float* dweight, int64_t rows, int64_t d, void* workspace, size_t workspace_bytes,
                         dst_stream_t stream);

/* One of a list of tensors: n contiguous elements of `type` (dst_dtype_t) at `data`.  The list itself is host memory,
 * read during the call. */
typedef struct {
    void* data;
    int64_t n;
    int32_t type;
    int32_t reserved;
} dst_tensor_t;

/*
 * clip[0] = the square root of the sum of all elements' squares (accumulated in 64 bits, so that squares neither overflow
 * nor vanish), clip[1] = the factor min(1, max_norm / (norm + 1e-6)), or 0 where the norm is not finite (a NaN or an
 * infinity among the elements): fp32 in DEVICE memory.  An empty list has norm 0.  max_norm >= 0.
 * workspace: dst_grad_norm_workspace_bytes(tensors, count) bytes, 256-byte aligned.
 */
size_t dst_grad_norm_workspace_bytes(const dst_tensor_t* tensors, int64_t count);
int dst_grad_norm(const dst_tensor_t* tensors, int64_t count, double max_norm, float* clip, void* workspace,
                  size_t workspace_bytes, dst_stream_t stream);

/*
 * outs[i] = clip[1] * tensors[i], rounded once to outs[i]'s type; the two lists have the same lengths.  A factor of 0
 * writes zeros whatever the elements are.  outs may be the same list: in place, where types agree, and a factor of 1
 * then touches nothing.  Otherwise an output that overlaps a tensor, or another output, is refused, in place too (a tensor that is
 * listed twice would be scaled twice; in the norm it counts twice).  Tensors may overlap one another.
 */
int dst_clip(const dst_tensor_t* tensors, const dst_tensor_t* outs, int64_t count, const float* clip, dst_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* DST_STEP_H_ */
