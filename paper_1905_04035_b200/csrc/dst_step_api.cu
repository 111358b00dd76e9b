// C ABI of a step's operators: argument checks and kernel sequencing.
#include <math.h>

#include <algorithm>
#include <memory>
#include <new>

#include "dst_step.cuh"

namespace dst {

constexpr int64_t kMaxLogits = int64_t(1) << 30, kMaxLogitRows = int64_t(1) << 27, kMaxNormRows = int64_t(1) << 31;
constexpr int64_t kMaxTensor = int64_t(1) << 44, kMaxTensors = int64_t(1) << 24;

// 0: fine.  What the three entries for log probabilities have in common.
static int logprob_params(LogprobParams& p, const void* logits, int64_t ld, int32_t type, int64_t rows, int64_t vocab, const void* targets,
                          int32_t index_type, float scale) {
    p = LogprobParams{};
    if (!dtype_ok(type) || !index_ok(index_type)) return DST_ERR_UNSUPPORTED;
    if (!matrix_ok(logits, ld, rows, vocab, type) || !(scale > 0.f) || !isfinite(scale)) return DST_ERR_INVALID_ARG;
    if (vocab > kMaxLogits || rows > kMaxLogitRows) return DST_ERR_UNSUPPORTED;
    if (misaligned(targets, index_type == DST_I64 ? 8 : 4) || (vocab == 0 && rows > 0)) return DST_ERR_INVALID_ARG;
    p.logits = logits; p.targets = targets; p.ld = ld; p.rows = rows; p.vocab = int(vocab); p.wide = index_type == DST_I64;
    p.scale = scale; p.scale2 = float(double(scale) * 1.4426950408889634);
    return isfinite(p.scale2) ? DST_OK : DST_ERR_INVALID_ARG;
}
static int logprob_grad(LogprobParams& p, int32_t type, const float* dlogprob, const float* dentropy, void* dlogits, int64_t ldd, int32_t d_type) {
    if (!dtype_ok(d_type)) return DST_ERR_UNSUPPORTED;
    if (!matrix_ok(dlogits, ldd, p.rows, p.vocab, d_type) || misaligned(dlogprob, 4) || misaligned(dentropy, 4)) return DST_ERR_INVALID_ARG;
    if (dlogprob && !p.targets && p.rows > 0) return DST_ERR_INVALID_ARG;
    if (dlogits && dlogits == p.logits && (ldd != p.ld || d_type != type)) return DST_ERR_INVALID_ARG;
    p.dlogprob = dlogprob; p.dentropy = dentropy; p.dlogits = dlogits; p.ldd = ldd;
    return DST_OK;
}
static int clear_result(dst_result_t* result, cudaStream_t stream) {
    return !result || cudaMemsetAsync(result, 0, sizeof *result, stream) == cudaSuccess ? DST_OK : DST_ERR_CUDA;
}

static bool tensors_ok(const dst_tensor_t* t, int64_t count) {
    if (count < 0 || (count > 0 && !t)) return false;
    for (int64_t i = 0; i < count; ++i)
        if (t[i].n < 0 || !dtype_ok(t[i].type) || (t[i].n > 0 && !t[i].data) || misaligned(t[i].data, type_size(t[i].type))) return false;
    return true;
}
static bool tensors_fit(const dst_tensor_t* t, int64_t count) {
    if (count > kMaxTensors) return false;
    for (int64_t i = 0; i < count; ++i) if (t[i].n > kMaxTensor) return false;
    return true;
}

// Whether every output has memory of its own: none lies on another, nor on a tensor other than the one that it takes the place of.
// A CTA writes an output's chunk while others have yet to read theirs.
struct Span { uintptr_t from, to; };
static Span span_of(const dst_tensor_t& t) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(t.data);
    return Span{at, t.n > kMaxTensor ? UINTPTR_MAX : at + uintptr_t(t.n) * type_size(t.type)};
}
static int outputs_apart(const dst_tensor_t* in, const dst_tensor_t* out, int64_t count) {
    constexpr int64_t kFew = 128;
    Span few[kFew];
    std::unique_ptr<Span[]> many;
    if (count > kFew) many.reset(new (std::nothrow) Span[size_t(count)]);
    Span* const spans = count > kFew ? many.get() : few;
    if (!spans) return DST_ERR_UNSUPPORTED;
    int64_t n = 0;
    for (int64_t i = 0; i < count; ++i) if (out[i].n > 0) spans[n++] = span_of(out[i]);
    std::sort(spans, spans + n, [](const Span& a, const Span& b) { return a.from < b.from; });
    for (int64_t i = 1; i < n; ++i) if (spans[i - 1].to > spans[i].from) return DST_ERR_INVALID_ARG;
    for (int64_t i = 0; i < count; ++i) {
        if (in[i].n == 0 || in[i].data == out[i].data) continue;             // (in place: where its output is)
        const Span s = span_of(in[i]);
        if (s.to <= spans[0].from || s.from >= spans[n - 1].to) continue;    // (as of lists that were made one after the other)
        const Span* const after = std::lower_bound(spans, spans + n, s.to, [](const Span& a, uintptr_t to) { return a.from < to; });
        if (after > spans && after[-1].to > s.from) return DST_ERR_INVALID_ARG;   // the last output that starts before its end
    }
    return DST_OK;
}

}  // namespace dst

using namespace dst;

extern "C" {

int dst_logprob(const void* logits, int64_t ld, int32_t type, int64_t rows, int64_t vocab, const void* targets,
                int32_t index_type, float scale, float* logprob, float* lse, float* entropy, float* stats, int64_t top_n,
                void* top_tokens, float* top_logprob, dst_result_t* result, dst_stream_t stream) {
    LogprobParams p;
    const int rc = logprob_params(p, logits, ld, type, rows, vocab, targets, index_type, scale);
    if (rc != DST_OK) return rc;
    if (top_n > DST_LOGPROB_MAX_TOP) return DST_ERR_UNSUPPORTED;
    if (top_n < 0 || (logprob && !targets && rows > 0) || misaligned(logprob, 4) || misaligned(lse, 4) || misaligned(entropy, 4) || misaligned(stats, 4) ||
        misaligned(top_tokens, index_type == DST_I64 ? 8 : 4) || misaligned(top_logprob, 4) || misaligned(result, 8))
        return DST_ERR_INVALID_ARG;
    if (clear_result(result, stream) != DST_OK) return DST_ERR_CUDA;
    if (rows == 0) return DST_OK;
    p.logprob = logprob; p.lse = lse; p.entropy = entropy; p.stats = stats; p.result = result;
    p.top_n = top_tokens || top_logprob ? int(top_n) : 0; p.top_tokens = top_tokens; p.top_logprob = top_logprob;
    return done(launch_logprob(p, type, device_sm_count(), stream), 1);
}

int dst_logprob_loss(const void* logits, int64_t ld, int32_t type, int64_t rows, int64_t vocab, const void* targets,
                     int32_t index_type, float scale, const float* dlogprob, const float* dentropy, float* logprob,
                     float* lse, float* entropy, void* dlogits, int64_t ldd, int32_t d_type, dst_result_t* result,
                     dst_stream_t stream) {
    LogprobParams p;
    int rc = logprob_params(p, logits, ld, type, rows, vocab, targets, index_type, scale);
    if (rc == DST_OK) rc = logprob_grad(p, type, dlogprob, dentropy, dlogits, ldd, d_type);
    if (rc != DST_OK) return rc;
    if ((logprob && !targets && rows > 0) || misaligned(logprob, 4) || misaligned(lse, 4) || misaligned(entropy, 4) || misaligned(result, 8)) return DST_ERR_INVALID_ARG;
    if (clear_result(result, stream) != DST_OK) return DST_ERR_CUDA;
    if (rows == 0) return DST_OK;
    p.logprob = logprob; p.lse = lse; p.entropy = entropy; p.result = result;
    return done(launch_logprob_loss(p, type, d_type, device_sm_count(), stream), 1);
}

int dst_logprob_backward(const void* logits, int64_t ld, int32_t type, int64_t rows, int64_t vocab, const void* targets,
                         int32_t index_type, float scale, const float* stats, const float* entropy, const float* dlogprob,
                         const float* dentropy, void* dlogits, int64_t ldd, int32_t d_type, dst_stream_t stream) {
    LogprobParams p;
    int rc = logprob_params(p, logits, ld, type, rows, vocab, targets, index_type, scale);
    if (rc == DST_OK) rc = logprob_grad(p, type, dlogprob, dentropy, dlogits, ldd, d_type);
    if (rc != DST_OK) return rc;
    if (misaligned(stats, 4) || misaligned(entropy, 4)) return DST_ERR_INVALID_ARG;
    if (rows == 0) return DST_OK;
    if (!stats || (dentropy && !entropy)) return DST_ERR_INVALID_ARG;
    p.saved_stats = stats; p.saved_entropy = entropy;
    return done(launch_logprob_backward(p, type, d_type, stream), 1);
}

int dst_rmsnorm(const void* x, int64_t ldx, int32_t x_type, const void* residual, int64_t ldr, void* sum_out,
                int64_t lds, int32_t sum_type, const float* weight, float eps, void* out, int64_t ldo, int32_t out_type,
                const dst_fp8_t* q, float* inv_rms, int64_t rows, int64_t d, dst_stream_t stream) {
    if (!dtype_ok(x_type) || !dtype_ok(sum_type) || !dtype_ok(out_type)) return DST_ERR_UNSUPPORTED;
    if (!matrix_ok(x, ldx, rows, d, x_type) || (residual && !matrix_ok(residual, ldr, rows, d, sum_type)) ||
        (sum_out && !matrix_ok(sum_out, lds, rows, d, sum_type)) || (out && !matrix_ok(out, ldo, rows, d, out_type)))
        return DST_ERR_INVALID_ARG;
    if (misaligned(weight, 4) || misaligned(inv_rms, 4) || !(eps >= 0.f) || !isfinite(eps)) return DST_ERR_INVALID_ARG;
    if (rows > kMaxNormRows || d > DST_RMSNORM_MAX_D) return DST_ERR_UNSUPPORTED;
    NormParams p{};
    if (q) {
        const int rc = fp8_view(q, p.q);
        if (rc != DST_OK) return rc;
        if (q->rows != rows || q->cols != d || q->block != DST_FP8_ROW) return DST_ERR_INVALID_ARG;
    }
    // in place only where every element stays where it is
    if (sum_out && ((sum_out == x && (lds != ldx || sum_type != x_type)) || (sum_out == residual && lds != ldr))) return DST_ERR_INVALID_ARG;
    if (out && ((out == x && (ldo != ldx || out_type != x_type)) || (out == residual && (ldo != ldr || out_type != sum_type)) || out == sum_out)) return DST_ERR_INVALID_ARG;
    if (rows == 0 || d == 0) return DST_OK;
    if (!out && !q) return DST_ERR_INVALID_ARG;
    p.x = x; p.residual = residual; p.sum_out = sum_out; p.weight = weight; p.out = out; p.inv_rms = inv_rms;
    p.ldx = ldx; p.ldr = ldr; p.lds = lds; p.ldo = ldo; p.rows = rows; p.d = int(d); p.eps = eps; p.keep = residual || sum_out;
    return done(launch_rmsnorm(p, x_type, sum_type, out_type, stream), 1);
}

size_t dst_rmsnorm_backward_workspace_bytes(int64_t rows, int64_t d) {
    if (rows <= 0 || d <= 0 || rows > kMaxNormRows || d > DST_RMSNORM_MAX_D) return 0;
    return rmsnorm_backward_workspace(rows, d);
}

int dst_rmsnorm_backward(const void* dy, int64_t ldy, int32_t dy_type, const void* h, int64_t ldh, int32_t h_type,
                         const float* weight, const float* inv_rms, const void* dsum, int64_t ldds, void* dx, int64_t lddx,
                         int32_t dx_type, float* dweight, int64_t rows, int64_t d, void* workspace, size_t workspace_bytes,
                         dst_stream_t stream) {
    if (!dtype_ok(dy_type) || !dtype_ok(h_type) || !dtype_ok(dx_type)) return DST_ERR_UNSUPPORTED;
    if (!matrix_ok(dy, ldy, rows, d, dy_type) || !matrix_ok(h, ldh, rows, d, h_type) || !matrix_ok(dx, lddx, rows, d, dx_type) ||
        (dsum && !matrix_ok(dsum, ldds, rows, d, dx_type)))
        return DST_ERR_INVALID_ARG;
    if (misaligned(weight, 4) || misaligned(inv_rms, 4) || misaligned(dweight, 4)) return DST_ERR_INVALID_ARG;
    if (rows > kMaxNormRows || d > DST_RMSNORM_MAX_D) return DST_ERR_UNSUPPORTED;
    if (dx && ((dx == dy && (lddx != ldy || dx_type != dy_type)) || (dx == h && (lddx != ldh || dx_type != h_type)) || (dx == dsum && lddx != ldds))) return DST_ERR_INVALID_ARG;
    if (d == 0) return DST_OK;
    if (rows == 0)   // an empty sum
        return !dweight || cudaMemsetAsync(dweight, 0, size_t(d) * 4, stream) == cudaSuccess ? DST_OK : DST_ERR_CUDA;
    if (!inv_rms) return DST_ERR_INVALID_ARG;
    if (dweight) {
        if (!workspace || misaligned(workspace, 256)) return DST_ERR_INVALID_ARG;
        if (workspace_bytes < rmsnorm_backward_workspace(rows, d)) return DST_ERR_WORKSPACE_TOO_SMALL;
    }
    const NormBackParams p{dy, h, weight, inv_rms, dsum, dx, dweight, dweight ? static_cast<float*>(workspace) : nullptr,
                           (long long)ldy, (long long)ldh, (long long)ldds, (long long)lddx, (long long)rows, int(d)};
    return done(launch_rmsnorm_backward(p, dy_type, h_type, dx_type, stream), dweight ? 2 : 1);
}

size_t dst_grad_norm_workspace_bytes(const dst_tensor_t* tensors, int64_t count) {
    if (!tensors_ok(tensors, count) || !tensors_fit(tensors, count)) return 0;
    return grad_norm_workspace(tensors, count);
}

int dst_grad_norm(const dst_tensor_t* tensors, int64_t count, double max_norm, float* clip, void* workspace,
                  size_t workspace_bytes, dst_stream_t stream) {
    if (!tensors_ok(tensors, count) || !clip || misaligned(clip, 4) || !(max_norm >= 0.)) return DST_ERR_INVALID_ARG;
    if (!tensors_fit(tensors, count)) return DST_ERR_UNSUPPORTED;
    const size_t need = grad_norm_workspace(tensors, count);
    if (need > 0 && (!workspace || misaligned(workspace, 256))) return DST_ERR_INVALID_ARG;
    if (workspace_bytes < need) return DST_ERR_WORKSPACE_TOO_SMALL;
    int launches = 0;
    const cudaError_t e = launch_grad_norm(tensors, count, max_norm, clip, workspace, &launches, stream);
    return done(e, launches);
}

int dst_clip(const dst_tensor_t* tensors, const dst_tensor_t* outs, int64_t count, const float* clip, dst_stream_t stream) {
    if (!tensors_ok(tensors, count) || !tensors_ok(outs, count) || !clip || misaligned(clip, 4)) return DST_ERR_INVALID_ARG;
    if (count > kMaxTensors) return DST_ERR_UNSUPPORTED;
    for (int64_t i = 0; i < count; ++i) {
        if (tensors[i].n != outs[i].n) return DST_ERR_INVALID_ARG;
        if (tensors[i].n > 0 && tensors[i].data == outs[i].data && tensors[i].type != outs[i].type) return DST_ERR_INVALID_ARG;
    }
    const int rc = outputs_apart(tensors, outs, count);
    if (rc != DST_OK) return rc;
    if (!tensors_fit(tensors, count)) return DST_ERR_UNSUPPORTED;
    int launches = 0;
    const cudaError_t e = launch_clip(tensors, outs, count, clip, &launches, stream);
    return done(e, launches);
}

}  // extern "C"
