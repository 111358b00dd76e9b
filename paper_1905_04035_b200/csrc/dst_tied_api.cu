// C ABI of the operators around the tied weight: argument checks, workspace carving, kernel sequencing.
#include <math.h>

#include "dst_tied.cuh"

namespace dst {

constexpr int64_t kMaxCols = int64_t(1) << 30;   // columns of a row, and rows of a matrix in 8 bits

// The generator's parameters; false: refused.
static bool drop_params(const dst_dropout_t* d, int64_t rows, DropParams& p) {
    p = DropParams{};
    p.none = 1; p.keep = 1.f;
    if (!d) return true;
    if (!(d->p >= 0.0 && d->p <= 1.0) || d->row_offset < 0 || d->row_offset > (int64_t(1) << 32) - rows) return false;
    if (misaligned(d->offset_device, 8)) return false;
    for (unsigned r = 0; r < 10; ++r) {                  // each round moves the keys by a fixed step
        p.key0[r] = unsigned(d->seed) + r * 0x9E3779B9u;
        p.key1[r] = unsigned(d->seed >> 32) + r * 0xBB67AE85u;
    }
    const unsigned cut = unsigned(rint(d->p * 65536.0));
    p.none = cut == 0;
    p.below = cut == 0 ? 0u : unsigned((uint64_t(cut) << 16) - 1);
    p.keep = cut >= 65536u ? 0.f : 65536.f / float(65536u - cut);
    p.offset = d->offset;
    p.offset_device = reinterpret_cast<const unsigned long long*>(d->offset_device);
    p.row_offset = unsigned(d->row_offset);
    return true;
}

// 0: fine; the view of a matrix in 8 bits whose buffers are there
int fp8_view(const dst_fp8_t* m, Fp8View& v) {
    if (!m || m->rows < 0 || m->cols < 0 || m->ld < m->cols) return DST_ERR_INVALID_ARG;
    if (m->block != DST_FP8_ROW && m->block != DST_FP8_SQUARE) return DST_ERR_INVALID_ARG;
    if (m->rows > kMaxCols || m->cols > kMaxCols) return DST_ERR_UNSUPPORTED;
    if (m->ld % 16 != 0 || m->ld_scale < (m->cols + 511) / 512) return DST_ERR_INVALID_ARG;
    if (m->rows > 0 && m->cols > 0 && (!m->q || !m->scale || misaligned(m->q, 16) || misaligned(m->scale, 16))) return DST_ERR_INVALID_ARG;
    v = Fp8View{static_cast<uint8_t*>(m->q), static_cast<uint8_t*>(m->scale), (long long)m->rows, (long long)m->cols, (long long)m->ld,
                (long long)m->ld_scale, m->block == DST_FP8_SQUARE};
    return DST_OK;
}

static int fp4_view(const dst_fp4_t* m, Fp8View& v) {
    if (!m || m->rows < 0 || m->cols < 0 || m->ld < (m->cols + 1) / 2) return DST_ERR_INVALID_ARG;
    if (m->rows > kMaxCols || m->cols > kMaxCols) return DST_ERR_UNSUPPORTED;
    if (m->ld % 16 != 0 || m->ld_scale < (m->cols + 127) / 128) return DST_ERR_INVALID_ARG;
    if (m->rows > 0 && m->cols > 0 && (!m->q || !m->scale || misaligned(m->q, 16) || misaligned(m->scale, 16))) return DST_ERR_INVALID_ARG;
    v = Fp8View{static_cast<uint8_t*>(m->q), static_cast<uint8_t*>(m->scale), (long long)m->rows, (long long)m->cols, (long long)m->ld,
                (long long)m->ld_scale, 0};
    return DST_OK;
}

// What the two kinds of matrix differ in, for the host.
struct Eight {
    static constexpr int64_t kScaleCols = 512;               // columns whose scales are one tile
    static int64_t row_bytes(int64_t cols) { return (cols + 15) / 16 * 16; }
    static size_t workspace(long long M, long long N, long long K) { return matmul_fp8_workspace(M, N, K); }
    static size_t bound(long long M, long long N, long long K) { return matmul_fp8_workspace_bound(M, N, K); }
    static constexpr auto matmul = launch_matmul_fp8;
    static constexpr auto quantize = launch_quantize;
    static constexpr auto fused = linear_fp8_fused;
    static constexpr auto linear = launch_linear_fp8_fused;
};
struct Four {
    static constexpr int64_t kScaleCols = 128;
    static int64_t row_bytes(int64_t cols) { return (cols + 31) / 32 * 16; }
    static size_t workspace(long long M, long long N, long long K) { return matmul_fp4_workspace(M, N, K); }
    static size_t bound(long long M, long long N, long long K) { return matmul_fp4_workspace_bound(M, N, K); }
    static constexpr auto matmul = launch_matmul_fp4;
    static constexpr auto quantize = launch_quantize_fp4;
    static constexpr auto fused = linear_fp4_fused;
    static constexpr auto linear = launch_linear_fp4_fused;
};

template <typename KIND>
static int matmul_impl(const Fp8View& va, const Fp8View& vb, void* out, int64_t ldo, int32_t out_type, void* workspace, size_t workspace_bytes,
                       cudaStream_t stream) {
    if (va.cols != vb.cols || !matrix_ok(out, ldo, va.rows, vb.rows, out_type)) return DST_ERR_INVALID_ARG;
    if (va.rows == 0 || vb.rows == 0) return DST_OK;
    if (va.cols == 0)   // an empty sum
        return cudaMemset2DAsync(out, size_t(ldo) * type_size(out_type), 0, size_t(vb.rows) * type_size(out_type), size_t(va.rows), stream) == cudaSuccess
                   ? DST_OK : DST_ERR_CUDA;
    const size_t need = KIND::workspace(va.rows, vb.rows, va.cols);
    if (need > 0 && (!workspace || misaligned(workspace, 256))) return DST_ERR_INVALID_ARG;
    if (workspace_bytes < need) return DST_ERR_WORKSPACE_TOO_SMALL;
    return done(KIND::matmul(va, vb, out, ldo, out_type, workspace, device_sm_count(), stream), need > 0 ? 2 : 1);
}

// the quantised left operand of a linear call in its workspace: q, scales, then the product's own workspace
struct LinearLayout { int64_t ld, ld_scale; size_t off_scale, off_matmul, total; };
template <typename KIND> static LinearLayout linear_layout(int64_t M, int64_t N, int64_t K) {
    LinearLayout L{};
    L.ld = KIND::row_bytes(K);
    L.ld_scale = (K + KIND::kScaleCols - 1) / KIND::kScaleCols;
    L.off_scale = align_up(size_t(M) * size_t(L.ld), 256);
    L.off_matmul = L.off_scale + size_t((M + 127) / 128) * size_t(L.ld_scale) * kScaleTile;
    L.total = L.off_matmul + KIND::bound(M, N, K);
    return L;
}

template <typename KIND>
static int linear_impl(const void* x, int64_t ldx, int32_t x_type, int64_t M, const Fp8View& w, void* out, int64_t ldo, int32_t out_type,
                       void* workspace, size_t workspace_bytes, cudaStream_t stream) {
    if (M > kMaxCols) return DST_ERR_UNSUPPORTED;
    if (!matrix_ok(x, ldx, M, w.cols, x_type) || !matrix_ok(out, ldo, M, w.rows, out_type)) return DST_ERR_INVALID_ARG;
    if (M == 0 || w.rows == 0) return DST_OK;
    const LinearLayout L = linear_layout<KIND>(M, w.rows, w.cols);
    Fp8View a{nullptr, nullptr, (long long)M, w.cols, (long long)L.ld, (long long)L.ld_scale, 0};
    if (w.cols > 0) {
        if (!workspace || misaligned(workspace, 256)) return DST_ERR_INVALID_ARG;
        if (workspace_bytes < L.off_matmul + KIND::workspace(M, w.rows, w.cols)) return DST_ERR_WORKSPACE_TOO_SMALL;
        if (KIND::fused(M, w.rows, w.cols))
            return done(KIND::linear(x, ldx, x_type, M, w, out, ldo, out_type, device_sm_count(), stream), 1);
        a.q = static_cast<uint8_t*>(workspace);
        a.scale = static_cast<uint8_t*>(workspace) + L.off_scale;
        const QuantParams p{x, (long long)ldx, (long long)M, w.cols, a, {}};
        const int rc = done(KIND::quantize(p, x_type, stream), 1);
        if (rc != DST_OK) return rc;
    }
    return matmul_impl<KIND>(a, w, out, ldo, out_type, workspace ? static_cast<char*>(workspace) + L.off_matmul : nullptr,
                             w.cols > 0 ? workspace_bytes - L.off_matmul : 0, stream);
}

}  // namespace dst

using namespace dst;

extern "C" {

int dst_dropout(const void* x, int64_t ldx, int32_t x_type, const void* residual, int64_t ldr, void* out, int64_t ldo,
                int32_t out_type, int64_t rows, int64_t d, float scale, const dst_dropout_t* drop, dst_stream_t stream) {
    if (!dtype_ok(x_type) || !dtype_ok(out_type)) return DST_ERR_UNSUPPORTED;
    if (!drop || !matrix_ok(x, ldx, rows, d, x_type) || !matrix_ok(out, ldo, rows, d, out_type)) return DST_ERR_INVALID_ARG;
    if (residual && !matrix_ok(residual, ldr, rows, d, out_type)) return DST_ERR_INVALID_ARG;
    if (d > kMaxCols || rows > (int64_t(1) << 32)) return DST_ERR_UNSUPPORTED;
    DropoutParams p;
    if (!drop_params(drop, rows, p.drop)) return DST_ERR_INVALID_ARG;
    // in place only where every element stays where it is
    if (out == x && (ldo != ldx || out_type != x_type)) return DST_ERR_INVALID_ARG;
    if (residual && out == residual && ldo != ldr) return DST_ERR_INVALID_ARG;
    if (rows == 0 || d == 0) return DST_OK;
    p.step = UnitStep{};
    p.x = x; p.residual = residual; p.out = out;
    p.ldx = ldx; p.ldr = ldr; p.ldo = ldo; p.rows = rows; p.d = int(d); p.scale = scale;
    return done(launch_dropout(p, x_type, out_type, device_sm_count(), stream), 1);
}

int dst_embed(const void* indices, int64_t n_rows, int32_t index_type, const void* weight, int64_t vocab, int64_t d,
              int32_t weight_type, const float* position, int64_t n_positions, void* out, int32_t out_type, float scale,
              const dst_dropout_t* drop, dst_result_t* result, dst_stream_t stream) {
    if (!index_ok(index_type) || !dtype_ok(weight_type) || !dtype_ok(out_type)) return DST_ERR_UNSUPPORTED;
    if (n_rows < 0 || vocab < 0 || d < 0 || n_positions < 0) return DST_ERR_INVALID_ARG;
    if (d > kMaxCols || vocab > kMaxVocab || n_rows > (int64_t(1) << 32) || n_positions > kMaxCols) return DST_ERR_UNSUPPORTED;
    if (misaligned(indices, index_type == DST_I64 ? 8 : 4) || misaligned(result, 8)) return DST_ERR_INVALID_ARG;
    if (!matrix_ok(weight, d, vocab, d, weight_type) || !matrix_ok(out, d, n_rows, d, out_type) || misaligned(position, 4)) return DST_ERR_INVALID_ARG;
    if (n_rows > 0 && !indices) return DST_ERR_INVALID_ARG;
    if (position && n_positions == 0 && n_rows > 0) return DST_ERR_INVALID_ARG;
    EmbedParams p;
    if (!drop_params(drop, n_rows, p.drop)) return DST_ERR_INVALID_ARG;
    if (result && cudaMemsetAsync(result, 0, sizeof *result, stream) != cudaSuccess) return DST_ERR_CUDA;
    if (n_rows == 0 || d == 0) return DST_OK;
    p.step = UnitStep{};
    p.indices = indices; p.weight = weight; p.position = position; p.out = out; p.result = result;
    p.rows = n_rows; p.vocab = vocab; p.n_positions = n_positions; p.d = int(d); p.scale = scale;
    return done(launch_embed(p, index_type, weight_type, out_type, device_sm_count(), stream), vocab > 0 || result ? 1 : 0);
}

int dst_quantize_fp8(const void* x, int64_t ldx, int32_t x_type, int64_t rows, int64_t cols, const dst_fp8_t* q,
                     const dst_fp8_t* qt, dst_stream_t stream) {
    if (!dtype_ok(x_type)) return DST_ERR_UNSUPPORTED;
    if ((!q && !qt) || !matrix_ok(x, ldx, rows, cols, x_type)) return DST_ERR_INVALID_ARG;
    QuantParams p{x, (long long)ldx, (long long)rows, (long long)cols, {}, {}};
    if (q) {
        const int rc = fp8_view(q, p.q);
        if (rc != DST_OK) return rc;
        if (q->rows != rows || q->cols != cols) return DST_ERR_INVALID_ARG;
    }
    if (qt) {
        const int rc = fp8_view(qt, p.qt);
        if (rc != DST_OK) return rc;
        if (qt->rows != cols || qt->cols != rows || (q && qt->block != q->block)) return DST_ERR_INVALID_ARG;
    }
    if (rows == 0 || cols == 0) return DST_OK;
    return done(launch_quantize(p, x_type, stream), 1);
}

size_t dst_matmul_fp8_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    if (M <= 0 || N <= 0 || K <= 0 || M > kMaxCols || N > kMaxCols || K > kMaxCols) return 0;
    return matmul_fp8_workspace_bound(M, N, K);
}

int dst_matmul_fp8(const dst_fp8_t* a, const dst_fp8_t* b, void* out, int64_t ldo, int32_t out_type, void* workspace,
                   size_t workspace_bytes, dst_stream_t stream) {
    if (!dtype_ok(out_type)) return DST_ERR_UNSUPPORTED;
    Fp8View va, vb;
    int rc = fp8_view(a, va);
    if (rc == DST_OK) rc = fp8_view(b, vb);
    return rc != DST_OK ? rc : matmul_impl<Eight>(va, vb, out, ldo, out_type, workspace, workspace_bytes, stream);
}

size_t dst_linear_fp8_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    if (M <= 0 || N <= 0 || K <= 0 || M > kMaxCols || N > kMaxCols || K > kMaxCols) return 0;
    return linear_layout<Eight>(M, N, K).total;
}

int dst_linear_fp8(const void* x, int64_t ldx, int32_t x_type, int64_t M, const dst_fp8_t* w, void* out, int64_t ldo,
                   int32_t out_type, void* workspace, size_t workspace_bytes, dst_stream_t stream) {
    if (!dtype_ok(x_type) || !dtype_ok(out_type)) return DST_ERR_UNSUPPORTED;
    Fp8View v;
    const int rc = fp8_view(w, v);
    return rc != DST_OK ? rc : linear_impl<Eight>(x, ldx, x_type, M, v, out, ldo, out_type, workspace, workspace_bytes, stream);
}

int dst_quantize_fp4(const void* x, int64_t ldx, int32_t x_type, int64_t rows, int64_t cols, const dst_fp4_t* q, dst_stream_t stream) {
    if (!dtype_ok(x_type)) return DST_ERR_UNSUPPORTED;
    if (!matrix_ok(x, ldx, rows, cols, x_type)) return DST_ERR_INVALID_ARG;
    QuantParams p{x, (long long)ldx, (long long)rows, (long long)cols, {}, {}};
    const int rc = fp4_view(q, p.q);
    if (rc != DST_OK) return rc;
    if (q->rows != rows || q->cols != cols) return DST_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return DST_OK;
    return done(launch_quantize_fp4(p, x_type, stream), 1);
}

size_t dst_matmul_fp4_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    if (M <= 0 || N <= 0 || K <= 0 || M > kMaxCols || N > kMaxCols || K > kMaxCols) return 0;
    return matmul_fp4_workspace_bound(M, N, K);
}

int dst_matmul_fp4(const dst_fp4_t* a, const dst_fp4_t* b, void* out, int64_t ldo, int32_t out_type, void* workspace,
                   size_t workspace_bytes, dst_stream_t stream) {
    if (!dtype_ok(out_type)) return DST_ERR_UNSUPPORTED;
    Fp8View va, vb;
    int rc = fp4_view(a, va);
    if (rc == DST_OK) rc = fp4_view(b, vb);
    return rc != DST_OK ? rc : matmul_impl<Four>(va, vb, out, ldo, out_type, workspace, workspace_bytes, stream);
}

size_t dst_linear_fp4_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    if (M <= 0 || N <= 0 || K <= 0 || M > kMaxCols || N > kMaxCols || K > kMaxCols) return 0;
    return linear_layout<Four>(M, N, K).total;
}

int dst_linear_fp4(const void* x, int64_t ldx, int32_t x_type, int64_t M, const dst_fp4_t* w, void* out, int64_t ldo,
                   int32_t out_type, void* workspace, size_t workspace_bytes, dst_stream_t stream) {
    if (!dtype_ok(x_type) || !dtype_ok(out_type)) return DST_ERR_UNSUPPORTED;
    Fp8View v;
    const int rc = fp4_view(w, v);
    return rc != DST_OK ? rc : linear_impl<Four>(x, ldx, x_type, M, v, out, ldo, out_type, workspace, workspace_bytes, stream);
}

int dst_sample(const void* logits, int64_t ld, int32_t type, int64_t rows, int64_t vocab, const float* uniform,
               const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p, void* tokens,
               int32_t token_type, float* prob, dst_stream_t stream) {
    if (!dtype_ok(type) || !index_ok(token_type)) return DST_ERR_UNSUPPORTED;
    if (!matrix_ok(logits, ld, rows, vocab, type)) return DST_ERR_INVALID_ARG;
    if (vocab > DST_SAMPLE_MAX_VOCAB || rows > (int64_t(1) << 27)) return DST_ERR_UNSUPPORTED;
    if (rows == 0) return DST_OK;
    if (vocab == 0 || !uniform || !tokens) return DST_ERR_INVALID_ARG;      // a row with no entries has no token
    if (misaligned(tokens, token_type == DST_I64 ? 8 : 4) || misaligned(uniform, 4) || misaligned(temperature, 4) ||
        misaligned(top_k, 4) || misaligned(top_p, 4) || misaligned(min_p, 4) || misaligned(prob, 4))
        return DST_ERR_INVALID_ARG;
    const SampleParams p{logits, uniform, temperature, top_k, top_p, min_p, tokens, prob, (long long)ld, (long long)rows,
                         int(vocab), token_type == DST_I64};
    return done(launch_sample(p, type, device_sm_count(), stream), 1);
}

}  // extern "C"
