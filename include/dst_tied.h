/*
 * The other uses of the tied embedding / pre-softmax projection weight (Section 3 of the paper: one [vocab, d]
 * variable read by the embedding lookups and by the projection to the logits):
 *
 *   dst_embed, dst_dropout           rows on the way in, and the value rows dst_densify takes on the way back
 *   dst_quantize_fp8, dst_matmul_fp8,
 *   dst_linear_fp8                   the projection and its gradients in 8-bit floating point; the weight's gradient
 *                                    is the dense partner dst_densify takes
 *   dst_sample                       a token per row of logits
 *
 * Conventions are those of dst.h: device pointers, caller-owned buffers, nothing allocated or synchronised, all work
 * on `stream`, bad arguments refused on the host before anything is enqueued.  A matrix argument has a leading
 * dimension in elements (the distance between rows; at least the number of columns); its rows are contiguous.
 * Element types are dst_dtype_t, index types dst_index_t.  Sizes of zero are valid and do nothing.
 */
#ifndef DST_TIED_H_
#define DST_TIED_H_

#include "dst.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Dropout's random bits are a function of position, never stored: Philox4x32-10 (Salmon et al., "Parallel random
 * numbers: as easy as 1, 2, 3", 2011) with the 64-bit `seed` as key and the counter
 *     (column / 8, row_offset + row, low and high word of the offset).
 * The eight 16-bit halves of its four words, low half first, belong to eight consecutive columns; an element is
 * dropped where its half is below rint(p * 65536), and kept ones are multiplied by 65536 / (65536 - rint(p * 65536)),
 * so that the expectation is exact for the probability actually used.  p = 0 keeps everything, p = 1 drops everything.
 * The offset is `offset` plus, if given, the 64-bit number at `offset_device` when the kernel runs: a captured graph
 * draws new bits on every replay when the program adds to that number in between.
 * row_offset + rows must not exceed 2^32.
 */
typedef struct {
    double p;
    uint64_t seed;
    uint64_t offset;
    const uint64_t* offset_device; /* device memory, or NULL */
    int64_t row_offset;            /* row number of the first row, for a tensor that is handled in parts */
} dst_dropout_t;

/*
 * out[r, c] = (residual ? residual[r, c] : 0) + scale * k[r, c] * x[r, c],   k the kept / dropped factor above.
 * The gradient with respect to x is the same call on the output's gradient (the residual's is that gradient itself).
 * x [rows, d] has x_type; residual and out have out_type.  `out` may be x or residual where type and leading dimension
 * agree; it must not overlap them otherwise.  fp32 arithmetic, rounded once.  A dropped element contributes zero
 * whatever its value.
 */
int dst_dropout(const void* x, int64_t ldx, int32_t x_type, const void* residual, int64_t ldr, void* out, int64_t ldo,
                int32_t out_type, int64_t rows, int64_t d, float scale, const dst_dropout_t* drop, dst_stream_t stream);

/*
 * out[i, c] = k[i, c] * (scale * weight[indices[i], c] + (position ? position[i % n_positions, c] : 0))
 * indices [n_rows]; weight [vocab, d] contiguous in weight_type; position [n_positions, d] contiguous fp32 or NULL;
 * out [n_rows, d] contiguous in out_type; drop NULL: k = 1.  A row whose index lies outside [0, vocab) is written as
 * zeros and counted in `result` (optional DEVICE memory, cleared by this call: status and n_out_of_range are set); with
 * vocab = 0 that is every row.
 * The value rows of this lookup's IndexedSlices gradient are dst_dropout(grad, scale, the same drop).
 */
int dst_embed(const void* indices, int64_t n_rows, int32_t index_type, const void* weight, int64_t vocab, int64_t d,
              int32_t weight_type, const float* position, int64_t n_positions, void* out, int32_t out_type, float scale,
              const dst_dropout_t* drop, dst_result_t* result, dst_stream_t stream);

/*
 * A matrix [rows, cols] in 8-bit floating point (4 exponent bits, 3 mantissa bits, largest value 448) with one scale, a
 * power of two, for each block: DST_FP8_ROW blocks are 128 consecutive columns of one row, DST_FP8_SQUARE blocks are
 * 128 rows by 128 columns (the last ones smaller).  The element stands for q * scale.
 *   q      [rows, ld], 16-byte aligned, ld a multiple of 16
 *   scale  one byte for each row and column block, the exponent plus 127 (255: NaN), whatever the kind of block, in the
 *          order in which the tensor cores take them: tiles of 512 bytes for 128 rows by 4 column blocks; the byte of
 *          row r and column block b is at (r % 32) * 16 + (r / 32 % 4) * 4 + b % 4 of tile (r / 128) * ld_scale + b / 4.
 *          ld_scale (tiles for 128 rows) is at least the number of column blocks / 4, rounded up; 16-byte aligned.
 */
typedef enum { DST_FP8_ROW = 0, DST_FP8_SQUARE = 1 } dst_fp8_block_t;
typedef struct {
    void* q;
    void* scale;
    int64_t rows, cols, ld, ld_scale;
    int32_t block; /* dst_fp8_block_t */
    int32_t reserved;
} dst_fp8_t;

/*
 * Quantise x [rows, cols] (fp32 or bf16).  The scale of a block is the smallest power of two 2^e with
 * max|x| <= 448 * 2^e (max|x| taken as at least 2^-100), so that the scaling is exact and the one rounding is the
 * one to 8 bits, to nearest even.  A block that holds an infinity or a NaN gets the scale NaN.
 * `q` receives x, `qt` its transpose [cols, rows] with blocks of its own (ROW: 128 consecutive rows of x of one
 * column); either may be NULL, both cost one read of x.  Their block kinds must agree.
 */
int dst_quantize_fp8(const void* x, int64_t ldx, int32_t x_type, int64_t rows, int64_t cols, const dst_fp8_t* q,
                     const dst_fp8_t* qt, dst_stream_t stream);

/*
 * out[m, n] = sum over column blocks b of a.scale(m, b) * b.scale(n, b) * sum_{k in b} a.q[m, k] * b.q[n, k]
 * a [M, K], b [N, K], out [M, N] in out_type (fp32 or bf16, rounded once).  All sums are fp32 in an order fixed by the
 * shapes and out_type.  The tensor cores' own additions truncate; an fp32 result leaves them every six blocks of 128 and is
 * added up to nearest from there, a bf16 result (whose own rounding is 2^-9) only at the end of the inner dimension, or of the
 * parts that it is cut into where the tiles are few: before its rounding it may be off by the order of 2^-23 of the largest
 * partial sum for every 32 elements (6.3e-5 where one block outweighs the 15,616 elements after it).  K = 0 gives zeros.  workspace: dst_matmul_fp8_workspace_bytes(M, N, K) bytes (may be 0), 256-byte aligned;
 * as much is enough for every smaller M, N and K too.  A device-side wait that gives up leaves NaN in the part of `out`
 * that was still to be written.
 */
size_t dst_matmul_fp8_workspace_bytes(int64_t M, int64_t N, int64_t K);
int dst_matmul_fp8(const dst_fp8_t* a, const dst_fp8_t* b, void* out, int64_t ldo, int32_t out_type, void* workspace,
                   size_t workspace_bytes, dst_stream_t stream);

/*
 * out[m, n] = sum_k x[m, k] w[n, k] with x quantised on the way (ROW blocks): dst_quantize_fp8 and dst_matmul_fp8 in one
 * call, and for a few rows (up to 40 blocks of 128 elements, of up to 2048 columns) in one kernel.
 */
size_t dst_linear_fp8_workspace_bytes(int64_t M, int64_t N, int64_t K);
int dst_linear_fp8(const void* x, int64_t ldx, int32_t x_type, int64_t M, const dst_fp8_t* w, void* out, int64_t ldo,
                   int32_t out_type, void* workspace, size_t workspace_bytes, dst_stream_t stream);

/*
 * Draw one token per row of logits [rows, vocab] (fp32 or bf16) from given uniform numbers.  Per row, with x the
 * logits as fp32 and m their maximum:
 *   z_i = (x_i - m) * (1 / temperature), 0 where x_i == m;  e_i = exp(z_i);  w_i = rint(2^31 * e_i)
 *   top_k   keeps the top_k largest logits (equal ones: lowest index first); 0 or less: all
 *   top_p   keeps, of those in descending order, the ones before which less than floor(top_p * S) has been summed,
 *           S the sum of w over what top_k kept; always at least one; 1 or more: all
 *   min_p   keeps the ones with e_i >= min(min_p, 1)
 *   token   the lowest index at which the sum of w over kept indices up to it exceeds floor(uniform * their sum)
 *   prob    (optional) w_token / that sum
 * The weights are whole numbers and every sum is exact in 64 bits, so the token depends on the inputs alone: not on
 * how a row is split over threads, nor on what else is in the batch.  top_p and uniform are used to 24 bits (rounded
 * down).  temperature of 0 (or anything not above 0) takes the largest logit, the lowest index among equals.
 * Logits of -infinity and NaN are never drawn; +infinity shares all mass.  A row with nothing left gives token -1 and
 * prob 0.  temperature, top_k, top_p, min_p: [rows] or NULL (1, off, off, off).  vocab <= DST_SAMPLE_MAX_VOCAB.
 */
#define DST_SAMPLE_MAX_VOCAB 327680
int dst_sample(const void* logits, int64_t ld, int32_t type, int64_t rows, int64_t vocab, const float* uniform,
               const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p, void* tokens,
               int32_t token_type, float* prob, dst_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* DST_TIED_H_ */
