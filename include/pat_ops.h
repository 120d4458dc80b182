/*
 * pat_ops.h -- operators for what stands on either side of the collectives of
 * pat.h in a program whose parameters are sharded over ranks: weights are
 * gathered, multiplied and looked up; gradients are formed and reduce-scattered.
 *
 *   - 4-bit block floating point: shards are quantised before an all-gather
 *     (4.25 bits a value instead of 16 or 32), and the gathered codes are
 *     widened or multiplied as they are.  Rows are independent, so the
 *     concatenation of ranks' codes and scales is the whole matrix's.
 *   - embedding lookup on a whole table or a rank's shard of its rows, and its
 *     dense gradient, which a reduce-scatter sums.
 *   - dropout whose mask is a function of a seed and of an element's index in
 *     the whole tensor, so that shards reproduce the whole's mask.
 *   - activations in 8-bit blocks, as inputs of products with the 4-bit weights
 *     and as checkpoints that a backward pass forms gradients from.
 *   - root-mean-square norm of a residual stream and the gated feed-forward
 *     block, with their gradients.
 *
 * Conventions, beside those of pat.h:
 *   - Matrices are row-major, `*_stride` is the distance of rows in ELEMENTS,
 *     at least the row's length; element-aligned addresses are enough.
 *   - Sums, scales and products are computed in float32 and rounded once
 *     (nearest even) to the output's type.
 *   - All buffers are device memory on the current device, owned by the caller
 *     and valid until `stream` has finished the call.  Calls are asynchronous
 *     and ordered on `stream`; they allocate nothing and keep nothing, so they
 *     can run on any number of streams and be captured into graphs.
 *   - A `workspace` is uninitialised device memory, 16-byte aligned, of at
 *     least the bytes that the operator's *_workspace function says (0: none
 *     is needed, NULL is accepted); its contents mean nothing after the call.
 *     Calls that may overlap need one each.  Fewer bytes: PAT_ERR_TOO_LARGE.
 *   - An output that overlaps an input or the workspace is
 *     PAT_ERR_INVALID_ARGUMENT, except where in place is named.  Columns of
 *     one matrix beside each other do not overlap; matrices of different
 *     strides (in bytes) whose rows alternate count as if they did.
 *   - Nothing is launched when an output has no elements.  Buffers without
 *     elements may be NULL.  Row and column counts are below 2^31.
 *   - Results are deterministic: no sum depends on the order of execution.
 */
#ifndef PAT_OPS_H_
#define PAT_OPS_H_

#include "pat.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * 4-bit block floating point (the MXFP4 encoding of the OCP Microscaling
 * Formats specification 1.0): 32 consecutive values of a row share a scale
 * 2^(s - 127), s one byte; a value is a 4-bit code of sign, 2 exponent bits and
 * 1 mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6.
 *
 * Stored form of a rows x cols matrix, with G = ceil(cols / 128):
 *   codes  [rows][64 * G] bytes, value 2i of a row in the low half of byte i;
 *          16-byte aligned;
 *   scales [rows][4 * G] bytes, one for each 32 values; 4-byte aligned.
 * Rows are filled up to whole groups of 128 values, codes and scales with
 * zeros, so every kernel may read whole groups, and both buffers of any number
 * of rows are whole 32-bit words: pat_allgather moves them as PAT_INT32.
 * Fewer than 2^31 groups in all (rows * G, else PAT_ERR_UNSUPPORTED).
 */
#define PAT_MX_GROUP 128
#define PAT_MX_CODE_BYTES(cols) (((size_t)(cols) + 127) / 128 * 64)
#define PAT_MX_SCALE_BYTES(cols) (((size_t)(cols) + 127) / 128 * 4)

/*
 * Quantises x[rows][cols] (PAT_FLOAT32 or PAT_BFLOAT16).  Per block, with E the
 * exponent field of the largest magnitude: s = max(E - 2, 0); code = the nearest
 * 4-bit value of x * 2^(127 - s), ties to the even code, 6 at most.  A block
 * that holds an infinity or a NaN gets s = 255 and stands for NaN in whole.
 */
pat_status_t pat_mx_quantize(const void* x, int64_t x_stride, size_t rows, size_t cols, pat_dtype_t dtype, void* codes,
                             void* scales, hipStream_t stream);

/* out[r][c] = the value that the stored form stands for (exact in both types). */
pat_status_t pat_mx_dequantize(const void* codes, const void* scales, size_t rows, size_t cols, void* out,
                               int64_t out_stride, pat_dtype_t dtype, hipStream_t stream);

/*
 * out[i][j] = sum over x < k of a[i][x] * b[j][x]: a (m rows) and b (n rows) in
 * the stored form, both of k columns; out PAT_FLOAT32 or PAT_BFLOAT16.  All
 * products here: fewer than 2^26 rows and columns of the output and 2^30 tiles of
 * 16 x 16 of it, 2^24 terms of a sum (else PAT_ERR_UNSUPPORTED).
 */
pat_status_t pat_mx_matmul(const void* a_codes, const void* a_scales, const void* b_codes, const void* b_scales, size_t m,
                           size_t n, size_t k, void* out, int64_t out_stride, pat_dtype_t dtype, hipStream_t stream);

/*
 * The same product of Q(x), where Q is pat_mx_quantize, with a weight w of n rows
 * in the stored form: out[i][j] = sum over c < k of Q(x)[i][c] * w[j][c].  Few
 * rows (single tokens, small batches) take one launch, which quantises x on its
 * way; the result is that of the two calls to the bit either way.
 */
pat_status_t pat_mx_linear(const void* x, int64_t x_stride, pat_dtype_t x_dtype, const void* w_codes, const void* w_scales,
                           size_t m, size_t n, size_t k, void* out, int64_t out_stride, pat_dtype_t dtype, void* workspace,
                           size_t workspace_bytes, hipStream_t stream);
size_t pat_mx_linear_workspace(size_t m, size_t n, size_t k);

/*
 * The product that both gradients of pat_mx_matmul are, straight through the
 * quantisation:
 *   transposed == 0: out[i][c] = sum over j < inner of g[i][j] * q[j][c],  g [rows][inner]
 *   transposed != 0: out[i][c] = sum over j < inner of g[j][i] * q[j][c],  g [inner][rows]
 * q: `inner` rows of `cols` columns in the stored form.  For out = a b^T with its
 * gradient g [m][n]: d a = (g, q = b), d b = (g, q = a, transposed).
 * g is PAT_BFLOAT16 (the matrix units' type; float32 gradients are rounded by the
 * caller); out PAT_FLOAT32 or PAT_BFLOAT16.  A value of q is exact in bfloat16.
 */
pat_status_t pat_mx_matmul_grad(const void* g, int64_t g_stride, int transposed, const void* q_codes, const void* q_scales,
                                size_t rows, size_t inner, size_t cols, void* out, int64_t out_stride, pat_dtype_t dtype,
                                void* workspace, size_t workspace_bytes, hipStream_t stream);
size_t pat_mx_matmul_grad_workspace(size_t rows, size_t inner, size_t cols);

/*
 * Embedding lookup: out[t][c] = scale * table[tokens[t] - first][c], zero where
 * tokens[t] is not in [first, first + rows).  table: rows x cols, the whole one
 * (first = 0) or a rank's rows of it (the ranks' outputs then sum to the whole's:
 * a reduce-scatter joins them).  tokens: PAT_INT32 (token_bytes = 4) or 64-bit
 * integers (token_bytes = 8); dtypes PAT_FLOAT32 or PAT_BFLOAT16, each on its own.
 */
pat_status_t pat_embedding(const void* tokens, int token_bytes, size_t ntokens, const void* table, int64_t table_stride,
                           pat_dtype_t table_dtype, int64_t first, size_t rows, size_t cols, float scale, void* out,
                           int64_t out_stride, pat_dtype_t dtype, hipStream_t stream);

/*
 * Its gradient, dense: out[v][c] = scale * sum of g[t][c] over the t with
 * tokens[t] == first + v, 0 where there is none.  g: ntokens x cols; out: rows x
 * cols, every element written.  A row's sum runs over its tokens in rising t, in
 * pieces whose partial sums are added in order.
 * Fewer than 2^28 tokens and rows, 2^23 columns (else PAT_ERR_UNSUPPORTED).
 */
pat_status_t pat_embedding_grad(const void* tokens, int token_bytes, size_t ntokens, const void* g, int64_t g_stride,
                                pat_dtype_t g_dtype, int64_t first, size_t rows, size_t cols, float scale, void* out,
                                int64_t out_stride, pat_dtype_t dtype, void* workspace, size_t workspace_bytes,
                                hipStream_t stream);
size_t pat_embedding_grad_workspace(size_t ntokens, size_t rows, size_t cols);

/*
 * Dropout: out[r][c] = keep(i) ? x[r][c] * 65536 / (65536 - P) : 0, plus
 * residual[r][c] where a residual is given (NULL: none); P = round(65536 * p),
 * i = index + r * index_stride + c the element's index in the whole tensor (modulo
 * 2^64).  keep(i): the 16 bits at place i mod 8 of the Philox4x32-10 output words
 * (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011)
 * of counter (i div 8, 0) and key `seed` are >= P; places run from the low half of
 * the first word to the high half of the last.  A rank that holds rows or columns
 * of a tensor gets the whole's mask by giving its place; the gradient is the same
 * call on the output's gradient.  p in [0, 1]; a dropped element gives 0 whatever x
 * is.  One dtype (PAT_FLOAT32 or PAT_BFLOAT16) for all.
 * In place: out == x, or out == residual, with equal strides.
 */
pat_status_t pat_dropout(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, void* out,
                         int64_t out_stride, size_t rows, size_t cols, pat_dtype_t dtype, double p, uint64_t seed,
                         uint64_t index, uint64_t index_stride, hipStream_t stream);

/*
 * 8-bit blocks, for activations: 32 consecutive values of a row share a scale
 * 2^(s - 127), s one byte; a value is an 8-bit code of sign, 4 exponent bits (bias
 * 7) and 3 mantissa bits, 448 at most, steps of 2^-9 the smallest (the E4M3
 * element of the OCP Microscaling Formats specification 1.0).  The quantisation
 * here uses codes up to 3.75.  The matrix instructions add products in eights and
 * keep 13 bits below the exponent of the largest, as measured; up to 3.75 the
 * products with 4-bit codes, multiples of 2^-10 below 2^5, all keep theirs, and
 * sums are float32's.  A block whose values go up to 448 is taken too; its
 * products lose up to 2^-13 of the largest of eight each.
 *
 * Stored form of a rows x cols matrix, with G = ceil(cols / 128):
 *   codes  [rows][128 * G] bytes; 16-byte aligned;
 *   scales [rows][4 * G] bytes, one for each 32 values; 4-byte aligned.
 * Rows are filled up with zeros, and rows * G < 2^31, as for 4-bit blocks.
 */
#define PAT_MXB_CODE_BYTES(cols) (((size_t)(cols) + 127) / 128 * 128)
#define PAT_MXB_SCALE_BYTES(cols) PAT_MX_SCALE_BYTES(cols)

/*
 * Quantises x[rows][cols] (PAT_FLOAT32 or PAT_BFLOAT16).  Per block: s = the least,
 * from 0, for which no magnitude is above 3.75 * 2^(s - 127); code = the nearest value
 * of x * 2^(127 - s), ties to the even code.  Off by half a step at most: 2^-4 of the value
 * from 2^-6 * 2^(s - 127) on, which is, where s > 0, at least down to 1/120 of the block's
 * largest magnitude, and 2^-10 * 2^(s - 127) below.  A block that holds an infinity or a
 * NaN gets s = 255 and stands for NaN in whole.
 */
pat_status_t pat_mxb_quantize(const void* x, int64_t x_stride, size_t rows, size_t cols, pat_dtype_t dtype, void* codes,
                              void* scales, hipStream_t stream);

/*
 * out[r][c] = the value that the stored form stands for: exact in float32 but for values of 2^128 and above, which are
 * infinite there (magnitudes from 1.9375 * 2^127 quantise to 2^128), and in bfloat16 down to 2^-126.
 */
pat_status_t pat_mxb_dequantize(const void* codes, const void* scales, size_t rows, size_t cols, void* out,
                                int64_t out_stride, pat_dtype_t dtype, hipStream_t stream);

/*
 * out[i][j] = sum over c < k of x[i][c] * w[j][c], plus residual[i][j] where a
 * residual is given (NULL: none): x (m rows) in 8-bit blocks, w (n rows) in 4-bit
 * blocks, residual of the output's type.  In place: out == residual with equal
 * strides.  Sizes: as pat_mx_matmul.
 */
pat_status_t pat_mxb_linear(const void* x_codes, const void* x_scales, const void* w_codes, const void* w_scales, size_t m,
                            size_t n, size_t k, const void* residual, int64_t residual_stride, void* out,
                            int64_t out_stride, pat_dtype_t dtype, hipStream_t stream);

/*
 * A weight's gradient from the 8-bit checkpoint of its input: out[i][c] = sum over
 * j < inner of g[j][i] * x[j][c], g [inner][rows] PAT_BFLOAT16, x `inner` rows of
 * `cols` columns in 8-bit blocks (widened to bfloat16).  Otherwise as
 * pat_mx_matmul_grad.
 */
pat_status_t pat_mxb_weight_grad(const void* g, int64_t g_stride, const void* x_codes, const void* x_scales, size_t rows,
                                 size_t inner, size_t cols, void* out, int64_t out_stride, pat_dtype_t dtype,
                                 void* workspace, size_t workspace_bytes, hipStream_t stream);
size_t pat_mxb_weight_grad_workspace(size_t rows, size_t inner, size_t cols);

/* The activation of a gated block: a / (1 + e^-a), or a * (1 + erf(a / sqrt 2)) / 2. */
typedef enum { PAT_SILU = 0, PAT_GELU = 1 } pat_activation_t;

/*
 * The first half of a gated feed-forward block: out[i][j] = act(a[i][j]) * b[i][j]
 * with a[i][j] = sum over c < k of x[i][c] * w[j][c] and b[i][j] the same of w[n + j]:
 * x (m rows) in 8-bit blocks, w (2 n rows, the gate's before the others) in 4-bit
 * blocks.  a and b are not rounded before the activation and the product.
 * The output is either `out`, PAT_FLOAT32 or PAT_BFLOAT16, or, where out is NULL,
 * 8-bit blocks in out_codes and out_scales (`dtype` and out_stride are not looked at).
 * saved_codes, saved_scales: both NULL, or a checkpoint for pat_gated_grad, 8-bit
 * blocks of 2 m rows of n columns: a, then b.
 * Sizes: as pat_mx_matmul with 2 n columns.
 */
pat_status_t pat_gated(const void* x_codes, const void* x_scales, const void* w_codes, const void* w_scales, size_t m,
                       size_t n, size_t k, pat_activation_t act, void* out, int64_t out_stride, pat_dtype_t dtype,
                       void* out_codes, void* out_scales, void* saved_codes, void* saved_scales, hipStream_t stream);

/*
 * Its gradient with respect to a and b, from the checkpoint: with g[m][n] the
 * output's gradient (PAT_FLOAT32 or PAT_BFLOAT16),
 *   out[i][j] = g[i][j] * b[i][j] * act'(a[i][j]),  out[i][n + j] = g[i][j] * act(a[i][j]),
 * out [m][2 n] PAT_BFLOAT16: what pat_mx_matmul_grad takes with w for the gradient of
 * x, and pat_mxb_weight_grad with x for that of w.
 */
pat_status_t pat_gated_grad(const void* g, int64_t g_stride, pat_dtype_t g_dtype, const void* saved_codes,
                            const void* saved_scales, size_t m, size_t n, pat_activation_t act, void* out,
                            int64_t out_stride, hipStream_t stream);

/*
 * Root-mean-square norm: t = x, or x + residual rounded to `dtype` where a residual
 * is given (NULL: none), and stored in `total` where that is not NULL;
 * out[r][c] = t[r][c] * weight[c] / sqrt(mean over c of t[r][c]^2 + eps), eps >= 0.
 * x, residual and total: dtype; weight: cols elements of weight_dtype; the output:
 * `out` of out_dtype, or, where out is NULL, 8-bit blocks in out_codes and out_scales.
 * Squares are summed in float32, to its full precision in rows whose sum of squares is
 * at most 2^127 and whose mean of squares plus eps is at least 2^-126.  Sums that
 * overflow, from 2^128 on, give a row of zeros; squares that vanish, below 2^-149, count
 * as zero, so that with eps = 0 a row of such values gives infinities or NaN.
 * In place: total or out == x, total or out == residual, with equal strides and types;
 * total and out are two buffers.
 */
pat_status_t pat_rms_norm(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, pat_dtype_t dtype,
                          const void* weight, pat_dtype_t weight_dtype, size_t rows, size_t cols, float eps, void* total,
                          int64_t total_stride, void* out, int64_t out_stride, pat_dtype_t out_dtype, void* out_codes,
                          void* out_scales, hipStream_t stream);

/*
 * Its gradients, x being t above (the stored total): with r = 1 / sqrt(mean x^2 + eps),
 *   out[r][c] = r * (g * weight - x * r^2 * mean over c of g * weight * x) + total_grad[r][c],
 *   dweight[c] = sum over rows of g * x * r  (PAT_FLOAT32, cols elements, 4-byte aligned).
 * out is the gradient of x and of the residual alike; total_grad (NULL: none) is what
 * reaches the total from elsewhere.  g, total_grad and out: dtype; x: x_dtype.  Sums are
 * float32's, in the norm's range; the magnitudes of g * weight * x, too, may sum to 2^127
 * at most in a row.  With no rows dweight is zero.
 * In place: out == g or out == total_grad with equal strides.
 * Fewer than 2^28 rows, 2^26 columns (else PAT_ERR_UNSUPPORTED).
 */
pat_status_t pat_rms_norm_grad(const void* g, int64_t g_stride, pat_dtype_t dtype, const void* x, int64_t x_stride,
                               pat_dtype_t x_dtype, const void* weight, pat_dtype_t weight_dtype, const void* total_grad,
                               int64_t total_grad_stride, size_t rows, size_t cols, float eps, void* out, int64_t out_stride,
                               void* dweight, void* workspace, size_t workspace_bytes, hipStream_t stream);
size_t pat_rms_norm_grad_workspace(size_t rows, size_t cols);

#ifdef __cplusplus
}
#endif

#endif /* PAT_OPS_H_ */
