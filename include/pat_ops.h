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

#ifdef __cplusplus
}
#endif

#endif /* PAT_OPS_H_ */
