// C entry points of pat_ops.h: argument checks, then one launch function each.
// Nothing here allocates or throws.
#include "ops_args.hpp"

extern "C" {

pat_status_t pat_mx_quantize(const void* x, int64_t x_stride, size_t rows, size_t cols, pat_dtype_t dtype, void* codes,
                             void* scales, hipStream_t stream) {
  Elem e;
  if (!elem_of(dtype, &e)) return PAT_ERR_UNSUPPORTED;
  if (!dims_ok(rows, cols) || !groups_ok(rows, cols)) return PAT_ERR_UNSUPPORTED;
  if (rows == 0 || cols == 0) return PAT_OK;
  Span in, c, s;
  if (!matrix_span(x, x_stride, rows, cols, elem_bytes(e), &in) || !mx_spans(codes, scales, rows, cols, &c, &s))
    return PAT_ERR_INVALID_ARGUMENT;
  if (any_overlap(c, {in, s}) || overlap(s, in)) return PAT_ERR_INVALID_ARGUMENT;
  return launched(pat::launch_mx_quantize({x, x_stride}, e, int64_t(rows), int64_t(cols), static_cast<uint8_t*>(codes),
                                          static_cast<uint8_t*>(scales), stream));
}

pat_status_t pat_mx_dequantize(const void* codes, const void* scales, size_t rows, size_t cols, void* out,
                               int64_t out_stride, pat_dtype_t dtype, hipStream_t stream) {
  Elem e;
  if (!elem_of(dtype, &e)) return PAT_ERR_UNSUPPORTED;
  if (!dims_ok(rows, cols) || !groups_ok(rows, cols)) return PAT_ERR_UNSUPPORTED;
  if (rows == 0 || cols == 0) return PAT_OK;
  Span o, c, s;
  if (!matrix_span(out, out_stride, rows, cols, elem_bytes(e), &o) || !mx_spans(codes, scales, rows, cols, &c, &s))
    return PAT_ERR_INVALID_ARGUMENT;
  if (any_overlap(o, {c, s})) return PAT_ERR_INVALID_ARGUMENT;
  return launched(pat::launch_mx_dequantize({static_cast<const uint8_t*>(codes), static_cast<const uint8_t*>(scales)},
                                            int64_t(rows), int64_t(cols), {out, out_stride}, e, stream));
}

pat_status_t pat_mx_matmul(const void* a_codes, const void* a_scales, const void* b_codes, const void* b_scales, size_t m,
                           size_t n, size_t k, void* out, int64_t out_stride, pat_dtype_t dtype, hipStream_t stream) {
  Elem e;
  if (!elem_of(dtype, &e)) return PAT_ERR_UNSUPPORTED;
  if (!product_ok(m, n, k) || !groups_ok(m, k) || !groups_ok(n, k)) return PAT_ERR_UNSUPPORTED;
  if (m == 0 || n == 0) return PAT_OK;
  Span ac, as, bc, bs, o;
  if (!mx_spans(a_codes, a_scales, m, k, &ac, &as) || !mx_spans(b_codes, b_scales, n, k, &bc, &bs) ||
      !matrix_span(out, out_stride, m, n, elem_bytes(e), &o))
    return PAT_ERR_INVALID_ARGUMENT;
  if (any_overlap(o, {ac, as, bc, bs})) return PAT_ERR_INVALID_ARGUMENT;
  return launched(pat::launch_mx_matmul({static_cast<const uint8_t*>(a_codes), static_cast<const uint8_t*>(a_scales)},
                                        {static_cast<const uint8_t*>(b_codes), static_cast<const uint8_t*>(b_scales)},
                                        int64_t(m), int64_t(n), int64_t(k), {out, out_stride}, e, stream));
}

size_t pat_mx_linear_workspace(size_t m, size_t n, size_t k) {
  if (!product_ok(m, n, k) || !m || !n || !groups_ok(m, k)) return 0;
  return pat::mx_linear_workspace(int64_t(m), int64_t(n), int64_t(k));
}

pat_status_t pat_mx_linear(const void* x, int64_t x_stride, pat_dtype_t x_dtype, const void* w_codes, const void* w_scales,
                           size_t m, size_t n, size_t k, void* out, int64_t out_stride, pat_dtype_t dtype, void* workspace,
                           size_t workspace_bytes, hipStream_t stream) {
  Elem xe, e;
  if (!elem_of(x_dtype, &xe) || !elem_of(dtype, &e)) return PAT_ERR_UNSUPPORTED;
  if (!product_ok(m, n, k) || !groups_ok(m, k) || !groups_ok(n, k)) return PAT_ERR_UNSUPPORTED;
  if (m == 0 || n == 0) return PAT_OK;
  Span in, wc, ws, o, w;
  if (!matrix_span(x, x_stride, m, k, elem_bytes(xe), &in) || !mx_spans(w_codes, w_scales, n, k, &wc, &ws) ||
      !matrix_span(out, out_stride, m, n, elem_bytes(e), &o))
    return PAT_ERR_INVALID_ARGUMENT;
  if (pat_status_t st = workspace_span(workspace, workspace_bytes, pat_mx_linear_workspace(m, n, k), &w)) return st;
  if (any_overlap(o, {in, wc, ws, w}) || any_overlap(w, {in, wc, ws})) return PAT_ERR_INVALID_ARGUMENT;
  return launched(pat::launch_mx_linear({x, x_stride}, xe,
                                        {static_cast<const uint8_t*>(w_codes), static_cast<const uint8_t*>(w_scales)},
                                        int64_t(m), int64_t(n), int64_t(k), {out, out_stride}, e, workspace, stream));
}

size_t pat_mx_matmul_grad_workspace(size_t rows, size_t inner, size_t cols) {
  if (!product_ok(rows, cols, inner) || !rows || !cols) return 0;
  return pat::mx_grad_workspace(int64_t(rows), int64_t(inner), int64_t(cols));
}

pat_status_t pat_mx_matmul_grad(const void* g, int64_t g_stride, int transposed, const void* q_codes, const void* q_scales,
                                size_t rows, size_t inner, size_t cols, void* out, int64_t out_stride, pat_dtype_t dtype,
                                void* workspace, size_t workspace_bytes, hipStream_t stream) {
  Elem e;
  if (!elem_of(dtype, &e)) return PAT_ERR_UNSUPPORTED;
  if (!product_ok(rows, cols, inner) || !groups_ok(inner, cols)) return PAT_ERR_UNSUPPORTED;
  if (rows == 0 || cols == 0) return PAT_OK;
  Span in, qc, qs, o, w;
  if (!matrix_span(g, g_stride, transposed ? inner : rows, transposed ? rows : inner, 2, &in) ||
      !mx_spans(q_codes, q_scales, inner, cols, &qc, &qs) || !matrix_span(out, out_stride, rows, cols, elem_bytes(e), &o))
    return PAT_ERR_INVALID_ARGUMENT;
  if (pat_status_t st = workspace_span(workspace, workspace_bytes, pat_mx_matmul_grad_workspace(rows, inner, cols), &w))
    return st;
  if (any_overlap(o, {in, qc, qs, w}) || any_overlap(w, {in, qc, qs})) return PAT_ERR_INVALID_ARGUMENT;
  return launched(pat::launch_mx_grad({g, g_stride}, transposed != 0,
                                      {static_cast<const uint8_t*>(q_codes), static_cast<const uint8_t*>(q_scales)},
                                      int64_t(rows), int64_t(inner), int64_t(cols), {out, out_stride}, e, workspace,
                                      stream));
}

pat_status_t pat_embedding(const void* tokens, int token_bytes, size_t ntokens, const void* table, int64_t table_stride,
                           pat_dtype_t table_dtype, int64_t first, size_t rows, size_t cols, float scale, void* out,
                           int64_t out_stride, pat_dtype_t dtype, hipStream_t stream) {
  Elem te, e;
  if (!elem_of(table_dtype, &te) || !elem_of(dtype, &e)) return PAT_ERR_UNSUPPORTED;
  if (token_bytes != 4 && token_bytes != 8) return PAT_ERR_UNSUPPORTED;
  if (!dims_ok(ntokens, rows, cols)) return PAT_ERR_UNSUPPORTED;
  if (ntokens == 0 || cols == 0) return PAT_OK;
  Span tk, tb, o;
  if (!span_of(tokens, ntokens * size_t(token_bytes), size_t(token_bytes), &tk) ||
      !matrix_span(table, table_stride, rows, cols, elem_bytes(te), &tb) ||
      !matrix_span(out, out_stride, ntokens, cols, elem_bytes(e), &o))
    return PAT_ERR_INVALID_ARGUMENT;
  if (any_overlap(o, {tk, tb})) return PAT_ERR_INVALID_ARGUMENT;
  return launched(pat::launch_embedding(tokens, token_bytes, int64_t(ntokens), {table, table_stride}, te, first,
                                        int64_t(rows), int64_t(cols), scale, {out, out_stride}, e, stream));
}

size_t pat_embedding_grad_workspace(size_t ntokens, size_t rows, size_t cols) {
  if (!grad_dims_ok(ntokens, rows, cols) || !rows || !cols) return 0;
  return pat::embedding_grad_workspace(int64_t(ntokens), int64_t(rows), int64_t(cols));
}

pat_status_t pat_embedding_grad(const void* tokens, int token_bytes, size_t ntokens, const void* g, int64_t g_stride,
                                pat_dtype_t g_dtype, int64_t first, size_t rows, size_t cols, float scale, void* out,
                                int64_t out_stride, pat_dtype_t dtype, void* workspace, size_t workspace_bytes,
                                hipStream_t stream) {
  Elem ge, e;
  if (!elem_of(g_dtype, &ge) || !elem_of(dtype, &e)) return PAT_ERR_UNSUPPORTED;
  if (token_bytes != 4 && token_bytes != 8) return PAT_ERR_UNSUPPORTED;
  if (!grad_dims_ok(ntokens, rows, cols)) return PAT_ERR_UNSUPPORTED;
  if (rows == 0 || cols == 0) return PAT_OK;
  Span tk, in, o, w;
  if (!span_of(tokens, ntokens * size_t(token_bytes), size_t(token_bytes), &tk) ||
      !matrix_span(g, g_stride, ntokens, cols, elem_bytes(ge), &in) ||
      !matrix_span(out, out_stride, rows, cols, elem_bytes(e), &o))
    return PAT_ERR_INVALID_ARGUMENT;
  if (pat_status_t st = workspace_span(workspace, workspace_bytes, pat_embedding_grad_workspace(ntokens, rows, cols), &w))
    return st;
  if (any_overlap(o, {tk, in, w}) || any_overlap(w, {tk, in})) return PAT_ERR_INVALID_ARGUMENT;
  return launched(pat::launch_embedding_grad(tokens, token_bytes, int64_t(ntokens), {g, g_stride}, ge, first,
                                             int64_t(rows), int64_t(cols), scale, {out, out_stride}, e, workspace,
                                             stream));
}

pat_status_t pat_dropout(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, void* out,
                         int64_t out_stride, size_t rows, size_t cols, pat_dtype_t dtype, double p, uint64_t seed,
                         uint64_t index, uint64_t index_stride, hipStream_t stream) {
  Elem e;
  if (!elem_of(dtype, &e)) return PAT_ERR_UNSUPPORTED;
  if (!(p >= 0.0 && p <= 1.0)) return PAT_ERR_INVALID_ARGUMENT;
  if (!dims_ok(rows, cols)) return PAT_ERR_UNSUPPORTED;
  if (rows == 0 || cols == 0) return PAT_OK;
  const size_t es = elem_bytes(e);
  Span in, res, o;
  if (!matrix_span(x, x_stride, rows, cols, es, &in) || !matrix_span(out, out_stride, rows, cols, es, &o) ||
      (residual && !matrix_span(residual, residual_stride, rows, cols, es, &res)))
    return PAT_ERR_INVALID_ARGUMENT;
  // Every element is read before it is written by the same lane, so equal layouts may share memory.
  const bool same_x = out == x && (out_stride == x_stride || rows == 1);
  const bool same_res = out == residual && (out_stride == residual_stride || rows == 1);
  if ((!same_x && overlap(o, in)) || (residual && !same_res && overlap(o, res))) return PAT_ERR_INVALID_ARGUMENT;
  pat::DropoutArgs a;
  a.x = {x, x_stride};
  a.residual = {residual, residual_stride};
  a.out = {out, out_stride};
  a.rows = int64_t(rows);
  a.cols = int64_t(cols);
  a.drop = uint32_t(std::floor(p * 65536.0 + 0.5));
  a.scale = a.drop < 65536 ? float(65536.0 / (65536.0 - double(a.drop))) : 0.0f;
  a.seed = seed;
  a.index = index;
  a.index_stride = index_stride;
  return launched(pat::launch_dropout(a, e, stream));
}

}  // extern "C"
