// C entry points of pat_ops.h for a layer's operators (8-bit blocks, products of them, the gated block, the norm): argument
// checks, then one launch function each.  Nothing here allocates or throws.
#include "ops_args.hpp"

namespace {

using pat::MxbMat;
using pat::MxbOut;
using pat::MxMat;

MxMat mx(const void* codes, const void* scales) {
  return {static_cast<const uint8_t*>(codes), static_cast<const uint8_t*>(scales)};
}
MxbMat mxb(const void* codes, const void* scales) {
  return {static_cast<const uint8_t*>(codes), static_cast<const uint8_t*>(scales)};
}
MxbOut mxb_out(void* codes, void* scales) { return {static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scales)}; }

bool mxb_spans(const void* codes, const void* scales, size_t rows, size_t cols, Span* c, Span* s) {
  return span_of(codes, rows * PAT_MXB_CODE_BYTES(cols), 16, c) && span_of(scales, rows * PAT_MXB_SCALE_BYTES(cols), 4, s);
}

bool act_of(pat_activation_t act, pat::Act* a) {
  if (act == PAT_SILU) *a = pat::Act::silu;
  else if (act == PAT_GELU) *a = pat::Act::gelu;
  else return false;
  return true;
}

// Where the result leaves: a matrix of `dtype`, or 8-bit blocks where `out` is null.
struct Result {
  Elem dtype = Elem::f32;
  Span matrix, codes, scales;
};
pat_status_t result_of(void* out, int64_t out_stride, pat_dtype_t dtype, void* codes, void* scales, size_t rows, size_t cols,
                       Result* r) {
  if (out && (codes || scales)) return PAT_ERR_INVALID_ARGUMENT;
  if (out) {
    if (!elem_of(dtype, &r->dtype)) return PAT_ERR_UNSUPPORTED;
    return matrix_span(out, out_stride, rows, cols, elem_bytes(r->dtype), &r->matrix) ? PAT_OK : PAT_ERR_INVALID_ARGUMENT;
  }
  if (!groups_ok(rows, cols)) return PAT_ERR_UNSUPPORTED;
  if (!mxb_spans(codes, scales, rows, cols, &r->codes, &r->scales) || overlap(r->codes, r->scales)) return PAT_ERR_INVALID_ARGUMENT;
  return PAT_OK;
}

// The same place for two matrices of the same rows: every element is read before the same lane writes it.
bool same_place(const void* a, int64_t a_stride, const void* b, int64_t b_stride, size_t rows) {
  return a == b && (rows == 1 || a_stride == b_stride);
}

}  // namespace

extern "C" {

pat_status_t pat_mxb_quantize(const void* x, int64_t x_stride, size_t rows, size_t cols, pat_dtype_t dtype, void* codes,
                              void* scales, hipStream_t stream) {
  Elem e;
  if (!elem_of(dtype, &e)) return PAT_ERR_UNSUPPORTED;
  if (!dims_ok(rows, cols) || !groups_ok(rows, cols)) return PAT_ERR_UNSUPPORTED;
  if (rows == 0 || cols == 0) return PAT_OK;
  Span in, c, s;
  if (!matrix_span(x, x_stride, rows, cols, elem_bytes(e), &in) || !mxb_spans(codes, scales, rows, cols, &c, &s))
    return PAT_ERR_INVALID_ARGUMENT;
  if (any_overlap(c, {in, s}) || overlap(s, in)) return PAT_ERR_INVALID_ARGUMENT;
  return launched(pat::launch_mxb_quantize({x, x_stride}, e, int64_t(rows), int64_t(cols), mxb_out(codes, scales), stream));
}

pat_status_t pat_mxb_dequantize(const void* codes, const void* scales, size_t rows, size_t cols, void* out,
                                int64_t out_stride, pat_dtype_t dtype, hipStream_t stream) {
  Elem e;
  if (!elem_of(dtype, &e)) return PAT_ERR_UNSUPPORTED;
  if (!dims_ok(rows, cols) || !groups_ok(rows, cols)) return PAT_ERR_UNSUPPORTED;
  if (rows == 0 || cols == 0) return PAT_OK;
  Span o, c, s;
  if (!matrix_span(out, out_stride, rows, cols, elem_bytes(e), &o) || !mxb_spans(codes, scales, rows, cols, &c, &s))
    return PAT_ERR_INVALID_ARGUMENT;
  if (any_overlap(o, {c, s})) return PAT_ERR_INVALID_ARGUMENT;
  return launched(pat::launch_mxb_dequantize(mxb(codes, scales), int64_t(rows), int64_t(cols), {out, out_stride}, e, stream));
}

pat_status_t pat_mxb_linear(const void* x_codes, const void* x_scales, const void* w_codes, const void* w_scales, size_t m,
                            size_t n, size_t k, const void* residual, int64_t residual_stride, void* out,
                            int64_t out_stride, pat_dtype_t dtype, hipStream_t stream) {
  Elem e;
  if (!elem_of(dtype, &e)) return PAT_ERR_UNSUPPORTED;
  if (!product_ok(m, n, k) || !groups_ok(m, k) || !groups_ok(n, k)) return PAT_ERR_UNSUPPORTED;
  if (m == 0 || n == 0) return PAT_OK;
  Span xc, xs, wc, ws, res, o;
  if (!mxb_spans(x_codes, x_scales, m, k, &xc, &xs) || !mx_spans(w_codes, w_scales, n, k, &wc, &ws) ||
      !matrix_span(out, out_stride, m, n, elem_bytes(e), &o) ||
      (residual && !matrix_span(residual, residual_stride, m, n, elem_bytes(e), &res)))
    return PAT_ERR_INVALID_ARGUMENT;
  if (any_overlap(o, {xc, xs, wc, ws})) return PAT_ERR_INVALID_ARGUMENT;
  if (!same_place(out, out_stride, residual, residual_stride, m) && overlap(o, res)) return PAT_ERR_INVALID_ARGUMENT;
  pat::Epilogue ep{};
  ep.residual = {residual, residual_stride};
  ep.out = {out, out_stride};
  ep.dtype = e;
  return launched(pat::launch_mxb_product(mxb(x_codes, x_scales), mx(w_codes, w_scales), int64_t(m), int64_t(n), int64_t(k), ep,
                                          stream));
}

size_t pat_mxb_weight_grad_workspace(size_t rows, size_t inner, size_t cols) {
  if (!product_ok(rows, cols, inner) || !rows || !cols) return 0;
  return pat::mx_grad_workspace(int64_t(rows), int64_t(inner), int64_t(cols));
}

pat_status_t pat_mxb_weight_grad(const void* g, int64_t g_stride, const void* x_codes, const void* x_scales, size_t rows,
                                 size_t inner, size_t cols, void* out, int64_t out_stride, pat_dtype_t dtype,
                                 void* workspace, size_t workspace_bytes, hipStream_t stream) {
  Elem e;
  if (!elem_of(dtype, &e)) return PAT_ERR_UNSUPPORTED;
  if (!product_ok(rows, cols, inner) || !groups_ok(inner, cols)) return PAT_ERR_UNSUPPORTED;
  if (rows == 0 || cols == 0) return PAT_OK;
  Span in, xc, xs, o, w;
  if (!matrix_span(g, g_stride, inner, rows, 2, &in) || !mxb_spans(x_codes, x_scales, inner, cols, &xc, &xs) ||
      !matrix_span(out, out_stride, rows, cols, elem_bytes(e), &o))
    return PAT_ERR_INVALID_ARGUMENT;
  if (pat_status_t st = workspace_span(workspace, workspace_bytes, pat_mxb_weight_grad_workspace(rows, inner, cols), &w))
    return st;
  if (any_overlap(o, {in, xc, xs, w}) || any_overlap(w, {in, xc, xs})) return PAT_ERR_INVALID_ARGUMENT;
  return launched(pat::launch_mxb_weight_grad({g, g_stride}, mxb(x_codes, x_scales), int64_t(rows), int64_t(inner), int64_t(cols),
                                              {out, out_stride}, e, workspace, stream));
}

pat_status_t pat_gated(const void* x_codes, const void* x_scales, const void* w_codes, const void* w_scales, size_t m,
                       size_t n, size_t k, pat_activation_t act, void* out, int64_t out_stride, pat_dtype_t dtype,
                       void* out_codes, void* out_scales, void* saved_codes, void* saved_scales, hipStream_t stream) {
  pat::Epilogue ep{};
  Elem e;
  if (out && !elem_of(dtype, &e)) return PAT_ERR_UNSUPPORTED;
  if (!act_of(act, &ep.act)) return PAT_ERR_UNSUPPORTED;
  if (n >= kMaxDim || !product_ok(m, 2 * n, k) || !groups_ok(m, k) || !groups_ok(2 * n, k)) return PAT_ERR_UNSUPPORTED;
  const bool saves = saved_codes || saved_scales;
  if (saves && !groups_ok(2 * m, n)) return PAT_ERR_UNSUPPORTED;
  if (m == 0 || n == 0) return PAT_OK;
  Span xc, xs, wc, ws, sc, ss;
  Result r;
  if (!mxb_spans(x_codes, x_scales, m, k, &xc, &xs) || !mx_spans(w_codes, w_scales, 2 * n, k, &wc, &ws) ||
      (saves && !mxb_spans(saved_codes, saved_scales, 2 * m, n, &sc, &ss)))
    return PAT_ERR_INVALID_ARGUMENT;
  if (pat_status_t st = result_of(out, out_stride, dtype, out_codes, out_scales, m, n, &r)) return st;
  for (const Span& o : {r.matrix, r.codes, r.scales})
    if (any_overlap(o, {xc, xs, wc, ws, sc, ss})) return PAT_ERR_INVALID_ARGUMENT;
  if (any_overlap(sc, {xc, xs, wc, ws, ss}) || any_overlap(ss, {xc, xs, wc, ws})) return PAT_ERR_INVALID_ARGUMENT;
  ep.gated = true;
  ep.out = {out, out_stride};
  ep.dtype = r.dtype;
  if (!out) ep.blocks = mxb_out(out_codes, out_scales);
  if (saves) {
    ep.saved_a = mxb_out(saved_codes, saved_scales);
    ep.saved_b = {ep.saved_a.codes + m * PAT_MXB_CODE_BYTES(n), ep.saved_a.scales + m * PAT_MXB_SCALE_BYTES(n)};
  }
  return launched(pat::launch_mxb_product(mxb(x_codes, x_scales), mx(w_codes, w_scales), int64_t(m), int64_t(n), int64_t(k), ep,
                                          stream));
}

pat_status_t pat_gated_grad(const void* g, int64_t g_stride, pat_dtype_t g_dtype, const void* saved_codes,
                            const void* saved_scales, size_t m, size_t n, pat_activation_t act, void* out,
                            int64_t out_stride, hipStream_t stream) {
  Elem e;
  pat::Act a;
  if (!elem_of(g_dtype, &e) || !act_of(act, &a)) return PAT_ERR_UNSUPPORTED;
  if (!dims_ok(m, n) || !dims_ok(2 * m, 2 * n) || !groups_ok(2 * m, n)) return PAT_ERR_UNSUPPORTED;
  if (m == 0 || n == 0) return PAT_OK;
  Span in, sc, ss, o;
  if (!matrix_span(g, g_stride, m, n, elem_bytes(e), &in) || !mxb_spans(saved_codes, saved_scales, 2 * m, n, &sc, &ss) ||
      !matrix_span(out, out_stride, m, 2 * n, 2, &o))
    return PAT_ERR_INVALID_ARGUMENT;
  if (any_overlap(o, {in, sc, ss})) return PAT_ERR_INVALID_ARGUMENT;
  const MxbMat sa = mxb(saved_codes, saved_scales);
  return launched(pat::launch_gated_grad({g, g_stride}, e, sa,
                                         {sa.codes + m * PAT_MXB_CODE_BYTES(n), sa.scales + m * PAT_MXB_SCALE_BYTES(n)}, int64_t(m),
                                         int64_t(n), a, {out, out_stride}, stream));
}

pat_status_t pat_rms_norm(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, pat_dtype_t dtype,
                          const void* weight, pat_dtype_t weight_dtype, size_t rows, size_t cols, float eps, void* total,
                          int64_t total_stride, void* out, int64_t out_stride, pat_dtype_t out_dtype, void* out_codes,
                          void* out_scales, hipStream_t stream) {
  pat::NormArgs a{};
  Elem e;
  if (!elem_of(dtype, &a.dtype) || !elem_of(weight_dtype, &a.weight_dtype) || (out && !elem_of(out_dtype, &e)))
    return PAT_ERR_UNSUPPORTED;
  if (!(eps >= 0.0f && std::isfinite(eps)) || (total && !residual)) return PAT_ERR_INVALID_ARGUMENT;
  if (!dims_ok(rows, cols)) return PAT_ERR_UNSUPPORTED;
  if (rows == 0 || cols == 0) return PAT_OK;
  const size_t es = elem_bytes(a.dtype), wes = elem_bytes(a.weight_dtype);
  Span in, res, w, tot;
  Result r;
  if (!matrix_span(x, x_stride, rows, cols, es, &in) || !span_of(weight, cols * wes, wes, &w) ||
      (residual && !matrix_span(residual, residual_stride, rows, cols, es, &res)) ||
      (total && !matrix_span(total, total_stride, rows, cols, es, &tot)))
    return PAT_ERR_INVALID_ARGUMENT;
  if (pat_status_t st = result_of(out, out_stride, out_dtype, out_codes, out_scales, rows, cols, &r)) return st;
  // A row's elements are read, for the sum and again for long rows, before the same lane writes them.  What long rows read
  // again is the total where there is one.
  auto clear = [&](const void* p, int64_t stride, const Span& s, bool may) {
    return (may && same_place(p, stride, x, x_stride, rows) ? true : !overlap(s, in)) &&
           (may && same_place(p, stride, residual, residual_stride, rows) ? true : !overlap(s, res)) && !overlap(s, w);
  };
  if (total && !clear(total, total_stride, tot, true)) return PAT_ERR_INVALID_ARGUMENT;
  if (out && (!clear(out, out_stride, r.matrix, r.dtype == a.dtype) || overlap(r.matrix, tot))) return PAT_ERR_INVALID_ARGUMENT;
  if (any_overlap(r.codes, {in, res, w, tot}) || any_overlap(r.scales, {in, res, w, tot})) return PAT_ERR_INVALID_ARGUMENT;
  a.x = {x, x_stride};
  a.residual = {residual, residual_stride};
  a.weight = weight;
  a.rows = int64_t(rows);
  a.cols = int64_t(cols);
  a.eps = eps;
  a.total = {total, total_stride};
  a.out = {out, out_stride};
  a.out_dtype = r.dtype;
  if (!out) a.blocks = mxb_out(out_codes, out_scales);
  return launched(pat::launch_rms_norm(a, stream));
}

// The launches' sizes, and partial sums of fewer than 2^40 bytes.
static bool norm_grad_ok(size_t rows, size_t cols) { return rows < size_t(1) << 28 && cols < size_t(1) << 26; }

size_t pat_rms_norm_grad_workspace(size_t rows, size_t cols) {
  if (!norm_grad_ok(rows, cols) || !rows || !cols) return 0;
  return pat::rms_norm_grad_workspace(int64_t(rows), int64_t(cols));
}

pat_status_t pat_rms_norm_grad(const void* g, int64_t g_stride, pat_dtype_t dtype, const void* x, int64_t x_stride,
                               pat_dtype_t x_dtype, const void* weight, pat_dtype_t weight_dtype, const void* total_grad,
                               int64_t total_grad_stride, size_t rows, size_t cols, float eps, void* out, int64_t out_stride,
                               void* dweight, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  pat::NormGradArgs a{};
  if (!elem_of(dtype, &a.dtype) || !elem_of(x_dtype, &a.x_dtype) || !elem_of(weight_dtype, &a.weight_dtype))
    return PAT_ERR_UNSUPPORTED;
  if (!(eps >= 0.0f && std::isfinite(eps))) return PAT_ERR_INVALID_ARGUMENT;
  if (!norm_grad_ok(rows, cols)) return PAT_ERR_UNSUPPORTED;
  if (cols == 0) return PAT_OK;
  const size_t es = elem_bytes(a.dtype), xes = elem_bytes(a.x_dtype), wes = elem_bytes(a.weight_dtype);
  Span in, xs, w, tg, o, dw, work;
  if (!matrix_span(g, g_stride, rows, cols, es, &in) || !matrix_span(x, x_stride, rows, cols, xes, &xs) ||
      !span_of(weight, cols * wes, wes, &w) || !matrix_span(out, out_stride, rows, cols, es, &o) ||
      (total_grad && !matrix_span(total_grad, total_grad_stride, rows, cols, es, &tg)) || !span_of(dweight, cols * 4, 4, &dw))
    return PAT_ERR_INVALID_ARGUMENT;
  if (pat_status_t st = workspace_span(workspace, workspace_bytes, pat_rms_norm_grad_workspace(rows, cols), &work)) return st;
  if (!same_place(out, out_stride, g, g_stride, rows) && overlap(o, in)) return PAT_ERR_INVALID_ARGUMENT;
  if (!same_place(out, out_stride, total_grad, total_grad_stride, rows) && overlap(o, tg)) return PAT_ERR_INVALID_ARGUMENT;
  if (any_overlap(o, {xs, w, dw, work}) || any_overlap(dw, {in, xs, w, tg, work}) || any_overlap(work, {in, xs, w, tg}))
    return PAT_ERR_INVALID_ARGUMENT;
  a.g = {g, g_stride};
  a.x = {x, x_stride};
  a.total_grad = {total_grad, total_grad_stride};
  a.weight = weight;
  a.rows = int64_t(rows);
  a.cols = int64_t(cols);
  a.eps = eps;
  a.out = {out, out_stride};
  a.dweight = static_cast<float*>(dweight);
  return launched(pat::launch_rms_norm_grad(a, workspace, stream));
}

}  // extern "C"
