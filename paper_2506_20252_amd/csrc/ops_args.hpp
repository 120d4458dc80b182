// What the C entry points of pat_ops.h check their arguments with: types, sizes, places of buffers.
#pragma once

#include <cmath>
#include <initializer_list>

#include "../../include/pat_ops.h"
#include "ops.hpp"

namespace {

using pat::Elem;

constexpr size_t kMaxDim = size_t(1) << 31;  // exclusive

inline bool elem_of(pat_dtype_t dtype, Elem* e) {
  if (dtype == PAT_FLOAT32) *e = Elem::f32;
  else if (dtype == PAT_BFLOAT16) *e = Elem::b16;
  else return false;
  return true;
}

inline size_t elem_bytes(Elem e) { return e == Elem::f32 ? 4 : 2; }

// The addresses of a buffer: `width` bytes from lo and from every `pitch` bytes after it, the last end at hi; pitch 0: one
// run of bytes.  Empty ones overlap nothing.
struct Span {
  uintptr_t lo = 0, hi = 0;
  size_t pitch = 0, width = 0;
};

// Runs of bytes of the same pitch may stand between each other's, as column slices of one matrix do; of two different
// pitches whole ranges are compared.
inline bool overlap(const Span& a, const Span& b) {
  if (!(a.lo < a.hi && b.lo < b.hi && a.lo < b.hi && b.lo < a.hi)) return false;
  const size_t pitch = a.pitch ? a.pitch : b.pitch;
  if (!pitch || (b.pitch && b.pitch != pitch)) return true;
  const size_t d = b.lo >= a.lo ? (b.lo - a.lo) % pitch : (pitch - (a.lo - b.lo) % pitch) % pitch;  // b's columns in a's rows
  return d < a.width || b.width > pitch - d;
}

// Span of `bytes` bytes at p; false where p is null, misaligned or wraps around.
inline bool span_of(const void* p, size_t bytes, size_t align, Span* s) {
  if (bytes == 0) {
    *s = Span{};
    return true;
  }
  const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
  if (!lo || lo % align || bytes > UINTPTR_MAX - lo) return false;
  *s = Span{lo, lo + bytes, 0, bytes};
  return true;
}

// Span of a row-major matrix; false also where the stride is below the row's length.
inline bool matrix_span(const void* p, int64_t stride, size_t rows, size_t cols, size_t es, Span* s) {
  if (rows == 0 || cols == 0) {
    *s = Span{};
    return true;
  }
  if (rows > 1 && (stride < 0 || uint64_t(stride) < cols)) return false;
  size_t elems = 0, bytes = 0;
  if (rows > 1 && __builtin_mul_overflow(rows - 1, size_t(stride), &elems)) return false;
  if (__builtin_add_overflow(elems, cols, &elems) || __builtin_mul_overflow(elems, es, &bytes)) return false;
  if (bytes > size_t(INT64_MAX)) return false;
  if (!span_of(p, bytes, es, s)) return false;
  if (rows > 1) s->pitch = size_t(stride) * es, s->width = cols * es;
  return true;
}

// Spans of a stored form's two buffers.
inline bool mx_spans(const void* codes, const void* scales, size_t rows, size_t cols, Span* c, Span* s) {
  return span_of(codes, rows * PAT_MX_CODE_BYTES(cols), 16, c) && span_of(scales, rows * PAT_MX_SCALE_BYTES(cols), 4, s);
}

inline bool any_overlap(const Span& out, std::initializer_list<Span> others) {
  for (const Span& o : others)
    if (overlap(out, o)) return true;
  return false;
}

inline pat_status_t launched(hipError_t e) {
  if (e == hipSuccess) return PAT_OK;
  pat::record_hip_error(e);
  return PAT_ERR_HIP;
}

// Workspace of at least `need` bytes; its span.
inline pat_status_t workspace_span(const void* p, size_t bytes, size_t need, Span* s) {
  if (bytes < need) return PAT_ERR_TOO_LARGE;
  return span_of(p, need, 16, s) ? PAT_OK : PAT_ERR_INVALID_ARGUMENT;
}

// Matrix sizes that every kernel's index arithmetic takes: fewer than 2^31 rows and columns, and for the
// stored form fewer than 2^31 groups of 128 values.
inline bool dims_ok(size_t a, size_t b, size_t c = 0) { return a < kMaxDim && b < kMaxDim && c < kMaxDim; }
inline bool groups_ok(size_t rows, size_t cols) { return rows * ((cols + 127) / 128) < kMaxDim; }

// Embedding gradients: what a launch's grid holds.
inline bool grad_dims_ok(size_t ntokens, size_t rows, size_t cols) {
  return ntokens < size_t(1) << 28 && rows < size_t(1) << 28 && cols < size_t(1) << 23;
}

// Products: what a launch's grid and its kernels' 32-bit offsets inside a tile's rows hold; fewer than 2^38 values of the
// output, in tiles of 16 x 16, which are more than the card's memory.
inline bool product_ok(size_t rows, size_t cols, size_t inner) {
  return rows < size_t(1) << 26 && cols < size_t(1) << 26 && inner < size_t(1) << 24 &&
         ((rows + 15) / 16) * ((cols + 15) / 16) < size_t(1) << 30;
}

}  // namespace
