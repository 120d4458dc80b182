// How a layer's operators are cut into workgroups: sizes only, no device code.
#pragma once

#include "ops_shape.hpp"

namespace pat {

// ---- root-mean-square norm --------------------------------------------------------------------------------------

// A row takes `lanes` lanes, each `vectors` times 8 columns, which stay in registers between the sum and the product;
// vectors == 0: rows that are too long for that are read again.  Workgroups have 256 lanes, or one row's; `wgs` of them go
// through the rows.
constexpr int kNormThreads = 256, kNormMost = 1024, kNormGradMost = 512;
struct NormPlan {
  int lanes, vectors;
  int64_t wgs;
};

inline NormPlan norm_plan(int64_t rows, int64_t cols, bool blocks) {
  const int64_t units = blocks ? groups_of(cols) * 16 : (int64_t)ceil_div(cols, 8);  // blocks are filled up to 128 columns
  NormPlan p;
  p.lanes = row_lanes(units, kNormThreads);
  while (p.lanes < kNormMost && units > 2 * p.lanes) p.lanes *= 2;
  // many rows: a wave each, whose sum needs no LDS
  if (rows >= 2048 && p.lanes > 64 && units <= 64 * 2) p.lanes = 64;
  if (blocks && p.lanes < 16) p.lanes = 16;
  p.vectors = units <= p.lanes ? 1 : units <= 2 * p.lanes ? 2 : 0;
  p.wgs = std::min((int64_t)ceil_div(rows, std::max(kNormThreads, p.lanes) / p.lanes), (int64_t)1 << 20);
  return p;
}

// The gradients: a workgroup goes through rows `wgs` apart and keeps its part of the weight's gradient in registers; the
// parts, `wgs` rows of `pitch` columns, are added up in order afterwards.  vectors == 0: each row's two sums first, then
// columns in strips of 2048 and rows in `wgs` parts.
struct NormGradPlan {
  int lanes, vectors;
  int64_t wgs, pitch, strips;
};
inline NormGradPlan norm_grad_plan(int64_t rows, int64_t cols) {
  NormGradPlan p;
  const int64_t units = (int64_t)ceil_div(cols, 8);
  p.lanes = row_lanes(units, kNormThreads);
  while (p.lanes < kNormGradMost && units > 2 * p.lanes) p.lanes *= 2;
  p.vectors = units <= p.lanes ? 1 : units <= 2 * p.lanes ? 2 : units <= 4 * p.lanes ? 4 : 0;
  p.pitch = units * 8;
  p.strips = (int64_t)ceil_div(units, kNormThreads);
  const int64_t most = p.vectors ? 512 : std::max<int64_t>(1, 1024 / p.strips);
  p.wgs = std::min((int64_t)ceil_div(rows, p.vectors ? std::max(kNormThreads, p.lanes) / p.lanes : 1), most);
  return p;
}

// ---- products of 8-bit with 4-bit blocks ------------------------------------------------------------------------

// Tiles of m tokens by n rows of the weight: 256 (256 x 256), 128 (128 x 128) or 64 (64 tokens x 128 rows).  The largest that
// gives more than half of the 256 CUs one.
inline int layer_tile(int64_t m, int64_t n) {
  auto tiles = [&](int rows_x, int rows_w) { return (int64_t)(ceil_div(m, rows_x) * ceil_div(n, rows_w)); };
  return tiles(256, 256) > 128 ? 256 : tiles(128, 128) > 128 ? 128 : 64;
}

// few_kernel: tokens and columns of the output of a workgroup, in sixteens (a gated column is two rows of the weight), and
// the tokens that go into one launch of fewer than 2^22 workgroups.
constexpr int kFewMost = 48;
inline int few_tokens_sixteens(int64_t m) { return m <= 16 ? 1 : m <= 32 ? 2 : 3; }
inline int few_columns_sixteens(int64_t n) { return n <= 16 * 256 ? 1 : n <= 32 * 256 ? 2 : 4; }
inline int64_t few_band(int64_t m, int64_t tiles_n, int64_t tokens) {
  return std::min(m, std::max<int64_t>(1, (((int64_t)1 << 22) - 1) / tiles_n) * tokens);
}

}  // namespace pat
