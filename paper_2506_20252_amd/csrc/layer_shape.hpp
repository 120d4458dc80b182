// How a layer's operators are cut into workgroups: sizes only, no device code.
#pragma once

#include "ops_shape.hpp"

namespace pat {

// ---- root-mean-square norm --------------------------------------------------------------------------------------

// A row takes `lanes` lanes, a power of two up to 64 or whole waves, each `vectors` times 8 columns, which stay in registers
// between the sum and the product; vectors == 0: rows that are too long for that are read again.  Workgroups have `threads`
// lanes for one row or several; `wgs` of them go through the rows.
constexpr int kNormMost = 1024, kNormGradMost = 512;
struct NormPlan {
  int lanes, vectors, threads;
  int64_t wgs;
};

// Lanes for `units` vectors, at most `most` of up to `vectors` each and at least `least`; where there are `many` rows a wave each
// as far as that goes, whose sum needs no LDS.
inline void norm_lanes(bool many, int64_t units, int most, int vectors, int least, NormPlan* p) {
  auto waves = [](int64_t n) { return (int)ceil_div(n, 64) * 64; };
  if (units <= 64) p->lanes = std::max(row_lanes(units, 64), least), p->vectors = 1;
  else if (many && units <= 128) p->lanes = 64, p->vectors = 2;
  else if (units <= 256) p->lanes = waves(units), p->vectors = 1;
  else {
    p->vectors = 2;
    while (p->vectors < vectors && units > (int64_t)most * p->vectors) p->vectors *= 2;
    if (units > (int64_t)most * p->vectors) p->lanes = most, p->vectors = 0;
    else p->lanes = waves(ceil_div(units, p->vectors));
  }
  p->threads = p->lanes * std::max(1, 256 / p->lanes);
}
// The same number of rows for each of at most `most` workgroups, up to one.
inline int64_t norm_wgs(int64_t rows, const NormPlan& p, int64_t most) {
  const int64_t turns = (int64_t)ceil_div(rows, p.threads / p.lanes);
  return (int64_t)ceil_div(turns, ceil_div(turns, most));
}

inline NormPlan norm_plan(int64_t rows, int64_t cols, bool blocks) {
  const int64_t units = blocks ? groups_of(cols) * 16 : (int64_t)ceil_div(cols, 8);  // blocks are filled up to 128 columns
  NormPlan p;
  norm_lanes(rows >= 2048, units, kNormMost, 2, blocks ? 16 : 1, &p);
  p.wgs = norm_wgs(rows, p, 256 * 16 * 64 / p.threads);  // 16 waves a CU
  return p;
}

// The gradients: a workgroup keeps its part of the weight's gradient in registers; the parts, `wgs` rows of `pitch` columns,
// are added up in order afterwards.  vectors == 0: each row's two sums first, then columns in strips of 2048 and rows in
// `wgs` parts.
constexpr int kStripThreads = 256;
struct NormGradPlan : NormPlan {
  int64_t pitch, strips;
};
inline NormGradPlan norm_grad_plan(int64_t rows, int64_t cols) {
  NormGradPlan p;
  const int64_t units = (int64_t)ceil_div(cols, 8);
  norm_lanes(false, units, kNormGradMost, 4, 1, &p);
  p.pitch = units * 8;
  p.strips = (int64_t)ceil_div(units, kStripThreads);
  p.wgs = p.vectors ? norm_wgs(rows, p, std::max(512, 512 * 256 / p.threads)) : std::min(rows, std::max<int64_t>(1, 1024 / p.strips));
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
