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

// Whole waves that hold n lanes.
inline int whole_waves(int64_t n) { return (int)ceil_div(n, 64) * 64; }
// The same number of rows for each workgroup, of which there are at most as many as stay on the chip together: `waves` of a
// CU's, 256 CUs.  (More go in rounds: 111 us instead of 89 for the gradients of 8192 x 8192 by 384 workgroups of 8 waves
// instead of 256.)
// `join`: what they leave is added up, for which two rows each cost less than a workgroup for every row, once each CU has one (us for
// 300 x 4096, 501 x 1333, 1001 x 1333 rows' gradients: 10.3 and 12.1, 10.7 and 10.9, 13.7 and 14.4; for 64 x 4096: 8.4 and 7.9).
inline int64_t norm_wgs(int64_t rows, const NormPlan& p, int waves, bool join) {
  const int64_t turns = (int64_t)ceil_div(rows, p.threads / p.lanes), most = 256 * std::max(1, waves * 64 / p.threads);
  return (int64_t)ceil_div(turns, std::max<int64_t>(ceil_div(turns, most), join && turns > 256 ? 2 : 1));
}
inline int norm_threads(int lanes) { return lanes * std::max(1, 256 / lanes); }

inline NormPlan norm_plan(int64_t rows, int64_t cols, bool blocks) {
  const int64_t units = blocks ? groups_of(cols) * 16 : (int64_t)ceil_div(cols, 8);  // blocks are filled up to 128 columns
  const int two = whole_waves((int64_t)ceil_div(units, 2));                          // lanes with two vectors each
  NormPlan p;
  if (units <= 64) p.lanes = std::max(row_lanes(units, 64), blocks ? 16 : 1), p.vectors = 1;
  // many rows: a wave each, whose sum needs no LDS
  else if (rows >= 2048 && units <= 128) p.lanes = 64, p.vectors = 2;
  // two vectors where they leave few lanes without (us with two and one: 44 and 44 for 8192 x 4096, 39 and 44 for 8192 x 3584, 54 and
  // 42 for 10513 x 2129)
  else if (units <= 256 || (units <= 512 && 2 * two * 4 > units * 5)) p.lanes = whole_waves(units), p.vectors = 1;
  else if (two <= kNormMost) p.lanes = two, p.vectors = 2;
  else p.lanes = kNormMost, p.vectors = 0;
  p.threads = norm_threads(p.lanes);
  p.wgs = norm_wgs(rows, p, 16, false);  // of 128 registers
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
  p.vectors = units <= kNormGradMost ? 1 : units <= 2 * kNormGradMost ? 2 : units <= 4 * kNormGradMost ? 4 : 0;
  p.lanes = units <= 64 ? row_lanes(units, 64) : p.vectors ? whole_waves((int64_t)ceil_div(units, p.vectors)) : kNormGradMost;
  p.threads = norm_threads(p.lanes);
  p.pitch = units * 8;
  p.strips = (int64_t)ceil_div(units, kStripThreads);
  // two workgroups of more than four waves (us for 10513 x 2129: 59 with two a CU, 74 with three)
  const int waves = p.vectors == 4 ? 8 : p.vectors == 2 ? 12 : p.threads > 256 ? p.threads / 32 : 16;
  p.wgs = p.vectors ? norm_wgs(rows, p, waves, true) : std::min(rows, std::max<int64_t>(1, 1024 / p.strips));
  return p;
}

// Their workspace: the parts, where there are several or rows are long, as floats from its start, then two floats a row where
// rows are long.
struct NormGradSpace {
  int64_t parts, rows_at;  // floats; the rows' first
  size_t bytes;
};
inline NormGradSpace norm_grad_space(const NormGradPlan& p, int64_t rows) {
  NormGradSpace s;
  s.parts = p.wgs > 1 || p.vectors == 0 ? p.wgs * p.pitch : 0;
  s.rows_at = s.parts;
  s.bytes = (size_t)(s.parts + (p.vectors ? 0 : 2 * rows)) * 4;
  return s;
}

// ---- products of 8-bit with 4-bit blocks ------------------------------------------------------------------------

// Tiles of m tokens by n rows of the weight: 256 (256 x 256), 128 (128 x 128), 64 (64 tokens by 128 rows), or 32 (64 x 64, in two
// parts of the terms).
//
// The largest of the first two that gives more than half of the 256 CUs one; else 64 x 64 as long as each CU has at most one.
// us with 64 x 64, 64 x 128, 128 x 128: 8.9, 10.8, 15.1 (64 tokens, 4096 rows and terms: 64, 32, 32 tiles), 13.1, 16.4, 21.9 (256
// tokens: 256, 128, 64), 20.1, 19.2, 22.7 (512: 512, 256, 128), 34, 31, 24 (1024: 1024, 512, 256), 9.4, 6.6, 8.6 (1001 tokens, 2000 rows,
// 1333 terms: 512, 256, 128).
inline int64_t layer_tiles(int64_t m, int64_t n, int rows_x, int rows_w) { return (int64_t)(ceil_div(m, rows_x) * ceil_div(n, rows_w)); }
inline int layer_tile(int64_t m, int64_t n) {
  if (layer_tiles(m, n, 256, 256) > 128) return 256;
  if (layer_tiles(m, n, 128, 128) > 128) return 128;
  return layer_tiles(m, n, 64, 64) > 256 ? 64 : 32;
}

// few_kernel: up to so many tokens.  us, and by tiles: 7.8 and 8.5 (32 tokens, 4096 columns and terms), 10.3 and 11.4 (33, 8192,
// 4096), 18.1 and 19.6 (48, 4096, 8192).  Gated, 33 tokens: 14.9 and 14.7 (8192, 4096), 48: 25.3 and 22.3 (4096, 8192).
//
// Gated products of 17 to 32 tokens go by tiles already where columns are few and terms are many (each of few_kernel's
// workgroups reads all tokens, as many bytes as its 32 rows of the weight or more).  With 17 and with 32 tokens: 4.1 and 4.9,
// 4.3 and 4.9 (2048 columns, 512 terms), 4.9 and 5.8, 5.4 and 5.9 (2048, 1333), 6.6 and 6.3, 7.4 and 6.4 (2048, 2000), 9.9 and
// 8.1, 11.4 and 8.3 (1024, 4096), 16.8 and 11.8, 19.9 and 12.3 (512, 8192), 17.4 and 17.5, 20.3 and 18.6 (2048, 8192); at 4096
// columns either way, 10.4 and 10.3, 11.9 and 11.4 (4096), 17.4 and 18.7, 20.3 and 20.2 (8192); 10.6 and 11.9, 12.1 and 13.6
// (8192, 4096).
constexpr int kFewLinear = 48, kFewGated = 32;
inline bool few_product(int64_t m, int64_t n, int64_t k, bool gated) {
  if (k == 0) return true;
  if (!gated) return m <= kFewLinear;
  return m <= 16 || (m <= kFewGated && (n > 2048 || k <= 1536));
}
// Its columns of the output, in sixteens (two where gated, each two rows of the weight): as many as leave a workgroup for each of
// the 256 CUs, since every workgroup reads the tokens.  And the tokens that go into one launch of fewer than 2^22 workgroups.
inline int few_columns_sixteens(int64_t n) { return n <= 16 * 256 ? 1 : n <= 32 * 256 ? 2 : 4; }
inline int64_t few_band(int64_t m, int64_t tiles_n, int64_t tokens) {
  return std::min(m, std::max<int64_t>(1, (((int64_t)1 << 22) - 1) / tiles_n) * tokens);
}

// A tile's tokens, its rows of the weight, its workgroup's lanes.
constexpr int tile_tokens(int tile) { return tile < 128 ? 64 : tile; }
constexpr int tile_rows(int tile) { return tile == 32 ? 64 : tile == 64 ? 128 : tile; }
constexpr int tile_threads(int tile) { return tile == 256 ? 512 : 256; }
constexpr int kFewWaves = 8;

// How x w^T is launched, for n columns of the output (`gated`: 2 n rows of the weight).  tile == 0: few_kernel, 16 * `tokens` by
// 16 * `columns` values of the output a workgroup.  `blocks`: something leaves in 8-bit blocks, which are filled up to 128
// columns.  `tiles_n` workgroups beside each other, `band` tokens a launch, `wgs` workgroups in the largest one.
struct ProductPlan {
  int tile, tokens, columns, threads;
  int64_t tiles_n, band, wgs;
};
inline ProductPlan product_plan(int64_t m, int64_t n, int64_t k, bool gated, bool blocks) {
  ProductPlan p{};
  const int64_t width = blocks ? groups_of(n) * 128 : n;
  if (!few_product(m, n, k, gated)) {
    p.tile = layer_tile(m, gated ? 2 * n : n);
    p.threads = tile_threads(p.tile);
    p.tiles_n = (int64_t)ceil_div(width, gated ? tile_rows(p.tile) / 2 : tile_rows(p.tile));
    p.band = m;
    p.wgs = (int64_t)ceil_div(ceil_div(m, tile_tokens(p.tile)) * p.tiles_n, 8) * 8;  // the same for each XCD
    return p;
  }
  p.tokens = m <= 16 ? 1 : m <= 32 || gated ? 2 : 3;
  p.columns = gated ? 2 : few_columns_sixteens(n);
  p.threads = 64 * kFewWaves;
  p.tiles_n = (int64_t)ceil_div(width, 16 * p.columns);
  p.band = few_band(m, p.tiles_n, 16 * p.tokens);
  p.wgs = (int64_t)ceil_div(p.band, 16 * p.tokens) * p.tiles_n;
  return p;
}

}  // namespace pat
