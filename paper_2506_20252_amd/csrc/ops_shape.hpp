// How the operators are cut into workgroups: sizes only, no device code.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

#include "ops.hpp"

namespace pat {

// Lanes of a power of two that take a row of `vectors` vectors, at most a workgroup of `threads`.
inline int row_lanes(int64_t vectors, int threads) {
  int lanes = 1;
  while (lanes < vectors && lanes < threads) lanes *= 2;
  return lanes;
}

// ---- dropout ---------------------------------------------------------------------------------------------------

// Rows without gaps in memory and in numbering (`dense`) are taken as one row where a launch holds its workgroups, which
// have 256 lanes: fewer than 2^32 lanes.  A row takes `lanes` lanes, kDropoutBlocks generator blocks a lane in turn, and
// `tiles` workgroups; `wgs` workgroups in all go through the rows.
constexpr int kDropoutBlocks = 2;
constexpr int64_t kDropoutFlat = 8 * (256 * kDropoutBlocks * (((int64_t)1 << 24) - 1) - 1);  // elements of 2^24 - 1 workgroups

struct DropoutPlan {
  bool flat;
  int lanes;
  int64_t tiles, wgs;
};

inline DropoutPlan dropout_plan(int64_t rows, int64_t cols, bool dense) {
  DropoutPlan p;
  p.flat = dense && rows > 1 && rows <= kDropoutFlat / cols;
  const int64_t blocks = ((p.flat ? rows * cols : cols) + 7) / 8 + 1;  // one more where rows begin inside a block
  p.lanes = row_lanes((int64_t)ceil_div(blocks, kDropoutBlocks), 256);
  p.tiles = (int64_t)ceil_div(blocks, (int64_t)p.lanes * kDropoutBlocks);
  const int64_t row_wgs = (int64_t)ceil_div(p.flat ? 1 : rows, 256 / p.lanes);
  p.wgs = std::min(row_wgs, std::max(((int64_t)1 << 22) / p.tiles, (int64_t)1)) * p.tiles;
  return p;
}

// ---- 4-bit product -----------------------------------------------------------------------------------------------

constexpr int kSplitWaves = 8;
constexpr int kSplitRows = 48;

// The product's tiles (256, 128 or 64 rows and columns), or 0: split_kernel.
//
// The largest tile that gives more than half of the 256 CUs one.  A tile's time grows with its area only once the chip is
// full; us with tiles of 64, 128, 256 at n = k = 8192: 24, 30, 51 for m = 256 (512, 128, 32 tiles), 48, 32, 51 for
// m = 512, 85, 52, 54 for m = 1024, 161, 96, 72 for m = 2048.  Up to 48 rows or columns the split is as fast or
// faster (n = 8192: 19 against 20; n = k = 1024: 5 against 6).
inline int64_t product_tiles(int64_t m, int64_t n, int size) { return (int64_t)(ceil_div(m, size) * ceil_div(n, size)); }
inline int product_tile(int64_t m, int64_t n) {
  if (m <= kSplitRows || n <= kSplitRows) return 0;
  return product_tiles(m, n, 256) > 128 ? 256 : product_tiles(m, n, 128) > 128 ? 128 : 64;
}
// Workgroups of such tiles: the same for each XCD.
inline int64_t tile_wgs(int64_t m, int64_t n, int size) { return (int64_t)ceil_div(product_tiles(m, n, size), 8) * 8; }

// Rows and columns of split_kernel's workgroups, in sixteens.
inline int split_rows(int64_t m) { return m <= 16 ? 1 : m <= 32 ? 2 : 4; }
// As many columns a workgroup as leave one for each of the 256 CUs: the rows of a are read and quantised once per
// workgroup.  us at 24 rows with 16, 32, 64 columns: 8.2, 9.2, 11.9 (n = k = 4096), 18, 14.6, 19 (8192), 18, 14.5, 13
// (n = 16384, k = 4096).
inline int split_columns(int64_t n) { return n <= 16 * 256 ? 1 : n <= 32 * 256 ? 2 : 4; }
inline int64_t split_wgs(int64_t m, int64_t n) {
  return (int64_t)(ceil_div(m, 16 * split_rows(m)) * ceil_div(n, 16 * split_columns(n)));
}

// ---- gradients of the 4-bit product ----------------------------------------------------------------------------

// How a product is cut: the tile's size, and slices of j that get workgroups and a float32 matrix of their own, which
// add_kernel adds up.
//
// The largest tile that gives more than half of the 256 CUs one, as for the 4-bit product (us with tiles of 64, 128, 256:
// 134, 80, 95 for 2048 rows, 4096 columns and values of j; 263, 154, 112 for 4096 rows).  Below, few tiles of 128 and
// a long sum are sliced (us, and with tiles of 64: 21 and 36 for 512 rows and columns, 8192 values of j; 19 and 20 for 64
// rows, 4096 columns and values of j), the others take tiles of 64 with two groups of waves (us, and with one group: 10.0 and
// 9.5, 13.7 and 13.6, 33 and 37 for 1001 x 1333 and 500, 1000, 4000 values of j; 19 and 27 for one tile and 4096).
struct GradPlan {
  int tile, slices;
  int64_t slice;
};

inline GradPlan grad_plan(int64_t rows, int64_t inner, int64_t cols) {
  auto tiles = [&](int size) { return (int64_t)(ceil_div(rows, size) * ceil_div(cols, size)); };
  GradPlan p{256, 1, inner};
  if (tiles(256) > 128) return p;
  p.tile = 128;
  if (tiles(128) > 128) return p;
  const int64_t slices = std::min<int64_t>(256 / tiles(128), inner / 512);
  if (slices >= 8) {
    p.slice = (int64_t)ceil_div(ceil_div(inner, slices), 64) * 64;
    p.slices = (int)ceil_div(inner, p.slice);
    // the kernel's vectors of 8 need 8 values of j in the last slice too
    while (inner - (p.slices - 1) * p.slice < 8) p.slice += 64, p.slices = (int)ceil_div(inner, p.slice);
    return p;
  }
  p.tile = 64;
  return p;
}

// narrow_kernel: workgroups of 64 lanes for `rows` rows, 16 x 16 values each, and the rows that go into one launch, fewer
// than 2^26 workgroups.  (Workgroups that take several tiles in turn: 147 us and not 120 for 8192 x 8192 of 4 terms.)
inline int64_t narrow_wgs(int64_t rows, int64_t cols) { return (int64_t)(ceil_div(rows, 16) * ceil_div(cols, 16)); }
inline int64_t narrow_band(int64_t rows, int64_t cols) {
  return std::min(rows, (((int64_t)1 << 26) - 1) / (int64_t)ceil_div(cols, 16) * 16);
}

// ---- embedding gradient ----------------------------------------------------------------------------------------

constexpr int kSortThreads = 256, kMaxBits = 10;  // of a sorting workgroup; of a pass's digit
constexpr int kZeroRows = 64;                     // rows that one workgroup looks through for ones without an entry

// Few tokens take one launch without a sort, in which each workgroup looks at all tokens; unless one workgroup would have
// many for few rows.  us, and sorted: 10 and 15 (256 tokens of 64 columns, 32768 rows), 9.5 and 10.1 (256, 64, 1 row), 28 and
// 40 (1024, 1024, 32768), 7.3 and 16.7 (1024, 1024, 100), 13.1 and 14.7 (1024, 64, 48), but 15.7 and 14.0 (1024, 64, 32), 26
// and 13 (1024, 8, 16).
constexpr int64_t kFewTokens = 1024;
inline bool few_tokens(int64_t ntokens, int64_t rows) {
  return ntokens <= 256 || (ntokens <= kFewTokens && ntokens <= 24 * rows);
}

struct SortPlan {
  int bits, passes;
  int64_t tile, tiles;  // entries per workgroup, workgroups
};

// The sort of not many tokens is one workgroup's.  us, and in workgroups of their own: 20 and 29 (2048 tokens of 64 columns,
// 32768 rows), 26 and 33 (4096, 64, 50000).
constexpr int kSmallBits = 8;
constexpr int64_t kSmallTokens = 4096;

inline SortPlan sort_plan(int64_t ntokens, int64_t rows) {
  int kb = 1;
  while (((int64_t)1 << kb) < rows) ++kb;
  const int most = ntokens <= kSmallTokens ? kSmallBits : kMaxBits;
  SortPlan s;
  s.passes = (kb + most - 1) / most;
  s.bits = std::max((kb + s.passes - 1) / s.passes, 2);  // histograms are read four digits at a time
  s.tile = (int64_t)ceil_div(ceil_div(ntokens, 128), kSortThreads) * kSortThreads;
  if (s.tile < 1024) s.tile = 1024;
  s.tiles = (int64_t)ceil_div(ntokens, s.tile);
  return s;
}

// How the sums are cut: lanes for the columns, entries per piece.  Longer pieces write and join fewer partial sums,
// shorter ones give more workgroups; 2048 of them keep the chip's loads in flight.
struct SumPlan {
  int lanes;
  int32_t piece;
  int64_t pieces, pitch, sum_wgs, zero_wgs, col_wgs;
};

inline SumPlan sum_plan(int64_t ntokens, int64_t rows, int64_t cols) {
  SumPlan s;
  s.lanes = row_lanes((cols + 7) / 8, 256);
  s.col_wgs = (int64_t)ceil_div(cols, 8 * s.lanes);
  s.piece = 64;
  while (s.piece > 16 && (int64_t)ceil_div(ntokens, s.piece) * s.lanes * s.col_wgs < 2048 * 256) s.piece /= 2;
  while ((int64_t)ceil_div(ntokens, s.piece) > 1 << 20) s.piece *= 2;  // bounds the launches and the workspace
  s.pieces = (int64_t)ceil_div(ntokens, s.piece);
  s.pitch = (cols + 7) / 8 * 8;
  s.sum_wgs = (int64_t)ceil_div(s.pieces, 256 / s.lanes);
  s.zero_wgs = (int64_t)ceil_div(rows, kZeroRows);
  return s;
}

}  // namespace pat
