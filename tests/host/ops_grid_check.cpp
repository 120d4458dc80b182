// What the operators' launches ask for (ops_shape.hpp): a launch holds fewer than 2^32 lanes, and has to reach all its work;
// and which places of an output beside an input the entry points (ops.cpp) take.
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "../../include/pat_ops.h"
#include "ops_shape.hpp"

using namespace pat;

static int g_failures = 0, g_checked = 0;
#define CHECK(cond, ...)                                     \
  do {                                                       \
    ++g_checked;                                             \
    if (!(cond)) {                                           \
      if (++g_failures < 20) std::printf("%s: ", #cond), std::printf(__VA_ARGS__), std::printf("\n"); \
    }                                                        \
  } while (0)

static const int64_t kLanes = (int64_t)1 << 32;

// Sizes that are accepted: 1 ... 2^31 - 1 rows and columns.
static void check_dropout(int64_t rows, int64_t cols) {
  const long long r = rows, c = cols;
  for (int dense = 0; dense < 2; ++dense) {
    const DropoutPlan p = dropout_plan(rows, cols, dense);
    CHECK(p.lanes >= 1 && p.lanes <= 256 && (p.lanes & (p.lanes - 1)) == 0, "%lld %lld", r, c);
    CHECK(p.wgs >= 1 && p.wgs * 256 < kLanes, "%lld %lld: %lld workgroups", r, c, (long long)p.wgs);
    CHECK(p.tiles >= 1 && p.wgs % p.tiles == 0, "%lld %lld: %lld of %lld", r, c, (long long)p.wgs, (long long)p.tiles);
    // a row's blocks of 8, one more where it begins inside one
    const int64_t blocks = ((p.flat ? rows * cols : cols) + 7) / 8 + 1;
    CHECK(p.tiles * p.lanes * kDropoutBlocks >= blocks, "%lld %lld", r, c);
    CHECK(dense || !p.flat, "%lld %lld", r, c);
  }
  // as one row as long as that fits: every tensor of up to 2^35 elements
  if (rows > 1 && rows * cols <= (int64_t)1 << 35) CHECK(dropout_plan(rows, cols, true).flat, "%lld %lld", r, c);
}

// What the C entry points of the products and their gradient hand to a launch: of accepted sizes it holds the lanes.
namespace pat {
static int64_t g_lanes = -1;
static int64_t narrow_lanes(int64_t rows, int64_t cols) {  // of the first, largest launch; 0: it would cut a tile
  const int64_t band = narrow_band(rows, cols);
  return band > 0 && (band == rows || band % 16 == 0) ? narrow_wgs(band, cols) * 64 : 0;
}
void record_hip_error(hipError_t) {}
hipError_t launch_mx_quantize(Mat, Elem, int64_t, int64_t, uint8_t*, uint8_t*, hipStream_t) { return hipSuccess; }
hipError_t launch_mx_dequantize(MxMat, int64_t, int64_t, MatOut, Elem, hipStream_t) { return hipSuccess; }
hipError_t launch_mx_matmul(MxMat, MxMat, int64_t m, int64_t n, int64_t k, MatOut, Elem, hipStream_t) {
  const int tile = product_tile(m, n);
  g_lanes = k == 0 ? narrow_lanes(m, n) : tile ? tile_wgs(m, n, tile) * (tile == 256 ? 512 : 256) : split_wgs(m, n) * 64 * kSplitWaves;
  return hipSuccess;
}
size_t mx_linear_workspace(int64_t, int64_t, int64_t) { return 0; }
hipError_t launch_mx_linear(Mat, Elem, MxMat, int64_t, int64_t, int64_t, MatOut, Elem, void*, hipStream_t) {
  return hipSuccess;
}
size_t mx_grad_workspace(int64_t, int64_t, int64_t) { return 0; }
hipError_t launch_mx_grad(Mat, bool, MxMat, int64_t rows, int64_t inner, int64_t cols, MatOut, Elem, void*, hipStream_t) {
  const GradPlan p = grad_plan(rows, inner, cols);
  g_lanes = narrow_lanes(rows, cols) ? std::max(narrow_lanes(rows, cols), tile_wgs(rows, cols, p.tile) * 512) : 0;
  return hipSuccess;
}
hipError_t launch_embedding(const void*, int, int64_t, Mat, Elem, int64_t, int64_t, int64_t, float, MatOut, Elem,
                            hipStream_t) {
  return hipSuccess;
}
size_t embedding_grad_workspace(int64_t, int64_t, int64_t) { return 0; }
hipError_t launch_embedding_grad(const void*, int, int64_t, Mat, Elem, int64_t, int64_t, int64_t, float, MatOut, Elem, void*,
                                 hipStream_t) {
  return hipSuccess;
}
hipError_t launch_dropout(const DropoutArgs&, Elem, hipStream_t) { return hipSuccess; }
}  // namespace pat

static void check_product(int64_t rows, int64_t cols) {
  auto at = [](uint64_t off) { return (void*)(uintptr_t)off; };  // never read: launches only record
  if (rows < 1 || cols < 1) return;
  for (int64_t terms : {0, 1, 200}) {
    g_lanes = 0;
    const pat_status_t st = pat_mx_matmul(at(1ull << 60), at(1ull << 59), at(1ull << 58), at(1ull << 57), rows, cols, terms, at(4096),
                                          cols, PAT_FLOAT32, nullptr);
    CHECK(st == PAT_OK ? g_lanes > 0 : st == PAT_ERR_UNSUPPORTED && rows * cols >= (int64_t)1 << 26, "%lld %lld: %d", (long long)rows,
          (long long)cols, st);
    CHECK(g_lanes < kLanes, "%lld %lld %lld: %lld lanes", (long long)rows, (long long)cols, (long long)terms, (long long)g_lanes);
    g_lanes = 0;
    const pat_status_t gr = pat_mx_matmul_grad(at(1ull << 60), rows, 1, at(1ull << 58), at(1ull << 57), rows, terms, cols, at(4096),
                                               cols, PAT_FLOAT32, nullptr, 0, nullptr);
    CHECK(gr == PAT_OK ? g_lanes > 0 : gr == PAT_ERR_UNSUPPORTED && rows * cols >= (int64_t)1 << 26, "%lld %lld: %d", (long long)rows,
          (long long)cols, gr);
    CHECK(g_lanes < kLanes, "%lld %lld %lld: %lld lanes", (long long)rows, (long long)cols, (long long)terms, (long long)g_lanes);
    // 2^37 values, 256 GiB in bfloat16, are taken
    if (rows < 1 << 26 && cols < 1 << 26 && rows * cols <= (int64_t)1 << 37 && rows >= 256 && cols >= 256)
      CHECK(st == PAT_OK && gr == PAT_OK, "%lld %lld: %d %d", (long long)rows, (long long)cols, st, gr);
  }
}

// An output in the columns that an input leaves free of the same rows shares no byte with it.  Matrices of the same pitch, or
// of one row, are refused where bytes are shared and only there; of other pitches at least there.
static void check_overlap(int64_t rows, int64_t g_rows, int64_t cols, int64_t inner, int64_t g_stride, int64_t o_stride, int64_t d) {
  const uint64_t g0 = 1 << 20, o0 = g0 + d;
  static char used[1 << 16];
  std::memset(used, 0, sizeof used);
  const int64_t lo = -(1 << 15);
  for (int64_t r = 0; r < g_rows; ++r)
    for (int64_t b = 0; b < 2 * inner; ++b) used[2 * r * g_stride + b - lo] = 1;
  bool shared = false;
  for (int64_t r = 0; r < rows; ++r)
    for (int64_t b = 0; b < 4 * cols; ++b) shared |= used[d + 4 * r * o_stride + b - lo] != 0;
  // the gradient's g (bfloat16) and output (float32): rows of g are rows of the output
  auto at = [](uint64_t a) { return (void*)(uintptr_t)a; };
  const bool exact = 2 * g_stride == 4 * o_stride || rows == 1;
  if (g_rows == rows) {
    const pat_status_t st = pat_mx_matmul_grad(at(g0), g_stride, 0, at(1 << 25), at(1 << 26), rows, inner, cols, at(o0), o_stride,
                                               PAT_FLOAT32, nullptr, 0, nullptr);
    CHECK(shared || exact ? st == (shared ? PAT_ERR_INVALID_ARGUMENT : PAT_OK) : true, "%lld %lld %lld %lld %lld %lld: %d", (long long)rows,
          (long long)cols, (long long)inner, (long long)g_stride, (long long)o_stride, (long long)d, st);
  }
  // an embedding's table (bfloat16) of g_rows, and as many columns as the output
  if (inner == cols) {
    const pat_status_t st = pat_embedding(at(1 << 25), 4, rows, at(g0), g_stride, PAT_BFLOAT16, 0, g_rows, cols, 1.0f, at(o0), o_stride,
                                          PAT_FLOAT32, nullptr);
    const bool same = exact || g_rows == 1;
    CHECK(shared || same ? st == (shared ? PAT_ERR_INVALID_ARGUMENT : PAT_OK) : true, "embedding %lld %lld %lld %lld %lld %lld: %d",
          (long long)rows, (long long)g_rows, (long long)cols, (long long)g_stride, (long long)o_stride, (long long)d, st);
  }
}

int main() {
  unsigned long long x = 88172645463325252ull;
  auto rnd = [&](int64_t most) {  // 1 ... most, spread over the logarithm
    x ^= x << 13, x ^= x >> 7, x ^= x << 17;
    int bits = 0;
    while ((most >> bits) > 1) ++bits;
    const int64_t v = 1 + (int64_t)((x >> 8) % (1ull << (x % (bits + 1))));
    return v < most ? v : most;
  };
  const int64_t most = ((int64_t)1 << 31) - 1;
  for (int e = 1; e < 31; ++e)
    for (int64_t total = (int64_t)1 << 34; total <= (int64_t)1 << 38; total *= 2)
      for (int64_t d = -3; d <= 3; ++d) {
        const int64_t rows = (int64_t)1 << e, cols = total / rows + d;
        if (cols >= 1 && cols <= most) check_dropout(rows, cols), check_dropout(cols, rows);
      }
  for (int i = 0; i < 200000; ++i) check_dropout(rnd(most), rnd(most));
  check_dropout(most, most);
  for (int e = 0; e <= 26; ++e)
    for (int f = 0; f <= 26; ++f)
      for (int d = -17; d <= 17; ++d) check_product(((int64_t)1 << e) + d, ((int64_t)1 << f) + d);
  for (int i = 0; i < 200000; ++i) check_product(rnd((1 << 26) + 100), rnd((1 << 26) + 100));
  for (int i = 0; i < 300000; ++i) {
    const int64_t rows = rnd(6), cols = rnd(12), inner = rnd(4) == 1 ? cols : rnd(20), o_stride = cols + rnd(30) - 1;
    int64_t g_stride = rnd(3) == 1 ? inner + rnd(40) - 1 : 2 * o_stride;
    if (g_stride < inner) g_stride = inner;
    check_overlap(rows, rnd(2) == 1 ? rnd(6) : rows, cols, inner, g_stride, o_stride, 4 * (rnd(600) - rnd(600)));
  }
  std::printf("%d checks, %d failures\n", g_checked, g_failures);
  return g_failures != 0;
}
