// Host side of a layer's operators (layer.cpp, layer_shape.hpp) with launches that only record: every size that is accepted
// gives launches of fewer than 2^32 lanes that reach all of their work, workspaces hold what is put there, and which places
// of outputs beside inputs the entry points take.
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "../../include/pat_ops.h"
#include "layer_shape.hpp"

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

namespace pat {
static hipError_t g_result = hipSuccess;
static int g_launches = 0;
static int64_t g_lanes = 0;
static Epilogue g_epilogue;
static NormArgs g_norm;
static NormGradArgs g_norm_grad;
static hipError_t launched() {
  ++g_launches;
  return g_result;
}
void record_hip_error(hipError_t) {}
hipError_t launch_mxb_quantize(Mat, Elem, int64_t, int64_t, MxbOut, hipStream_t) { return launched(); }
hipError_t launch_mxb_dequantize(MxbMat, int64_t, int64_t, MatOut, Elem, hipStream_t) { return launched(); }
hipError_t launch_mxb_product(MxbMat, MxMat, int64_t m, int64_t n, int64_t k, const Epilogue& e, hipStream_t) {
  g_epilogue = e;
  const bool blocks = e.gated && (!e.out.p || e.saved_a.codes);
  const int64_t columns = blocks ? groups_of(n) * 128 : n, rows = e.gated ? 2 : 1;
  if (k > 0 && m > (e.gated ? kFewGated : kFewLinear)) {
    const int tile = layer_tile(m, rows * n), side = tile == 32 ? 64 : tile == 64 ? 128 : tile;  // of the weight's rows
    const int64_t tiles = (int64_t)ceil_div(m, tile < 128 ? 64 : tile) * (int64_t)ceil_div(columns, side / rows);
    g_lanes = (int64_t)ceil_div(tiles, 8) * 8 * (tile == 256 ? 512 : 256);
  } else {
    const int tokens = m <= 16 ? 16 : m <= 32 || e.gated ? 32 : 48, each = e.gated ? 32 : 16 * few_columns_sixteens(n);
    const int64_t tiles_n = (int64_t)ceil_div(columns, each), band = few_band(m, tiles_n, tokens);
    CHECK(band > 0 && (band == m || band % tokens == 0), "%lld %lld", (long long)m, (long long)n);
    g_lanes = (int64_t)ceil_div(band, tokens) * tiles_n * 512;
  }
  return launched();
}
size_t mx_grad_workspace(int64_t rows, int64_t, int64_t cols) { return (size_t)(rows * cols); }
hipError_t launch_mxb_weight_grad(Mat, MxbMat, int64_t, int64_t, int64_t, MatOut, Elem, void*, hipStream_t) { return launched(); }
hipError_t launch_gated_grad(Mat, Elem, MxbMat, MxbMat, int64_t, int64_t, Act, MatOut, hipStream_t) { return launched(); }
hipError_t launch_rms_norm(const NormArgs& a, hipStream_t) {
  g_norm = a;
  return launched();
}
size_t rms_norm_grad_workspace(int64_t rows, int64_t cols) {
  const NormGradPlan p = norm_grad_plan(rows, cols);
  return (size_t)(p.wgs * p.pitch) * 4 + (size_t)rows * 8;
}
hipError_t launch_rms_norm_grad(const NormGradArgs& a, void*, hipStream_t) {
  g_norm_grad = a;
  return launched();
}
}  // namespace pat

static void check_plan(const NormPlan& p, int64_t rows, int64_t units, int most, int vectors) {
  const long long r = rows, u = units;
  CHECK(p.lanes >= 1 && p.lanes <= most && (p.lanes <= 64 ? (p.lanes & (p.lanes - 1)) == 0 : p.lanes % 64 == 0), "%lld %lld: %d", r, u, p.lanes);
  CHECK(p.threads % p.lanes == 0 && p.threads % 64 == 0 && p.threads <= most, "%lld %lld: %d of %d", r, u, p.threads, p.lanes);
  CHECK(p.vectors == 0 ? units > (int64_t)most * vectors : (int64_t)p.lanes * p.vectors >= units && p.vectors <= vectors, "%lld %lld: %d x %d", r, u,
        p.lanes, p.vectors);
  // a wave is of one row where lanes have several vectors
  CHECK(p.vectors < 2 || p.lanes % 64 == 0, "%lld %lld: %d x %d", r, u, p.lanes, p.vectors);
  CHECK(p.wgs >= 1 && p.wgs * p.threads < kLanes, "%lld %lld: %lld", r, u, (long long)p.wgs);
}

static void check_norm(int64_t rows, int64_t cols) {
  const int64_t units = (cols + 7) / 8;
  check_plan(norm_plan(rows, cols, false), rows, units, kNormMost, 2);
  const NormPlan q = norm_plan(rows, cols, true);
  check_plan(q, rows, groups_of(cols) * 16, kNormMost, 2);
  CHECK(q.lanes % 16 == 0, "%lld: %d", (long long)cols, q.lanes);  // sixteen lanes have a group
  if (rows >= (int64_t)1 << 28 || cols >= (int64_t)1 << 26) return;
  const NormGradPlan g = norm_grad_plan(rows, cols);
  check_plan(g, rows, units, kNormGradMost, 4);
  // rows beside each other in a workgroup are joined in LDS for 256 lanes of one vector
  CHECK(g.threads == g.lanes || (g.vectors == 1 && g.threads <= kStripThreads), "%lld %lld: %d", (long long)rows, (long long)cols, g.threads);
  CHECK(g.pitch >= cols && g.pitch % 8 == 0 && g.strips * 8 * kStripThreads >= cols, "%lld", (long long)cols);
  CHECK(g.wgs <= rows && g.wgs < 65536 && g.strips * g.wgs * kStripThreads < kLanes, "%lld %lld: %lld", (long long)rows, (long long)cols, (long long)g.wgs);
}

static void* at(uint64_t a) { return (void*)(uintptr_t)a; }

static void check_products(int64_t m, int64_t n) {
  if (m < 1 || n < 1) return;
  for (int64_t k : {0, 1, 200})
    for (int kind = 0; kind < 4; ++kind) {  // linear, gated to a matrix, with a checkpoint, to blocks
      g_lanes = 0;
      const pat_status_t st =
          kind == 0 ? pat_mxb_linear(at(1ull << 60), at(1ull << 59), at(1ull << 58), at(1ull << 57), m, n, k, nullptr, 0, at(4096), n, PAT_FLOAT32, nullptr)
                    : pat_gated(at(1ull << 60), at(1ull << 59), at(1ull << 58), at(1ull << 57), m, n, k, PAT_SILU, kind == 3 ? nullptr : at(4096), n,
                                PAT_FLOAT32, kind == 3 ? at(4096) : nullptr, kind == 3 ? at(1ull << 55) : nullptr, kind == 2 ? at(1ull << 62) : nullptr,
                                kind == 2 ? at(1ull << 56) : nullptr, nullptr);
      CHECK(st == PAT_OK ? g_lanes > 0 : st == PAT_ERR_UNSUPPORTED && m * n >= (int64_t)1 << 24, "%lld %lld %d: %d", (long long)m, (long long)n, kind, st);
      CHECK(g_lanes < kLanes, "%lld %lld %lld %d: %lld lanes", (long long)m, (long long)n, (long long)k, kind, (long long)g_lanes);
    }
}

// Where the norm's total and output may stand: nowhere that shares a byte with what is read, but in its place.
static void check_norm_places(int64_t rows, int64_t cols, int64_t x_stride, int64_t o_stride, int64_t d, bool total) {
  const uint64_t x0 = 1 << 20, o0 = x0 + d;
  static char used[1 << 16];
  std::memset(used, 0, sizeof used);
  const int64_t lo = -(1 << 15);
  for (int64_t r = 0; r < rows; ++r)
    for (int64_t b = 0; b < 4 * cols; ++b) used[4 * r * x_stride + b - lo] = 1;
  bool shared = false;
  for (int64_t r = 0; r < rows; ++r)
    for (int64_t b = 0; b < 4 * cols; ++b) shared |= used[d + 4 * r * o_stride + b - lo] != 0;
  const bool same = d == 0 && (rows == 1 || x_stride == o_stride), exact = x_stride == o_stride || rows == 1;
  const pat_status_t st = total ? pat_rms_norm(at(x0), x_stride, at(1 << 24), cols, PAT_FLOAT32, at(1 << 25), PAT_FLOAT32, rows, cols, 0.1f, at(o0), o_stride,
                                               at(1 << 26), cols, PAT_BFLOAT16, nullptr, nullptr, nullptr)
                                : pat_rms_norm(at(x0), x_stride, nullptr, 0, PAT_FLOAT32, at(1 << 25), PAT_FLOAT32, rows, cols, 0.1f, nullptr, 0, at(o0),
                                               o_stride, PAT_FLOAT32, nullptr, nullptr, nullptr);
  CHECK(same ? st == PAT_OK : shared || exact ? st == (shared ? PAT_ERR_INVALID_ARGUMENT : PAT_OK) : true, "%lld %lld %lld %lld %lld: %d", (long long)rows,
        (long long)cols, (long long)x_stride, (long long)o_stride, (long long)d, st);
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
  const int64_t top = ((int64_t)1 << 31) - 1;
  for (int64_t cols = 1; cols < 40000; ++cols)
    for (int64_t rows : {1, 7, 2047, 2048, 100000}) check_norm(rows, cols);
  for (int i = 0; i < 200000; ++i) check_norm(rnd(top), rnd(top));
  check_norm(top, top), check_norm(top, 1), check_norm(1, top);
  for (int e = 0; e <= 26; ++e)
    for (int f = 0; f <= 26; ++f)
      for (int d = -17; d <= 17; ++d) check_products(((int64_t)1 << e) + d, ((int64_t)1 << f) + d);
  for (int i = 0; i < 100000; ++i) check_products(rnd((1 << 26) + 100), rnd((1 << 26) + 100));
  for (int i = 0; i < 200000; ++i) {
    const int64_t rows = rnd(6), cols = rnd(12), x_stride = cols + rnd(30) - 1, o_stride = rnd(3) == 1 ? cols + rnd(30) - 1 : x_stride;
    check_norm_places(rows, cols, x_stride, o_stride, rnd(4) == 1 ? 0 : 4 * (rnd(600) - rnd(600)), i & 1);
  }

  // The checkpoint's halves, and what reaches the launches.
  g_launches = 0;
  CHECK(pat_gated(at(1 << 20), at(1 << 21), at(1 << 22), at(1 << 23), 3, 200, 300, PAT_GELU, nullptr, 0, PAT_INT32, at(1 << 24), at(1 << 25), at(1 << 26),
                  at(1 << 27), nullptr) == PAT_OK, "blocks");
  CHECK(g_epilogue.gated && g_epilogue.act == Act::gelu && !g_epilogue.out.p && g_epilogue.blocks.codes == at(1 << 24), "epilogue");
  CHECK(g_epilogue.saved_b.codes == (uint8_t*)at(1 << 26) + 3 * 256 && g_epilogue.saved_b.scales == (uint8_t*)at(1 << 27) + 3 * 8, "halves");
  g_result = hipErrorUnknown;
  CHECK(pat_mxb_linear(at(1 << 20), at(1 << 21), at(1 << 22), at(1 << 23), 3, 200, 300, nullptr, 0, at(1 << 24), 200, PAT_BFLOAT16, nullptr) == PAT_ERR_HIP,
        "a launch's error");
  CHECK(!g_epilogue.gated && !g_epilogue.residual.p && g_epilogue.dtype == Elem::b16 && g_launches == 2, "linear");
  g_result = hipSuccess;
  const size_t need = pat_rms_norm_grad_workspace(5, 100);
  CHECK(need > 0 && need % 4 == 0, "%zu", need);
  CHECK(pat_rms_norm_grad(at(1 << 20), 100, PAT_FLOAT32, at(1 << 21), 100, PAT_BFLOAT16, at(1 << 22), PAT_FLOAT32, nullptr, 0, 5, 100, 0.0f, at(1 << 20), 100,
                          at(1 << 23), at(1 << 24), need, nullptr) == PAT_OK && g_norm_grad.out.p == g_norm_grad.g.p, "in place");
  CHECK(pat_rms_norm_grad_workspace(0, 100) == 0 && pat_rms_norm_grad_workspace((size_t)1 << 28, 1) == 0, "no workspace");
  CHECK(pat_mxb_weight_grad_workspace((size_t)1 << 26, 8, 8) == 0, "no workspace");
  std::printf("%d checks, %d failures\n", g_checked, g_failures);
  return g_failures != 0;
}
