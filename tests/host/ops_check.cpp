// Host side of the operators (ops.cpp, ops_shape.hpp) with launches that only record their arguments: how sizes are cut
// into workgroups, slices and pieces, and what reaches a launch from the C entry points.
#include <cstdio>
#include <cstdlib>

#include "../../include/pat_ops.h"
#include "ops_shape.hpp"

namespace pat {

int g_launches = 0;
hipError_t g_result = hipSuccess;
hipError_t g_recorded = hipSuccess;

void record_hip_error(hipError_t e) { g_recorded = e; }
static hipError_t launched() {
  ++g_launches;
  return g_result;
}
hipError_t launch_mx_quantize(Mat, Elem, int64_t, int64_t, uint8_t*, uint8_t*, hipStream_t) { return launched(); }
hipError_t launch_mx_dequantize(MxMat, int64_t, int64_t, MatOut, Elem, hipStream_t) { return launched(); }
hipError_t launch_mx_matmul(MxMat, MxMat, int64_t, int64_t, int64_t, MatOut, Elem, hipStream_t) { return launched(); }
size_t mx_linear_workspace(int64_t m, int64_t, int64_t k) { return (size_t)(m * groups_of(k)) * 68; }
hipError_t launch_mx_linear(Mat, Elem, MxMat, int64_t, int64_t, int64_t, MatOut, Elem, void*, hipStream_t) {
  return launched();
}
size_t mx_grad_workspace(int64_t rows, int64_t inner, int64_t cols) {
  const GradPlan p = grad_plan(rows, inner, cols);
  return p.slices > 1 ? (size_t)(p.slices * rows * ((cols + 7) / 8 * 8)) * 4 : 0;
}
hipError_t launch_mx_grad(Mat, bool, MxMat, int64_t, int64_t, int64_t, MatOut, Elem, void*, hipStream_t) {
  return launched();
}
hipError_t launch_embedding(const void*, int, int64_t, Mat, Elem, int64_t, int64_t, int64_t, float, MatOut, Elem,
                            hipStream_t) {
  return launched();
}
size_t embedding_grad_workspace(int64_t ntokens, int64_t, int64_t) { return (size_t)ntokens * 16; }
hipError_t launch_embedding_grad(const void*, int, int64_t, Mat, Elem, int64_t, int64_t, int64_t, float, MatOut, Elem, void*,
                                 hipStream_t) {
  return launched();
}
DropoutArgs g_dropout;
hipError_t launch_dropout(const DropoutArgs& a, Elem, hipStream_t) {
  g_dropout = a;
  return launched();
}

}  // namespace pat

using namespace pat;

static int g_failures = 0, g_checked = 0;
#define CHECK(cond, ...)                                     \
  do {                                                       \
    ++g_checked;                                             \
    if (!(cond)) {                                           \
      if (++g_failures < 20) std::printf("%s: ", #cond), std::printf(__VA_ARGS__), std::printf("\n"); \
    }                                                        \
  } while (0)

static void check_grad(int64_t rows, int64_t inner, int64_t cols) {
  const GradPlan p = grad_plan(rows, inner, cols);
  const long long r = rows, n = inner, c = cols;
  CHECK(p.tile == 64 || p.tile == 128 || p.tile == 256, "%lld %lld %lld", r, n, c);
  CHECK(p.slices >= 1 && p.slices <= 65535, "%lld %lld %lld: %d", r, n, c, p.slices);
  if (p.slices == 1) return;
  const int64_t last = inner - (p.slices - 1) * p.slice;
  CHECK(p.tile == 128 && p.slice % 64 == 0, "%lld %lld %lld", r, n, c);
  CHECK(last >= 8 && last <= p.slice, "%lld %lld %lld: slice %lld, last %lld", r, n, c, (long long)p.slice, (long long)last);
}

static void check_embedding(int64_t ntokens, int64_t rows, int64_t cols) {
  const long long t = ntokens, r = rows, c = cols;
  const SortPlan s = sort_plan(ntokens, rows);
  CHECK(((int64_t)1 << (s.bits * s.passes)) >= rows, "%lld %lld: %d bits, %d passes", t, r, s.bits, s.passes);
  CHECK(s.bits >= 1 && s.bits <= (ntokens <= kSmallTokens ? kSmallBits : kMaxBits), "%lld %lld", t, r);
  CHECK(s.bits * s.passes < 64 && s.tile % kSortThreads == 0, "%lld %lld", t, r);
  CHECK(s.tile * s.tiles >= ntokens && s.tiles <= 128, "%lld: %lld tiles of %lld", t, (long long)s.tiles, (long long)s.tile);
  const SumPlan u = sum_plan(ntokens, rows, cols);
  CHECK(u.lanes >= 1 && u.lanes <= 256 && (u.lanes & (u.lanes - 1)) == 0, "%lld", c);
  CHECK(u.piece % 8 == 0 && u.pieces * u.piece >= ntokens && u.pieces <= 1 << 20, "%lld", t);
  CHECK(u.sum_wgs * (256 / u.lanes) >= u.pieces, "%lld %lld", t, c);
  CHECK(u.col_wgs * 8 * u.lanes >= cols && u.pitch >= cols && u.pitch % 8 == 0, "%lld", c);
  CHECK(u.zero_wgs * kZeroRows >= rows, "%lld", r);
  // what a launch holds: fewer than 2^32 lanes, 65536 rows of workgroups
  CHECK((u.sum_wgs + u.zero_wgs) * 256 < (int64_t)1 << 32 && u.col_wgs < 65536 && (cols + 255) / 256 < 65536, "%lld %lld %lld",
        t, r, c);
}

static void check_calls() {
  char* base = (char*)(uintptr_t)0x100000000ull;  // never read: launches only record
  auto at = [&](size_t off) { return (void*)(base + off); };
  // an error of a launch comes back as one, and is kept
  g_result = hipErrorInvalidConfiguration;
  CHECK(pat_mx_quantize(at(0), 64, 4, 64, PAT_FLOAT32, at(0x10000), at(0x20000), nullptr) == PAT_ERR_HIP, "quantize");
  CHECK(g_recorded == hipErrorInvalidConfiguration, "recorded");
  g_result = hipSuccess;
  // sizes whose products pass 64 bits are refused, not wrapped
  CHECK(pat_mx_quantize(at(0), INT64_MAX, 4, 64, PAT_FLOAT32, at(0x10000), at(0x20000), nullptr) == PAT_ERR_INVALID_ARGUMENT,
        "stride");
  CHECK(pat_embedding(at(0), 8, SIZE_MAX, at(0x1000), 8, PAT_FLOAT32, 0, 4, 8, 1.0f, at(0x2000), 8, PAT_FLOAT32, nullptr) ==
            PAT_ERR_UNSUPPORTED, "tokens");
  CHECK(pat_mx_linear_workspace(SIZE_MAX, 1, 1) == 0 && pat_embedding_grad_workspace(SIZE_MAX, 1, 1) == 0, "workspace");
  // dropout: P and the scale of what is kept; in place and not
  const int before = g_launches;
  CHECK(pat_dropout(at(0), 8, nullptr, 0, at(0), 8, 4, 8, PAT_FLOAT32, 0.5, 7, 9, 8, nullptr) == PAT_OK, "in place");
  CHECK(g_dropout.drop == 32768 && g_dropout.scale == 2.0f && g_dropout.seed == 7 && g_dropout.index == 9, "half");
  CHECK(pat_dropout(at(0), 8, at(0x1000), 8, at(0x1000), 8, 4, 8, PAT_BFLOAT16, 1.0, 7, 9, 8, nullptr) == PAT_OK, "residual");
  CHECK(g_dropout.drop == 65536 && g_dropout.scale == 0.0f, "all");
  CHECK(pat_dropout(at(0), 9, nullptr, 0, at(0), 8, 4, 8, PAT_FLOAT32, 0.5, 7, 9, 8, nullptr) == PAT_ERR_INVALID_ARGUMENT,
        "strides differ");
  CHECK(g_launches == before + 2, "launches %d", g_launches - before);
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
  for (int64_t tiles = 1; tiles <= 33; ++tiles)
    for (int64_t inner = 4000; inner < 9000; ++inner) check_grad(128, inner, 128 * tiles);
  for (int64_t e = 12; e < 24; ++e)
    for (int64_t d = -70; d <= 70; ++d) check_grad(100, ((int64_t)1 << e) + d, 500);
  for (int i = 0; i < 200000; ++i) check_grad(rnd((1 << 26) - 1), rnd((1 << 24) - 1), rnd((1 << 26) - 1));
  for (int64_t n = 1; n < 9000; ++n) check_embedding(n, 1 + n * 37 % 70000, 1 + n * 13 % 5000);
  for (int i = 0; i < 200000; ++i) check_embedding(rnd((1 << 28) - 1), rnd((1 << 28) - 1), rnd((1 << 23) - 1));
  check_calls();
  std::printf("%d checks, %d failures\n", g_checked, g_failures);
  return g_failures != 0;
}
