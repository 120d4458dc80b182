// What the operators' launches ask for (ops_shape.hpp): a launch holds fewer than 2^32 lanes, and has to reach all its work.
#include <cstdio>
#include <cstdlib>

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

// Accepted: fewer than 2^26 rows and columns, and 2^31 tiles of 16 x 16.
static void check_product(int64_t rows, int64_t cols) {
  const int64_t most = ((int64_t)1 << 26) - 1;
  if (rows < 1 || cols < 1 || rows > most || cols > most) return;
  if ((rows + 15) / 16 * ((cols + 15) / 16) >= (int64_t)1 << 31) return;
  const int64_t wgs = narrow_wgs(rows, cols);
  CHECK(wgs >= 1 && wgs * 64 < kLanes, "%lld %lld: %lld workgroups", (long long)rows, (long long)cols, (long long)wgs);
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
  for (int i = 0; i < 200000; ++i) check_product(rnd(most >> 5), rnd(most >> 5));
  std::printf("%d checks, %d failures\n", g_checked, g_failures);
  return g_failures != 0;
}
