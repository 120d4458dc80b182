// How a layer's operators are launched, by the functions that the launches themselves use (layer_shape.hpp): every accepted size
// of a product gets workgroups for all of its output and fewer than 2^32 lanes a launch, and the workspace of the norm's
// gradients holds everything that the kernels put there, each part in its own place.
#include <cstdio>
#include <utility>

#include "layer_shape.hpp"

using namespace pat;

static int g_failures = 0;
static long long g_checked = 0;
#define CHECK(cond, ...)                                     \
  do {                                                       \
    ++g_checked;                                             \
    if (!(cond)) {                                           \
      if (++g_failures < 20) std::printf("%s: ", #cond), std::printf(__VA_ARGS__), std::printf("\n"); \
    }                                                        \
  } while (0)

static const int64_t kLanes = (int64_t)1 << 32;

static void check_product(int64_t m, int64_t n, int64_t k, bool gated, bool blocks) {
  const int64_t rows = gated ? 2 * n : n;
  if (m < 1 || n < 1 || m >= 1 << 26 || rows >= 1 << 26) return;
  if ((int64_t)ceil_div(m, 16) * (int64_t)ceil_div(rows, 16) >= 1 << 30) return;  // refused
  const ProductPlan p = product_plan(m, n, k, gated, blocks);
  const long long M = m, N = n, K = k;
  const int64_t width = blocks ? groups_of(n) * 128 : n;
  CHECK(p.wgs > 0 && p.wgs * p.threads < kLanes, "%lld %lld %lld %d: %lld", M, N, K, gated, (long long)p.wgs);
  if (p.tile) {
    CHECK(k > 0, "%lld %lld", M, N);  // the tiles' first loads need a group
    const int64_t tokens = tile_tokens(p.tile), columns = gated ? tile_rows(p.tile) / 2 : tile_rows(p.tile);
    CHECK(p.tile == 256 || p.tile == 128 || p.tile == 64 || p.tile == 32, "%d", p.tile);
    CHECK(p.tiles_n * columns >= width && (p.tiles_n - 1) * columns < width, "%lld %lld: %lld", M, N, (long long)p.tiles_n);
    CHECK(p.wgs % 8 == 0 && p.wgs >= (int64_t)ceil_div(m, tokens) * p.tiles_n, "%lld %lld: %lld", M, N, (long long)p.wgs);
    CHECK(p.band == m, "%lld %lld", M, N);
  } else {
    const int64_t tokens = 16 * p.tokens, columns = 16 * p.columns;
    CHECK(p.tokens >= 1 && p.tokens <= (gated ? 2 : 3) && p.threads == 64 * kFewWaves, "%lld %lld: %d", M, N, p.tokens);
    CHECK(gated ? p.columns == 2 : p.columns == 1 || p.columns == 2 || p.columns == 4, "%lld %lld: %d", M, N, p.columns);
    CHECK(p.tiles_n * columns >= width && (p.tiles_n - 1) * columns < width, "%lld %lld: %lld", M, N, (long long)p.tiles_n);
    // launches follow each other a band apart: each of whole workgroups' tokens but the last
    CHECK(p.band > 0 && p.band <= m && (p.band == m || p.band % tokens == 0), "%lld %lld: %lld", M, N, (long long)p.band);
    CHECK(p.wgs == (int64_t)ceil_div(p.band, tokens) * p.tiles_n, "%lld %lld: %lld", M, N, (long long)p.wgs);
    CHECK(kFewWaves * p.tokens * p.columns * (gated ? 2 : 1) <= 160, "%lld %lld", M, N);  // KB of LDS
  }
}

static void check_space(int64_t rows, int64_t cols) {
  if (rows < 1 || cols < 1 || rows >= 1 << 28 || cols >= 1 << 26) return;
  const NormGradPlan p = norm_grad_plan(rows, cols);
  const NormGradSpace s = norm_grad_space(p, rows);
  const long long r = rows, c = cols;
  CHECK(p.pitch >= cols && p.pitch % 8 == 0, "%lld %lld: %lld", r, c, (long long)p.pitch);
  // parts that are added up: rows of whole vectors of four floats
  if (p.wgs > 1) CHECK(s.parts >= p.wgs * p.pitch, "%lld %lld: %lld", r, c, (long long)s.parts);
  if (p.vectors == 0) CHECK(s.rows_at >= s.parts && s.rows_at % 2 == 0 && s.bytes >= (size_t)(s.rows_at + 2 * rows) * 4, "%lld %lld", r, c);
  CHECK(s.bytes >= (size_t)s.parts * 4 && s.bytes < (size_t)1 << 40, "%lld %lld: %zu", r, c, s.bytes);
  CHECK((s.bytes == 0) == (p.vectors > 0 && p.wgs == 1), "%lld %lld: %zu", r, c, s.bytes);
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
  auto products = [&](int64_t m, int64_t n) {
    for (int64_t k : {0, 1, 200, 2048, 2049, 20000, (1 << 24) - 1})
      for (int kind = 0; kind < 3; ++kind) check_product(m, n, k, kind > 0, kind > 1);
  };
  for (int64_t m = 1; m < 70; ++m)
    for (int64_t n = 1; n < 20000; n += 1 + n / 37) products(m, n);
  for (int e = 0; e <= 26; ++e)
    for (int f = 0; f <= 26; ++f)
      for (int d = -17; d <= 17; ++d) products(((int64_t)1 << e) + d, ((int64_t)1 << f) + d);
  for (int i = 0; i < 100000; ++i) products(rnd((1 << 26) + 100), rnd((1 << 26) + 100));
  // Gated products of 17 to 32 tokens: the faster kernel of each side of the rule, as measured.
  for (int64_t m : {17, 24, 32}) {
    for (const auto& s : {std::pair{512, 2000}, {2048, 2000}, {1024, 4096}, {512, 8192}, {1024, 8192}, {512, 16384}})
      CHECK(product_plan(m, s.first, s.second, true, false).tile != 0, "%lld %d %d", (long long)m, s.first, s.second);
    for (const auto& s : {std::pair{512, 512}, {2048, 1333}, {8192, 1333}, {8192, 4096}, {16384, 4096}, {8192, 8192}})
      CHECK(product_plan(m, s.first, s.second, true, false).tile == 0, "%lld %d %d", (long long)m, s.first, s.second);
  }
  for (int64_t cols = 1; cols < 40000; ++cols)
    for (int64_t rows : {1, 2, 7, 255, 256, 257, 513, 2048, 100000}) check_space(rows, cols);
  for (int i = 0; i < 200000; ++i) check_space(rnd(1 << 28), rnd(1 << 26));
  std::printf("%lld checks, %d failures\n", g_checked, g_failures);
  return g_failures != 0;
}
