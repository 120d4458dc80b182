// Root-mean-square norm of rows, after a residual's addition, and its gradients.
#include <algorithm>

#include "layer_device.hpp"
#include "layer_shape.hpp"

namespace pat {
namespace {

// How a wave's part of a row of `cols` columns is cut into lanes' eights (fours, with the second four `gap` columns after the
// first, where a type has 4 bytes):
//   kAll   every vector exists;
//   kSome  a vector exists or does not;
//   kEnds  one that would go over the row's end ends there and is moved down (rows of 4 columns and more);
//   kOne   columns one by one.
// I: the type of places in a row, int where rows are short enough.
enum Cut { kAll, kSome, kEnds, kOne };
template <Cut C>
struct CutOf {
  static constexpr Cut value = C;
};
// f by what this wave has; `last`: the lane's columns from the first of its last vector to the row's end.  Waves of one
// workgroup may go different ways, through as many barriers.
template <bool SPLIT, typename I, typename F>
__device__ __forceinline__ void cut(I cols, I last, I gap, F f) {
  if (__all(last >= gap + 4)) f(CutOf<kAll>{});
  else if (cols % (SPLIT ? 4 : 8) == 0) f(CutOf<kSome>{});
  else if (cols >= 4) f(CutOf<kEnds>{});
  else f(CutOf<kOne>{});
}

// Bytes from a row's start to its column `col`; without a sign where they fit, an address is a scalar and 32 bits.
template <int BYTES>
__device__ __forceinline__ uint32_t bytes_to(int col) { return (uint32_t)col * BYTES; }
template <int BYTES>
__device__ __forceinline__ int64_t bytes_to(int64_t col) { return col * BYTES; }

// A lane's 8 columns from `col` of a row as they are in memory; nothing is done with what is loaded, so that a row's loads are
// on their way together.  Columns behind the row's end are zero once they are widened.
template <typename T>
struct Raw {
  typename T::vec4 lo, hi;
};
template <typename T, bool SPLIT, Cut C, bool NT = false, typename I>
__device__ __forceinline__ Raw<T> load_raw(const void* row, I col, I cols, I gap) {
  typedef typename T::vec4 V;
  const I n = cols - col;
  const char* p = (const char*)row + bytes_to<T::kBytes>(col);
  if constexpr (C == kOne) {
    float v[8];
    load8<T, SPLIT, false, kFew>(p, n, gap, v);
    return {T::narrow(v), T::narrow(v + 4)};
  } else if constexpr (C <= kSome && !SPLIT && T::kBytes == 2) {
    const v4u a = ldg<v4u, NT, 2>(C == kAll ? p : p + min((I)0, n - 8) * 2);
    return {{a[0], a[1]}, {a[2], a[3]}};
  } else {
    const I at = C == kAll ? 0 : min((I)0, n - 4), to = C == kAll ? gap : min(gap, n - 4);
    return {ldg<V, NT, T::kBytes>(p + at * T::kBytes), ldg<V, NT, T::kBytes>(p + to * T::kBytes)};
  }
}
template <typename T, bool SPLIT, Cut C, typename I>
__device__ __forceinline__ void widen(const Raw<T>& r, I col, I cols, I gap, float (&v)[8]) {
  const I n = cols - col;
  T::widen(r.lo, v);
  T::widen(r.hi, v + 4);
  if constexpr (C == kSome) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = n > (SPLIT && i >= 4 ? gap : 0) ? v[i] : 0.0f;
  } else if constexpr (C == kEnds) {
    move_down(v, max((I)0, 4 - n));
    move_down(v + 4, max((I)0, gap + 4 - n));
  }
}
// The same of a vector whose type is known at the launch alone.
struct RawWeight {
  v4u lo, hi;
};
template <bool SPLIT, Cut C, typename I>
__device__ __forceinline__ RawWeight load_raw(Elem e, const void* weight, I col, I cols, I gap) {
  if (e == Elem::f32) {
    const Raw<F32> r = load_raw<F32, SPLIT, C>(weight, col, cols, gap);
    return {__builtin_bit_cast(v4u, r.lo), __builtin_bit_cast(v4u, r.hi)};
  }
  const Raw<B16> r = load_raw<B16, SPLIT, C>(weight, col, cols, gap);
  return {v4u{r.lo[0], r.lo[1], r.hi[0], r.hi[1]}, v4u{0, 0, 0, 0}};
}
template <bool SPLIT, Cut C, typename I>
__device__ __forceinline__ void widen(Elem e, const RawWeight& r, I col, I cols, I gap, float (&v)[8]) {
  if (e == Elem::f32) widen<F32, SPLIT, C>({__builtin_bit_cast(v4f, r.lo), __builtin_bit_cast(v4f, r.hi)}, col, cols, gap, v);
  else widen<B16, SPLIT, C>({{r.lo[0], r.lo[1]}, {r.lo[2], r.lo[3]}}, col, cols, gap, v);
}
template <typename T, bool SPLIT, Cut C, bool NT = false, typename I>
__device__ __forceinline__ void store_cols(void* row, I col, I cols, I gap, const float (&v)[8]) {
  char* p = (char*)row + bytes_to<T::kBytes>(col);
  const I n = cols - col;
  if constexpr (C == kAll) store8<T, SPLIT, NT, kWhole>(p, n, gap, v);
  else if constexpr (C == kSome && !SPLIT) {
    if (n > 0) store8<T, SPLIT, NT, kWhole>(p, n, gap, v);
  } else store8<T, SPLIT, NT, kEnd>(p, n, gap, v);
}
template <typename T>
__device__ __forceinline__ const char* row_of(Mat m, int64_t r) {
  return (const char*)m.p + r * m.stride * T::kBytes;
}
template <typename T>
__device__ __forceinline__ char* row_of(MatOut m, int64_t r) {
  return (char*)m.p + r * m.stride * T::kBytes;
}

// The same in every turn of a loop, and read again there: kept over the loop it would take more registers than there are.
__device__ __forceinline__ const void* again(const void* weight) {
  asm volatile("" : "+s"(weight));
  return weight;
}

// N sums over the row's lanes; `part` is LDS of this turn, N floats a wave.
template <int N>
__device__ __forceinline__ void sum_of_row(float (&v)[N], int lanes, float* part) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = sum_of_lanes(v[i], min(lanes, 64));
  if (lanes <= 64) return;
  const int wave = threadIdx.x / 64, waves = lanes / 64, first = wave / waves * waves;
  if (threadIdx.x % 64 == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) part[wave * N + i] = v[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = part[first * N + i];
  for (int w = 1; w < waves; ++w)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += part[(first + w) * N + i];
}

// The first of a lane's columns in its u-th of U vectors: a wave's are beside each other, so that the last wave of a row alone
// meets its end.
template <bool SPLIT, int U>
struct Place {
  int lane, width;
  __device__ __forceinline__ Place(int lanes) : lane(threadIdx.x % lanes), width(min(lanes, 64)) {}
  __device__ __forceinline__ int operator()(int u) const { return (lane / width * U + u) * 8 * width + (int)lane_column<SPLIT>(lane % width); }
  __device__ __forceinline__ int gap() const { return (int)lane_gap<SPLIT>(width); }
};

// What leaves of a lane's 8 columns: t * scale * weight.
template <typename O, bool SPLIT, Cut C, typename I>
__device__ __forceinline__ void finish(const NormArgs& a, int64_t row, bool real, I col, I cols, I gap, const float (&t)[8], const RawWeight& raw,
                                       float scale) {
  float w[8], y[8];
  widen<SPLIT, C>(a.weight_dtype, raw, col, cols, gap, w);
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = t[i] * scale * w[i];
  if constexpr (O::kBytes == 1) {
    const int64_t groups = (a.cols + 127) / 128;
    uint32_t high = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (C != kAll) y[i] = col + i < cols ? y[i] : 0.0f;
      high = max(high, __float_as_uint(y[i]) & 0x7FFFFFFFu);
    }
    const uint32_t s = mxb_scale_byte(max_of_4(high)), sub = threadIdx.x % 16;
    const uint32_t four = or_of_16_by_4(s << (sub / 4 * 8));
    if (!real || col >= groups * 128) return;
    const int64_t g = row * groups + col / 128;
    stg<false>((char*)a.blocks.codes + g * 128 + sub * 8, v2u{mxb_codes(y[0], y[1], y[2], y[3], s), mxb_codes(y[4], y[5], y[6], y[7], s)});
    if (sub == 0) stg<false>((char*)a.blocks.scales + g * 4, four);
  } else {
    if (real) store_cols<O, SPLIT, C>(row_of<O>(a.out, row), col, cols, gap, y);
  }
}

// The sum of eight squares, added up apart, so that long rows' sums have an eighth of the terms.
__device__ __forceinline__ float squares(const float (&t)[8]) {
  float eight = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) eight = fmaf(t[i], t[i], eight);
  return eight;
}

// t of a lane's columns: x, or x + residual as its type holds it.
template <typename X, bool SPLIT, Cut C, typename I>
__device__ __forceinline__ void total_of(const Raw<X>& x, const Raw<X>& r, bool residual, I col, I cols, I gap, float (&t)[8]) {
  widen<X, SPLIT, C>(x, col, cols, gap, t);
  if (residual) {
    float v[8];
    widen<X, SPLIT, C>(r, col, cols, gap, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = round_to(X{}, t[i] + v[i]);
  }
}

// Workgroups go through rows gridDim.x apart; a row's values stay in registers, the weight too, and the next row's loads are on
// their way before this row's sum.  Bound by memory: 8192 x 8192 bfloat16 with a residual (537 MB) in 80 us, 6.7 TB/s (94 with
// a workgroup for every row), float32 (1.07 GB) in 155, 6.9, float32 to 8 bits (874 MB) in 160, 5.5; loads and the total's
// stores are nontemporal, the output's, which are read next, are not.
template <typename X, typename O, int U>
__global__ __launch_bounds__(kNormMost) void norm_kernel(NormArgs a, int lanes) {
  constexpr bool SPLIT = O::kBytes > 1 && Split<X, O>::value;
  __shared__ float part[2][kNormMost / 64];
  const int side = blockDim.x / lanes, cols = (int)a.cols;
  const int64_t step = (int64_t)gridDim.x * side;
  const Place<SPLIT, U> at(lanes);
  const int gap = at.gap();
  // which of the rows beside each other; of lanes with several vectors a whole wave has one
  const int mine = U > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / lanes) : threadIdx.x / lanes;
  const bool residual = a.residual.p != nullptr;
  auto all = [&](auto how) {
    constexpr Cut C = decltype(how)::value;
    Raw<X> x[U], r[U];
    RawWeight weight[U];
    auto fetch = [&](int64_t base) {
      const int64_t row = min(base + mine, a.rows - 1);
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = load_raw<X, SPLIT, C, true>(row_of<X>(a.x, row), at(u), cols, gap);
      if (residual) {
#pragma unroll
        for (int u = 0; u < U; ++u) r[u] = load_raw<X, SPLIT, C, true>(row_of<X>(a.residual, row), at(u), cols, gap);
      }
    };
    int turn = 0;
    int64_t base = (int64_t)blockIdx.x * side;
    fetch(base);
#pragma unroll
    for (int u = 0; u < U; ++u) weight[u] = load_raw<SPLIT, C>(a.weight_dtype, a.weight, at(u), cols, gap);
    for (; base < a.rows; base += step, turn ^= 1) {
      const int64_t row = min(base + mine, a.rows - 1);
      const bool real = base + mine < a.rows;
      float t[U][8], sum[1] = {0.0f};
#pragma unroll
      for (int u = 0; u < U; ++u) {
        total_of<X, SPLIT, C>(x[u], r[u], residual, at(u), cols, gap, t[u]);
        if (a.total.p && real) store_cols<X, SPLIT, C, true>(row_of<X>(a.total, row), at(u), cols, gap, t[u]);
        sum[0] += squares(t[u]);
      }
      if (base + step < a.rows) fetch(base + step);
      sum_of_row(sum, lanes, part[turn]);
      const float scale = rsqrtf(sum[0] / (float)cols + a.eps);
#pragma unroll
      for (int u = 0; u < U; ++u) finish<O, SPLIT, C>(a, row, real, at(u), cols, gap, t[u], weight[u], scale);
    }
  };
  cut<SPLIT>(cols, cols - at(U - 1), gap, all);
}

// Rows that are too long for registers are read again, out of the total where there is one.  2048 x 20000 bfloat16 with a
// residual: 90 us, 5.4 TB/s without what is read again.
template <typename X, typename O>
__global__ __launch_bounds__(kNormMost) void norm_long_kernel(NormArgs a) {
  constexpr bool SPLIT = O::kBytes > 1 && Split<X, O>::value;
  __shared__ float part[2][kNormMost / 64];
  const int64_t gap = lane_gap<SPLIT>(kNormMost), first = lane_column<SPLIT>(threadIdx.x);
  const int64_t width = O::kBytes == 1 ? (a.cols + 127) / 128 * 128 : a.cols;  // blocks are filled up
  const bool residual = a.residual.p != nullptr, total = a.total.p != nullptr;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const char *x_row = row_of<X>(a.x, row), *r_row = residual ? row_of<X>(a.residual, row) : x_row;
    float sum[1] = {0.0f};
    for (int64_t col = first; col - first < width; col += 8 * kNormMost)
      cut<SPLIT>(a.cols, a.cols - col, gap, [&](auto how) {
        constexpr Cut C = decltype(how)::value;
        float t[8];
        const Raw<X> x = load_raw<X, SPLIT, C>(x_row, col, a.cols, gap), r = load_raw<X, SPLIT, C>(r_row, col, a.cols, gap);
        total_of<X, SPLIT, C>(x, r, residual, col, a.cols, gap, t);
        if (total) store_cols<X, SPLIT, C>(row_of<X>(a.total, row), col, a.cols, gap, t);
        sum[0] += squares(t);
      });
    sum_of_row(sum, kNormMost, part[turn]);
    const float scale = rsqrtf(sum[0] / (float)a.cols + a.eps);
    for (int64_t col = first; col - first < width; col += 8 * kNormMost)
      cut<SPLIT>(a.cols, a.cols - col, gap, [&](auto how) {
        constexpr Cut C = decltype(how)::value;
        float t[8];
        const Raw<X> x = load_raw<X, SPLIT, C>(total ? row_of<X>(a.total, row) : x_row, col, a.cols, gap);
        const Raw<X> r = load_raw<X, SPLIT, C>(total ? row_of<X>(a.total, row) : r_row, col, a.cols, gap);
        const RawWeight weight = load_raw<SPLIT, C>(a.weight_dtype, a.weight, col, a.cols, gap);
        total_of<X, SPLIT, C>(x, r, residual && !total, col, a.cols, gap, t);
        finish<O, SPLIT, C>(a, row, true, col, a.cols, gap, t, weight, scale);
      });
  }
}

// ---- gradients

// With r = 1 / sqrt(mean(x^2) + eps):  out = total_grad + r (g w - x r^2 mean(g w x)),  dweight = the rows' sum of g x r.
//
// Bound by memory.  A row's loads are all on their way before its sums, and, where the registers suffice (AHEAD, up to 16
// columns a lane), the next row's before this row's results; the weight stays in registers then too (KEEP).  Wider lanes load
// it twice, the second time under the sums, and the total's gradient with the rest where that fits (EARLY: 4096 x 16384 in
// 122 us, 147 with both after the sums, 175 with the next row's x and g before them).  8192 x 8192 bfloat16 with a total's
// gradient (537 MB) in 88 us with the parts' sum, 6.1 TB/s (97 without that gradient ahead), 16384 x 4096 in 95, 8192 x 2560
// in 40, 10513 x 2129 in 59; without the next row ahead float32 (1.07 GB) in 184, 5.8 TB/s, x alone float32 (671 MB) in 129, 5.2.
template <typename X, typename G, int U>
__global__ __launch_bounds__(kNormGradMost, U == 1 ? 4 : U == 2 && X::kBytes >= G::kBytes ? 3 : 2) void norm_grad_kernel(
    NormGradArgs a, int lanes, float* sums, int64_t pitch) {
  constexpr bool SPLIT = Split<X, G>::value, AHEAD = X::kBytes + G::kBytes == 4 && U <= 2, KEEP = U <= 2,
                 EARLY = KEEP || X::kBytes + G::kBytes == 4;
  __shared__ float part[2][2 * kNormGradMost / 64];
  __shared__ float joined[U == 1 ? 8 * kStripThreads : 1];
  const int side = blockDim.x / lanes;
  int cols = (int)a.cols;
  const int64_t step = (int64_t)gridDim.x * side;
  Place<SPLIT, U> at(lanes);
  const int gap = at.gap();
  // which of the rows beside each other; of lanes with several vectors a whole wave has one
  const int mine = U > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / lanes) : threadIdx.x / lanes;
  float dw[U][8];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[u][i] = 0.0f;
  auto all = [&](auto how) {
    constexpr Cut C = decltype(how)::value;
    RawWeight weight[U];
    if constexpr (KEEP) {
#pragma unroll
      for (int u = 0; u < U; ++u) weight[u] = load_raw<SPLIT, C>(a.weight_dtype, a.weight, at(u), cols, gap);
    }
    const bool more = a.total_grad.p != nullptr;
    Raw<X> x_raw[U];
    Raw<G> g_raw[U], t_raw[U];
    auto fetch = [&](int64_t base) {
      const int64_t row = min(base + mine, a.rows - 1);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        x_raw[u] = load_raw<X, SPLIT, C, true>(row_of<X>(a.x, row), at(u), cols, gap);
        g_raw[u] = load_raw<G, SPLIT, C, true>(row_of<G>(a.g, row), at(u), cols, gap);
      }
      if (EARLY && more) {
#pragma unroll
        for (int u = 0; u < U; ++u) t_raw[u] = load_raw<G, SPLIT, C, true>(row_of<G>(a.total_grad, row), at(u), cols, gap);
      }
    };
    int turn = 0;
    int64_t base = (int64_t)blockIdx.x * side;
    fetch(base);
    for (; base < a.rows; base += step, turn ^= 1) {
      // what follows from these is formed again in every turn, and not kept
      if constexpr (U > 1 && !AHEAD) asm volatile("" : "+s"(cols), "+v"(at.lane));
      const int64_t row = min(base + mine, a.rows - 1);
      const bool real = base + mine < a.rows;
      float x[U][8], g[U][8], s[2] = {0.0f, 0.0f};
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float w[8];
        widen<X, SPLIT, C>(x_raw[u], at(u), cols, gap, x[u]);
        widen<G, SPLIT, C>(g_raw[u], at(u), cols, gap, g[u]);
        if (!KEEP) weight[u] = load_raw<SPLIT, C>(a.weight_dtype, again(a.weight), at(u), cols, gap);
        widen<SPLIT, C>(a.weight_dtype, weight[u], at(u), cols, gap, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0] = fmaf(x[u][i], x[u][i], s[0]), s[1] = fmaf(g[u][i] * w[i], x[u][i], s[1]);
      }
      Raw<G> t_now[U];
#pragma unroll
      for (int u = 0; u < U; ++u) t_now[u] = t_raw[u];
      if (AHEAD && base + step < a.rows) fetch(base + step);
      if constexpr (!KEEP && EARLY) {
#pragma unroll
        for (int u = 0; u < U; ++u) weight[u] = load_raw<SPLIT, C>(a.weight_dtype, again(a.weight), at(u), cols, gap);
      }
      sum_of_row(s, lanes, part[turn]);
      const float n = (float)cols, r = rsqrtf(s[0] / n + a.eps), k = r * r * (s[1] / n);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float w[8], d[8];
        if (!EARLY) weight[u] = load_raw<SPLIT, C>(a.weight_dtype, again(a.weight), at(u), cols, gap);
        widen<SPLIT, C>(a.weight_dtype, weight[u], at(u), cols, gap, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          d[i] = r * (g[u][i] * w[i] - x[u][i] * k);
          dw[u][i] += real ? g[u][i] * (x[u][i] * r) : 0.0f;
        }
        if (more) {
          if (!EARLY) t_now[u] = load_raw<G, SPLIT, C, true>(row_of<G>(a.total_grad, row), at(u), cols, gap);
          float t[8];
          widen<G, SPLIT, C>(t_now[u], at(u), cols, gap, t);
#pragma unroll
          for (int i = 0; i < 8; ++i) d[i] += t[i];
        }
        if (real) store_cols<G, SPLIT, C>(row_of<G>(a.out, row), at(u), cols, gap, d);
      }
      if (!AHEAD && base + step < a.rows) fetch(base + step);
    }
  };
  cut<SPLIT>(cols, cols - at(U - 1), gap, all);

  // The groups' parts in order.
  if constexpr (U == 1) {
    if (side > 1) {
#pragma unroll
      for (int i = 0; i < 8; ++i) joined[i * kStripThreads + threadIdx.x] = dw[0][i];
      __syncthreads();
      if (threadIdx.x >= lanes) return;
      for (int p = 1; p < side; ++p)
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[0][i] += joined[i * kStripThreads + p * lanes + threadIdx.x];
    }
  }
  char* to = (char*)(sums + blockIdx.x * pitch);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t col = at(u);
    store8<F32, true, false, kFew>(to + col * 4, a.cols - col, gap, dw[u]);
  }
}

// Long rows: r and r^2 times the mean of g w x of every row.
template <typename X, typename G>
__global__ __launch_bounds__(kStripThreads) void norm_sums_kernel(NormGradArgs a, v2f* rows) {
  constexpr bool SPLIT = Split<X, G>::value;
  __shared__ float part[2][2 * kStripThreads / 64];
  const int64_t first = lane_column<SPLIT>(threadIdx.x), gap = lane_gap<SPLIT>(kStripThreads);
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    float s[2] = {0.0f, 0.0f};
    for (int64_t c = 0; c < a.cols; c += 8 * kStripThreads) {
      const int64_t col = first + c;
      float x[8], g[8], w[8];
      auto take = [&](auto how) {
        constexpr Cut C = decltype(how)::value;
        const Raw<X> x_raw = load_raw<X, SPLIT, C>(row_of<X>(a.x, row), col, a.cols, gap);
        const Raw<G> g_raw = load_raw<G, SPLIT, C>(row_of<G>(a.g, row), col, a.cols, gap);
        const RawWeight w_raw = load_raw<SPLIT, C>(a.weight_dtype, a.weight, col, a.cols, gap);
        widen<X, SPLIT, C>(x_raw, col, a.cols, gap, x);
        widen<G, SPLIT, C>(g_raw, col, a.cols, gap, g);
        widen<SPLIT, C>(a.weight_dtype, w_raw, col, a.cols, gap, w);
      };
      cut<SPLIT>(a.cols, a.cols - col, gap, take);
      float e[2] = {0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < 8; ++i) e[0] = fmaf(x[i], x[i], e[0]), e[1] = fmaf(g[i] * w[i], x[i], e[1]);
      s[0] += e[0], s[1] += e[1];
    }
    sum_of_row(s, kStripThreads, part[turn]);
    const float n = (float)a.cols, r = rsqrtf(s[0] / n + a.eps);
    if (threadIdx.x == 0) rows[row] = v2f{r, r * r * (s[1] / n)};
  }
}

// Then a strip of columns a workgroup, every gridDim.y-th row.  Both: 2048 x 20000 bfloat16 with a total's gradient in 95 to
// 100 us (328 MB, and g and x once more).
template <typename X, typename G>
__global__ __launch_bounds__(kStripThreads) void norm_strip_kernel(NormGradArgs a, const v2f* rows, float* sums, int64_t pitch) {
  constexpr bool SPLIT = Split<X, G>::value;
  const int64_t c0 = (int64_t)blockIdx.x * 8 * kStripThreads, col = c0 + lane_column<SPLIT>(threadIdx.x);
  const int64_t gap = lane_gap<SPLIT>(kStripThreads);
  float w[8], dw[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  auto all = [&](auto how) {
    constexpr Cut C = decltype(how)::value;
    widen<SPLIT, C>(a.weight_dtype, load_raw<SPLIT, C>(a.weight_dtype, a.weight, col, a.cols, gap), col, a.cols, gap, w);
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
      float x[8], g[8], d[8];
      const Raw<X> x_raw = load_raw<X, SPLIT, C>(row_of<X>(a.x, row), col, a.cols, gap);
      const Raw<G> g_raw = load_raw<G, SPLIT, C>(row_of<G>(a.g, row), col, a.cols, gap);
      widen<X, SPLIT, C>(x_raw, col, a.cols, gap, x);
      widen<G, SPLIT, C>(g_raw, col, a.cols, gap, g);
      const v2f rk = rows[row];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        d[i] = rk[0] * (g[i] * w[i] - x[i] * rk[1]);
        dw[i] += g[i] * (x[i] * rk[0]);
      }
      if (a.total_grad.p) {
        float t[8];
        widen<G, SPLIT, C>(load_raw<G, SPLIT, C>(row_of<G>(a.total_grad, row), col, a.cols, gap), col, a.cols, gap, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] += t[i];
      }
      store_cols<G, SPLIT, C>(row_of<G>(a.out, row), col, a.cols, gap, d);
    }
  };
  cut<SPLIT>(a.cols, a.cols - col, gap, all);
  store8<F32, true, false, kFew>((char*)(sums + blockIdx.y * pitch + col), a.cols - col, gap, dw);
}

// The sum of `parts` rows of float32: LANES lanes of a workgroup take 4 columns each, and each of its 256 / LANES such groups a
// share of the rows in order; the groups' sums are added in pairs, then by waves.
template <int LANES>
__global__ __launch_bounds__(256) void norm_join_kernel(const float* sums, int64_t parts, int64_t pitch, int64_t cols, float* out) {
  __shared__ v4f joined[4][LANES];
  constexpr int GROUPS = 256 / LANES;
  const int64_t c = ((int64_t)blockIdx.x * LANES + threadIdx.x % LANES) * 4, each = (parts + GROUPS - 1) / GROUPS;
  const int64_t begin = threadIdx.x / LANES * each, end = min(begin + each, parts);
  v4f v = {0, 0, 0, 0};
  if (c < pitch) {
#pragma unroll 8
    for (int64_t p = begin; p < end; ++p) v += ldg<v4f, false>((const char*)(sums + p * pitch + c));
  }
#pragma unroll
  for (int s = LANES; s < 64; s *= 2)
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += __shfl_xor(v[i], s);
  if (threadIdx.x % 64 < LANES) joined[threadIdx.x / 64][threadIdx.x % 64] = v;
  __syncthreads();
  if (threadIdx.x >= LANES) return;
  for (int w = 1; w < 4; ++w) v += joined[w][threadIdx.x];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (c + i < cols) out[c + i] = v[i];
}

__global__ __launch_bounds__(256) void norm_zero_kernel(float* out, int64_t cols) {
  for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < cols; c += (int64_t)gridDim.x * 256) out[c] = 0.0f;
}

template <typename X, typename O>
hipError_t run_norm(const NormArgs& a, hipStream_t stream) {
  const NormPlan p = norm_plan(a.rows, a.cols, O::kBytes == 1);
  if (p.vectors)
    hipLaunchKernelGGL((p.vectors == 1 ? norm_kernel<X, O, 1> : norm_kernel<X, O, 2>), dim3((unsigned)p.wgs), dim3(p.threads), 0, stream, a,
                       p.lanes);
  else
    hipLaunchKernelGGL((norm_long_kernel<X, O>), dim3((unsigned)p.wgs), dim3(kNormMost), 0, stream, a);
  return hipGetLastError();
}

template <typename X, typename G>
hipError_t run_norm_grad(const NormGradArgs& a, void* workspace, hipStream_t stream) {
  const NormGradPlan p = norm_grad_plan(a.rows, a.cols);
  float* parts = (float*)workspace;
  if (p.vectors) {
    const auto kernel = p.vectors == 1   ? norm_grad_kernel<X, G, 1>
                        : p.vectors == 2 ? norm_grad_kernel<X, G, 2>
                                         : norm_grad_kernel<X, G, 4>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)p.wgs), dim3(p.threads), 0, stream, a, p.lanes, p.wgs > 1 ? parts : a.dweight,
                       p.pitch);
  } else {
    v2f* rows = (v2f*)(parts + norm_grad_space(p, a.rows).rows_at);
    hipLaunchKernelGGL((norm_sums_kernel<X, G>), dim3((unsigned)std::min<int64_t>(a.rows, 1 << 20)), dim3(kStripThreads), 0, stream,
                       a, rows);
    hipLaunchKernelGGL((norm_strip_kernel<X, G>), dim3((unsigned)p.strips, (unsigned)p.wgs), dim3(kStripThreads), 0, stream, a, rows,
                       p.wgs > 1 ? parts : a.dweight, p.pitch);
  }
  if (p.wgs > 1) {
    // few columns in narrow workgroups, for more of them (us with 4 and 16 lanes: 3.7 and 4.6 for 501 x 1333, 7.0 and 4.9 for
    // 512 x 8192)
    const bool wide = a.cols >= 4096;
    hipLaunchKernelGGL(wide ? norm_join_kernel<16> : norm_join_kernel<4>, dim3((unsigned)ceil_div(a.cols, wide ? 64 : 16)), dim3(256), 0,
                       stream, parts, p.wgs, p.pitch, a.cols, a.dweight);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rms_norm(const NormArgs& a, hipStream_t stream) {
  const bool blocks = a.blocks.codes != nullptr, f32 = a.out_dtype == Elem::f32;
  if (a.dtype == Elem::f32)
    return blocks ? run_norm<F32, Q8>(a, stream) : f32 ? run_norm<F32, F32>(a, stream) : run_norm<F32, B16>(a, stream);
  return blocks ? run_norm<B16, Q8>(a, stream) : f32 ? run_norm<B16, F32>(a, stream) : run_norm<B16, B16>(a, stream);
}

size_t rms_norm_grad_workspace(int64_t rows, int64_t cols) { return norm_grad_space(norm_grad_plan(rows, cols), rows).bytes; }

hipError_t launch_rms_norm_grad(const NormGradArgs& a, void* workspace, hipStream_t stream) {
  if (a.rows == 0) {
    hipLaunchKernelGGL(norm_zero_kernel, dim3((unsigned)std::min<size_t>(ceil_div(a.cols, 256), 4096)), dim3(256), 0, stream,
                       a.dweight, a.cols);
    return hipGetLastError();
  }
  if (a.x_dtype == Elem::f32)
    return a.dtype == Elem::f32 ? run_norm_grad<F32, F32>(a, workspace, stream) : run_norm_grad<F32, B16>(a, workspace, stream);
  return a.dtype == Elem::f32 ? run_norm_grad<B16, F32>(a, workspace, stream) : run_norm_grad<B16, B16>(a, workspace, stream);
}

}  // namespace pat
