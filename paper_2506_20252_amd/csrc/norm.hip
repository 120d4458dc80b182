// Root-mean-square norm of rows, after a residual's addition, and its gradients.
#include <algorithm>

#include "layer_device.hpp"
#include "layer_shape.hpp"

namespace pat {
namespace {

// A lane's 8 columns of a row as they are in memory, as load8 takes them (the second four `gap` columns after the first, those
// behind the row's end zero once they are widened); nothing is done with what is loaded, so that a row's loads are on their
// way together.
template <typename T>
struct Raw {
  typename T::vec4 lo, hi;
};
template <typename T, bool SPLIT, Cover C, bool NT = false>
__device__ __forceinline__ Raw<T> load_raw(const void* row, int64_t col, int64_t cols, int64_t gap) {
  typedef typename T::vec4 V;
  const int64_t n = cols - col;
  const char* p = (const char*)row + col * T::kBytes;
  if constexpr (C == kWhole && !SPLIT && T::kBytes == 2) {
    const v4u a = ldg<v4u, NT, 2>(p);
    return {{a[0], a[1]}, {a[2], a[3]}};
  } else if constexpr (C == kWhole) {
    return {ldg<V, NT, T::kBytes>(p), ldg<V, NT, T::kBytes>(p + gap * T::kBytes)};
  } else if constexpr (C == kEnd) {
    return {ldg<V, NT, T::kBytes>(p + min((int64_t)0, n - 4) * T::kBytes), ldg<V, NT, T::kBytes>(p + min(gap, n - 4) * T::kBytes)};
  } else {
    float v[8];
    load8<T, SPLIT, false, kFew>(p, n, gap, v);
    return {T::narrow(v), T::narrow(v + 4)};
  }
}
template <typename T, Cover C>
__device__ __forceinline__ void widen(const Raw<T>& r, int64_t col, int64_t cols, int64_t gap, float (&v)[8]) {
  T::widen(r.lo, v);
  T::widen(r.hi, v + 4);
  if constexpr (C == kEnd) {
    const int64_t n = cols - col;
    move_down(v, max((int64_t)0, 4 - n));
    move_down(v + 4, max((int64_t)0, gap + 4 - n));
  }
}
// The same of a vector whose type is known at the launch alone.
struct RawWeight {
  v4u lo, hi;
};
template <bool SPLIT, Cover C>
__device__ __forceinline__ RawWeight load_raw(Elem e, const void* weight, int64_t col, int64_t cols, int64_t gap) {
  if (e == Elem::f32) {
    const Raw<F32> r = load_raw<F32, SPLIT, C>(weight, col, cols, gap);
    return {__builtin_bit_cast(v4u, r.lo), __builtin_bit_cast(v4u, r.hi)};
  }
  const Raw<B16> r = load_raw<B16, SPLIT, C>(weight, col, cols, gap);
  return {v4u{r.lo[0], r.lo[1], r.hi[0], r.hi[1]}, v4u{0, 0, 0, 0}};
}
template <Cover C>
__device__ __forceinline__ void widen(Elem e, const RawWeight& r, int64_t col, int64_t cols, int64_t gap, float (&v)[8]) {
  if (e == Elem::f32) widen<F32, C>({__builtin_bit_cast(v4f, r.lo), __builtin_bit_cast(v4f, r.hi)}, col, cols, gap, v);
  else widen<B16, C>({{r.lo[0], r.lo[1]}, {r.lo[2], r.lo[3]}}, col, cols, gap, v);
}
template <typename T, bool SPLIT, Cover C, bool NT = false>
__device__ __forceinline__ void store_cols(void* row, int64_t col, int64_t cols, int64_t gap, const float (&v)[8]) {
  store8<T, SPLIT, NT, C>((char*)row + col * T::kBytes, cols - col, gap, v);
}
template <typename T>
__device__ __forceinline__ const char* row_of(Mat m, int64_t r) {
  return (const char*)m.p + r * m.stride * T::kBytes;
}
template <typename T>
__device__ __forceinline__ char* row_of(MatOut m, int64_t r) {
  return (char*)m.p + r * m.stride * T::kBytes;
}

// The same in every turn of a loop, and made again there: kept over the loop, places and weights of all vectors would take
// more registers than there are.
__device__ __forceinline__ int64_t again(int lane_column) {
  asm volatile("" : "+v"(lane_column));
  return lane_column;
}
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

// U > 0: a row's values stay in registers; 0: they are read again.
template <typename X, typename O, int U>
__global__ __launch_bounds__(kNormMost) void norm_kernel(NormArgs a, int lanes) {
  constexpr bool BLOCKS = O::kBytes == 1, SPLIT = !BLOCKS && Split<X, O>::value;
  constexpr int V = U ? U : 1;
  __shared__ float part[2][kNormMost / 64];
  const int lane = threadIdx.x % lanes, side = blockDim.x / lanes;
  const int64_t groups = (a.cols + 127) / 128, gap = lane_gap<SPLIT>(lanes);
  const int64_t turns = U ? 1 : ((BLOCKS ? groups * 128 : a.cols) + 8 * lanes - 1) / (8 * lanes);
  int turn = 0;
  for (int64_t base = (int64_t)blockIdx.x * side; base < a.rows; base += (int64_t)gridDim.x * side, turn ^= 1) {
    const int64_t row = min(base + threadIdx.x / lanes, a.rows - 1);
    const bool real = base + threadIdx.x / lanes < a.rows;
    const int64_t first = again((int)lane_column<SPLIT>(lane));
    const void* weight = again(a.weight);
    auto finish = [&](int64_t col, auto cover, const float (&t)[8], const RawWeight& raw, float r) {
      constexpr Cover C = decltype(cover)::value;
      float w[8], y[8];
      widen<C>(a.weight_dtype, raw, col, a.cols, gap, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = t[i] * r * w[i];
      if constexpr (BLOCKS) {
        uint32_t high = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (C != kWhole) y[i] = col + i < a.cols ? y[i] : 0.0f;
          high = max(high, __float_as_uint(y[i]) & 0x7FFFFFFFu);
        }
        const uint32_t s = mxb_scale_byte(max_of_4(high)), sub = lane % 16;
        const uint32_t four = or_of_16_by_4(s << (sub / 4 * 8));
        if (!real || col >= groups * 128) return;
        const int64_t g = row * groups + col / 128;
        stg<false>((char*)a.blocks.codes + g * 128 + sub * 8, v2u{mxb_codes(y[0], y[1], y[2], y[3], s), mxb_codes(y[4], y[5], y[6], y[7], s)});
        if (sub == 0) stg<false>((char*)a.blocks.scales + g * 4, four);
      } else {
        if (real) store_cols<O, SPLIT, C>(row_of<O>(a.out, row), col, a.cols, gap, y);
      }
    };
    auto go = [&](auto cover) {
      constexpr Cover C = decltype(cover)::value;
      const bool residual = a.residual.p != nullptr;
      const char* x_row = row_of<X>(a.x, row);
      const char* res_row = residual ? row_of<X>(a.residual, row) : x_row;
      float t[V][8], sum[1] = {0.0f};
      RawWeight w[V];
      auto at = [&](int64_t u) { return first + u * 8 * lanes; };
      // V vectors from column `at(u)`: t, its part of the sum, the total where that is wanted
      auto take = [&](int64_t u0) {
        Raw<X> x[V], r[V];
#pragma unroll
        for (int u = 0; u < V; ++u) x[u] = load_raw<X, SPLIT, C, true>(x_row, at(u0 + u), a.cols, gap);
        if (residual) {
#pragma unroll
          for (int u = 0; u < V; ++u) r[u] = load_raw<X, SPLIT, C, true>(res_row, at(u0 + u), a.cols, gap);
        }
        if constexpr (U > 0) {
#pragma unroll
          for (int u = 0; u < V; ++u) w[u] = load_raw<SPLIT, C>(a.weight_dtype, weight, at(u), a.cols, gap);
        }
#pragma unroll
        for (int u = 0; u < V; ++u) {
          widen<X, C>(x[u], at(u0 + u), a.cols, gap, t[u]);
          if (residual) {
            float v[8];
            widen<X, C>(r[u], at(u0 + u), a.cols, gap, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) t[u][i] = round_to(X{}, t[u][i] + v[i]);
            if (a.total.p && real) store_cols<X, SPLIT, C, true>(row_of<X>(a.total, row), at(u0 + u), a.cols, gap, t[u]);
          }
          float eight = 0.0f;  // added up apart, so that long rows' sums have an eighth of the terms
#pragma unroll
          for (int i = 0; i < 8; ++i) eight = fmaf(t[u][i], t[u][i], eight);
          sum[0] += eight;
        }
      };
      if constexpr (U > 0) take(0);
      else
        for (int64_t u = 0; u < turns; ++u) take(u);
      sum_of_row(sum, lanes, part[turn]);
      const float r = rsqrtf(sum[0] / (float)a.cols + a.eps);
      if constexpr (U > 0) {
#pragma unroll
        for (int u = 0; u < V; ++u) finish(at(u), cover, t[u], w[u], r);
      } else {
        for (int64_t u = 0; u < turns; ++u) {  // again, out of the total where there is one
          const bool total = a.total.p != nullptr;
          const Raw<X> x = load_raw<X, SPLIT, C>(total ? (const char*)row_of<X>(a.total, row) : x_row, at(u), a.cols, gap);
          widen<X, C>(x, at(u), a.cols, gap, t[0]);
          if (residual && !total) {
            float v[8];
            widen<X, C>(load_raw<X, SPLIT, C>(res_row, at(u), a.cols, gap), at(u), a.cols, gap, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) t[0][i] = round_to(X{}, t[0][i] + v[i]);
          }
          finish(at(u), cover, t[0], load_raw<SPLIT, C>(a.weight_dtype, weight, at(u), a.cols, gap), r);
        }
      }
    };
    if (a.cols == (U ? U : turns) * 8 * lanes) go(CoverOf<kWhole>{});
    else if (a.cols >= 4) go(CoverOf<kEnd>{});
    else go(CoverOf<kFew>{});
  }
}

// ---- gradients

// A row's loads are all on their way before its sums, and, where the registers suffice (up to 16 columns a lane), the next
// row's before this row's results; the weight stays in registers then too.  Wider lanes load it, and the total's gradient, where
// they use them.
template <typename X, typename G, int U>
__global__ __launch_bounds__(U == 1 ? kNormThreads : kNormGradMost) void norm_grad_kernel(NormGradArgs a, int lanes, float* sums, int64_t pitch) {
  constexpr bool SPLIT = Split<X, G>::value, AHEAD = X::kBytes + G::kBytes == 4 && U <= 2, KEEP = U <= 2;
  __shared__ float part[2][2 * kNormGradMost / 64];
  __shared__ float joined[U == 1 ? 8 * kNormThreads : 1];
  const int lane = threadIdx.x % lanes, side = blockDim.x / lanes;
  const int64_t gap = lane_gap<SPLIT>(lanes), step = (int64_t)gridDim.x * side;
  float dw[U][8];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[u][i] = 0.0f;
  auto all = [&](auto cover) {
    constexpr Cover C = decltype(cover)::value;
    auto at = [&](int u) { return lane_column<SPLIT>(lane) + u * 8 * lanes; };
    RawWeight weight[U];
    if constexpr (KEEP) {
#pragma unroll
      for (int u = 0; u < U; ++u) weight[u] = load_raw<SPLIT, C>(a.weight_dtype, a.weight, at(u), a.cols, gap);
    }
    Raw<X> x_raw[U];
    Raw<G> g_raw[U];
    auto fetch = [&](int64_t base) {
      const int64_t row = min(base + threadIdx.x / lanes, a.rows - 1);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        x_raw[u] = load_raw<X, SPLIT, C, true>(row_of<X>(a.x, row), at(u), a.cols, gap);
        g_raw[u] = load_raw<G, SPLIT, C, true>(row_of<G>(a.g, row), at(u), a.cols, gap);
      }
    };
    int turn = 0;
    int64_t base = (int64_t)blockIdx.x * side;
    if (base < a.rows) fetch(base);
    for (; base < a.rows; base += step, turn ^= 1) {
      const int64_t row = min(base + threadIdx.x / lanes, a.rows - 1);
      const bool real = base + threadIdx.x / lanes < a.rows, more = a.total_grad.p != nullptr;
      Raw<G> t_raw[U];
      if (KEEP && more) {
#pragma unroll
        for (int u = 0; u < U; ++u) t_raw[u] = load_raw<G, SPLIT, C, true>(row_of<G>(a.total_grad, row), at(u), a.cols, gap);
      }
      float x[U][8], g[U][8], s[2] = {0.0f, 0.0f};
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float w[8];
        widen<X, C>(x_raw[u], at(u), a.cols, gap, x[u]);
        widen<G, C>(g_raw[u], at(u), a.cols, gap, g[u]);
        if (!KEEP) weight[u] = load_raw<SPLIT, C>(a.weight_dtype, again(a.weight), at(u), a.cols, gap);
        widen<C>(a.weight_dtype, weight[u], at(u), a.cols, gap, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0] = fmaf(x[u][i], x[u][i], s[0]), s[1] = fmaf(g[u][i] * w[i], x[u][i], s[1]);
      }
      if (AHEAD && base + step < a.rows) fetch(base + step);
      sum_of_row(s, lanes, part[turn]);
      const float n = (float)a.cols, r = rsqrtf(s[0] / n + a.eps), k = r * r * (s[1] / n);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float w[8], d[8];
        if (!KEEP) weight[u] = load_raw<SPLIT, C>(a.weight_dtype, again(a.weight), at(u), a.cols, gap);
        widen<C>(a.weight_dtype, weight[u], at(u), a.cols, gap, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          d[i] = r * (g[u][i] * w[i] - x[u][i] * k);
          dw[u][i] += real ? g[u][i] * (x[u][i] * r) : 0.0f;
        }
        if (more) {
          if (!KEEP) t_raw[u] = load_raw<G, SPLIT, C, true>(row_of<G>(a.total_grad, row), at(u), a.cols, gap);
          float t[8];
          widen<G, C>(t_raw[u], at(u), a.cols, gap, t);
#pragma unroll
          for (int i = 0; i < 8; ++i) d[i] += t[i];
        }
        if (real) store_cols<G, SPLIT, C, true>(row_of<G>(a.out, row), at(u), a.cols, gap, d);
      }
      if (!AHEAD && base + step < a.rows) fetch(base + step);
    }
  };
  if (a.cols == U * 8 * lanes) all(CoverOf<kWhole>{});
  else if (a.cols >= 4) all(CoverOf<kEnd>{});
  else all(CoverOf<kFew>{});

  // The groups' parts in order.
  if constexpr (U == 1) {
    if (side > 1) {
#pragma unroll
      for (int i = 0; i < 8; ++i) joined[i * kNormThreads + threadIdx.x] = dw[0][i];
      __syncthreads();
      if (threadIdx.x >= lanes) return;
      for (int p = 1; p < side; ++p)
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[0][i] += joined[i * kNormThreads + p * lanes + threadIdx.x];
    }
  }
  char* to = (char*)(sums + blockIdx.x * pitch);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t col = lane_column<SPLIT>(lane) + u * 8 * lanes;
    store8<F32, true, false, kFew>(to + col * 4, a.cols - col, gap, dw[u]);
  }
}

// Long rows: r and r^2 times the mean of g w x of every row.
template <typename X, typename G>
__global__ __launch_bounds__(kNormThreads) void norm_sums_kernel(NormGradArgs a, v2f* rows) {
  constexpr bool SPLIT = Split<X, G>::value;
  __shared__ float part[2][2 * kNormThreads / 64];
  const int64_t first = lane_column<SPLIT>(threadIdx.x), gap = lane_gap<SPLIT>(kNormThreads);
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    float s[2] = {0.0f, 0.0f};
    for (int64_t c = 0; c < a.cols; c += 8 * kNormThreads) {
      const int64_t col = first + c;
      float x[8], g[8], w[8];
      auto take = [&](auto cover) {
        constexpr Cover C = decltype(cover)::value;
        const Raw<X> x_raw = load_raw<X, SPLIT, C>(row_of<X>(a.x, row), col, a.cols, gap);
        const Raw<G> g_raw = load_raw<G, SPLIT, C>(row_of<G>(a.g, row), col, a.cols, gap);
        const RawWeight w_raw = load_raw<SPLIT, C>(a.weight_dtype, a.weight, col, a.cols, gap);
        widen<X, C>(x_raw, col, a.cols, gap, x);
        widen<G, C>(g_raw, col, a.cols, gap, g);
        widen<C>(a.weight_dtype, w_raw, col, a.cols, gap, w);
      };
      if (c + 8 * kNormThreads <= a.cols) take(CoverOf<kWhole>{});
      else take(CoverOf<kEnd>{});
      float e[2] = {0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < 8; ++i) e[0] = fmaf(x[i], x[i], e[0]), e[1] = fmaf(g[i] * w[i], x[i], e[1]);
      s[0] += e[0], s[1] += e[1];
    }
    sum_of_row(s, kNormThreads, part[turn]);
    const float n = (float)a.cols, r = rsqrtf(s[0] / n + a.eps);
    if (threadIdx.x == 0) rows[row] = v2f{r, r * r * (s[1] / n)};
  }
}

// Then a strip of columns a workgroup, every gridDim.y-th row.
template <typename X, typename G>
__global__ __launch_bounds__(kNormThreads) void norm_strip_kernel(NormGradArgs a, const v2f* rows, float* sums, int64_t pitch) {
  constexpr bool SPLIT = Split<X, G>::value;
  const int64_t c0 = (int64_t)blockIdx.x * 8 * kNormThreads, col = c0 + lane_column<SPLIT>(threadIdx.x);
  const int64_t gap = lane_gap<SPLIT>(kNormThreads);
  float w[8], dw[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  auto all = [&](auto cover) {
    constexpr Cover C = decltype(cover)::value;
    widen<C>(a.weight_dtype, load_raw<SPLIT, C>(a.weight_dtype, a.weight, col, a.cols, gap), col, a.cols, gap, w);
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
      float x[8], g[8], d[8];
      const Raw<X> x_raw = load_raw<X, SPLIT, C>(row_of<X>(a.x, row), col, a.cols, gap);
      const Raw<G> g_raw = load_raw<G, SPLIT, C>(row_of<G>(a.g, row), col, a.cols, gap);
      widen<X, C>(x_raw, col, a.cols, gap, x);
      widen<G, C>(g_raw, col, a.cols, gap, g);
      const v2f rk = rows[row];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        d[i] = rk[0] * (g[i] * w[i] - x[i] * rk[1]);
        dw[i] += g[i] * (x[i] * rk[0]);
      }
      if (a.total_grad.p) {
        float t[8];
        widen<G, C>(load_raw<G, SPLIT, C>(row_of<G>(a.total_grad, row), col, a.cols, gap), col, a.cols, gap, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] += t[i];
      }
      store_cols<G, SPLIT, C>(row_of<G>(a.out, row), col, a.cols, gap, d);
    }
  };
  if (c0 + 8 * kNormThreads <= a.cols) all(CoverOf<kWhole>{});
  else all(CoverOf<kEnd>{});
  store8<F32, true, false, kFew>((char*)(sums + blockIdx.y * pitch + col), a.cols - col, gap, dw);
}

// The sum of `parts` rows of float32, in order: 16 groups of lanes take a share of the rows each, 4 columns a lane.
__global__ __launch_bounds__(256) void norm_join_kernel(const float* sums, int64_t parts, int64_t pitch, int64_t cols, float* out) {
  __shared__ v4f joined[256];
  const int64_t c = (int64_t)blockIdx.x * 64 + threadIdx.x % 16 * 4, each = (parts + 15) / 16;
  const int64_t begin = threadIdx.x / 16 * each, end = min(begin + each, parts);
  v4f v = {0, 0, 0, 0};
  if (c < pitch) {
#pragma unroll 8
    for (int64_t p = begin; p < end; ++p) v += ldg<v4f, false>((const char*)(sums + p * pitch + c));
  }
  joined[threadIdx.x] = v;
  __syncthreads();
  if (threadIdx.x >= 16) return;
  for (int p = 1; p < 16; ++p) v += joined[16 * p + threadIdx.x];
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
  const auto kernel = p.vectors == 1 ? norm_kernel<X, O, 1> : p.vectors == 2 ? norm_kernel<X, O, 2> : norm_kernel<X, O, 0>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)p.wgs), dim3(std::max(kNormThreads, p.lanes)), 0, stream, a, p.lanes);
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
    hipLaunchKernelGGL(kernel, dim3((unsigned)p.wgs), dim3(std::max(kNormThreads, p.lanes)), 0, stream, a, p.lanes, p.wgs > 1 ? parts : a.dweight,
                       p.pitch);
  } else {
    v2f* rows = (v2f*)(parts + p.wgs * p.pitch);
    hipLaunchKernelGGL((norm_sums_kernel<X, G>), dim3((unsigned)std::min<int64_t>(a.rows, 1 << 20)), dim3(kNormThreads), 0, stream,
                       a, rows);
    hipLaunchKernelGGL((norm_strip_kernel<X, G>), dim3((unsigned)p.strips, (unsigned)p.wgs), dim3(kNormThreads), 0, stream, a, rows,
                       p.wgs > 1 ? parts : a.dweight, p.pitch);
  }
  if (p.wgs > 1)
    hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)ceil_div(a.cols, 64)), dim3(256), 0, stream, parts, p.wgs, p.pitch, a.cols,
                       a.dweight);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rms_norm(const NormArgs& a, hipStream_t stream) {
  const bool blocks = a.blocks.codes != nullptr, f32 = a.out_dtype == Elem::f32;
  if (a.dtype == Elem::f32)
    return blocks ? run_norm<F32, Q8>(a, stream) : f32 ? run_norm<F32, F32>(a, stream) : run_norm<F32, B16>(a, stream);
  return blocks ? run_norm<B16, Q8>(a, stream) : f32 ? run_norm<B16, F32>(a, stream) : run_norm<B16, B16>(a, stream);
}

// The parts' sums, then two floats a row where rows are long.
size_t rms_norm_grad_workspace(int64_t rows, int64_t cols) {
  const NormGradPlan p = norm_grad_plan(rows, cols);
  if (p.vectors) return p.wgs > 1 ? (size_t)(p.wgs * p.pitch) * 4 : 0;
  return (size_t)(p.wgs * p.pitch) * 4 + (size_t)rows * 8;
}

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
