// 8-bit blocks: quantise and widen.
#include "layer_device.hpp"

namespace pat {
namespace {

// As the 4-bit blocks': a lane takes 8 values at a time, 4 lanes a block, 16 lanes a group of 128; a workgroup takes 16
// groups side by side and kGroups of those in turn, all read before any is written.  Bound by memory: 8192 x 8192 bfloat16
// (203 MB) in 33 us, 6.1 TB/s, float32 (338 MB) in 61, 5.6.
constexpr int kGroups = 4;

template <typename T>
__global__ __launch_bounds__(256) void mxb_quantize_kernel(Mat x, uint32_t total, int64_t cols, Divisor groups, MxbOut q) {
  const uint32_t sub = threadIdx.x % 16;
  for (uint32_t base = blockIdx.x * (16 * kGroups); base < total; base += gridDim.x * (16 * kGroups)) {
    auto take = [&](auto cover) {
      constexpr Cover C = decltype(cover)::value;
      Raw8<T> r[kGroups];
#pragma unroll
      for (int u = 0; u < kGroups; ++u) {
        const uint32_t g = min(base + u * 16 + threadIdx.x / 16, total - 1), row = groups.divide(g);
        r[u] = load_raw8<T, C, true>((const char*)x.p + (int64_t)row * x.stride * T::kBytes,
                                     (int64_t)(g - row * groups.d) * 128 + sub * 8, cols);
      }
#pragma unroll
      for (int u = 0; u < kGroups; ++u) {
        const uint32_t g = base + u * 16 + threadIdx.x / 16, h = min(g, total - 1), row = groups.divide(h);
        settle<C>(r[u], (int64_t)(h - row * groups.d) * 128 + sub * 8, cols);
        const uint32_t s = mxb_scale_byte(max_of_4(high_bits(r[u])));
        const uint32_t four = or_of_16_by_4(s << (sub / 4 * 8));
        if (g >= total) continue;
        stg<false>((char*)q.codes + (int64_t)g * 128 + sub * 8, mxb_codes(r[u], s));
        if (sub == 0) stg<false>((char*)q.scales + (int64_t)g * 4, four);
      }
    };
    if (cols % 8 == 0) take(CoverOf<kWhole>{});  // a lane's 8 columns exist or do not
    else if (cols >= 8) take(CoverOf<kEnd>{});
    else take(CoverOf<kFew>{});
  }
}

// A lane takes VALUES columns at a time, 16 bytes of the output.  Through float32, which holds every value of the stored
// form; the rounding to bfloat16 shows below 2^-133 alone.  Bound by memory: 8192 x 8192 to bfloat16 (203 MB) in 30 us, 6.8 TB/s,
// to float32 (338 MB) in 48, 7.0.
template <typename T>
__global__ __launch_bounds__(256) void mxb_dequantize_kernel(MxbMat q, uint32_t total, int64_t cols, Divisor groups, MatOut out) {
  constexpr int VALUES = 16 / T::kBytes, LANES = 128 / VALUES, SIDE = 256 / LANES;
  const uint32_t sub = threadIdx.x % LANES;
  for (uint32_t base = blockIdx.x * (SIDE * kGroups); base < total; base += gridDim.x * (SIDE * kGroups)) {
    v2u code[kGroups];
    uint32_t four[kGroups];
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
      const int64_t g = min(base + u * SIDE + threadIdx.x / LANES, total - 1);
      const char* p = (const char*)q.codes + g * 128 + sub * VALUES;
      if constexpr (VALUES == 8) code[u] = ldg<v2u, false>(p);
      else code[u] = v2u{ldg<uint32_t, false>(p), 0};
      four[u] = ldg<uint32_t, false>((const char*)q.scales + g * 4);
    }
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
      const uint32_t g = base + u * SIDE + threadIdx.x / LANES, row = groups.divide(min(g, total - 1));
      const int64_t c = (int64_t)(g - row * groups.d) * 128 + sub * VALUES, left = cols - c;
      if (g >= total || left <= 0) continue;
      const uint32_t s = four[u] >> (sub * VALUES / 32 * 8) & 255u;
      float v[8];
      mxb_values(code[u][0], s, v);
      if constexpr (VALUES == 8) mxb_values(code[u][1], s, v + 4);
      char* p = (char*)out.p + ((int64_t)row * out.stride + c) * T::kBytes;
      if (left >= VALUES) {
        if constexpr (VALUES == 8) stg<true, 2>(p, v4u{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])});
        else stg<true, 4>(p, v4f{v[0], v[1], v[2], v[3]});
      } else {
#pragma unroll
        for (int i = 0; i < VALUES; ++i)
          if (i < left) T::store(p, i, v[i]);
      }
    }
  }
}

unsigned grid_for(int64_t groups, int per_workgroup) {
  const size_t wgs = ceil_div((size_t)groups, per_workgroup);
  return (unsigned)(wgs < (1 << 20) ? wgs : 1 << 20);
}

}  // namespace

hipError_t launch_mxb_quantize(Mat x, Elem dtype, int64_t rows, int64_t cols, MxbOut q, hipStream_t stream) {
  const int64_t groups = groups_of(cols), total = rows * groups;
  const auto kernel = dtype == Elem::f32 ? mxb_quantize_kernel<F32> : mxb_quantize_kernel<B16>;
  hipLaunchKernelGGL(kernel, dim3(grid_for(total, 16 * kGroups)), dim3(256), 0, stream, x, (uint32_t)total, cols,
                     Divisor((uint32_t)groups), q);
  return hipGetLastError();
}

hipError_t launch_mxb_dequantize(MxbMat q, int64_t rows, int64_t cols, MatOut out, Elem dtype, hipStream_t stream) {
  const int64_t groups = groups_of(cols), total = rows * groups;
  const auto kernel = dtype == Elem::f32 ? mxb_dequantize_kernel<F32> : mxb_dequantize_kernel<B16>;
  const int side = dtype == Elem::f32 ? 8 : 16;
  hipLaunchKernelGGL(kernel, dim3(grid_for(total, side * kGroups)), dim3(256), 0, stream, q, (uint32_t)total, cols,
                     Divisor((uint32_t)groups), out);
  return hipGetLastError();
}

}  // namespace pat
