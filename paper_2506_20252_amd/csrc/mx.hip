// 4-bit block floating point: quantise and widen.
#include "ops_device.hpp"

namespace pat {
namespace {

// A lane takes 8 values at a time, 4 lanes a block, 16 lanes a group of 128; the stored form of groups that follow
// each other, also from row to row, is consecutive, so codes and scales leave as whole words in order.  A workgroup
// takes 16 groups side by side and kGroups of those in turn, all read before any is written.
//
// Bound by memory: 8192 x 8192 bfloat16 (170 MB) in 27 us, 6.3 TB/s, by nontemporal loads (29 otherwise, and
// 8192 x 8192 x 8192 with it took 12 longer); 1001 x 1000 float32 (4.5 MB) in 3.4 us, of which 3 are a launch of anything.
constexpr int kGroups = 4;

template <typename T>
__global__ __launch_bounds__(256) void quantize_kernel(Mat x, uint32_t total, int64_t cols, Divisor groups, uint8_t* codes,
                                                       uint8_t* scales) {
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
        const uint32_t s = mx_scale_byte(max_of_4(high_bits(r[u])));
        const uint32_t word = mx_codes(r[u], s), four = or_of_16_by_4(s << (sub / 4 * 8));
        if (g >= total) continue;
        stg<false>((char*)codes + (int64_t)g * 64 + sub * 4, word);
        if (sub == 0) stg<false>((char*)scales + (int64_t)g * 4, four);
      }
    };
    if (cols % 8 == 0) take(CoverOf<kWhole>{});  // a lane's 8 columns exist or do not
    else if (cols >= 8) take(CoverOf<kEnd>{});
    else take(CoverOf<kFew>{});
  }
}

// A lane takes VALUES columns at a time (8 bfloat16 or 4 float32: 16 bytes), 128 / VALUES lanes a group: stores are whole
// vectors of consecutive lanes.  Bound by memory: 8192 x 8192 to bfloat16 in 25 us, 6.8 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void dequantize_kernel(MxMat q, uint32_t total, int64_t cols, Divisor groups, MatOut out) {
  constexpr int VALUES = 16 / T::kBytes, LANES = 128 / VALUES, SIDE = 256 / LANES;
  const uint32_t sub = threadIdx.x % LANES;
  for (uint32_t base = blockIdx.x * (SIDE * kGroups); base < total; base += gridDim.x * (SIDE * kGroups)) {
    uint32_t code[kGroups], four[kGroups];
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
      const int64_t g = min(base + u * SIDE + threadIdx.x / LANES, total - 1);
      const char* p = (const char*)q.codes + g * 64 + sub * (VALUES / 2);
      code[u] = VALUES == 8 ? ldg<uint32_t, false>(p) : ldg<uint16_t, false>(p);
      four[u] = ldg<uint32_t, false>((const char*)q.scales + g * 4);
    }
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
      const uint32_t g = base + u * SIDE + threadIdx.x / LANES, row = groups.divide(min(g, total - 1));
      const int64_t c = (int64_t)(g - row * groups.d) * 128 + sub * VALUES, left = cols - c;
      if (g >= total || left <= 0) continue;
      const uint32_t s = four[u] >> (sub * VALUES / 32 * 8) & 255u;
      const float scale = mx_scale_operand(s);
      v4u v;
      if constexpr (VALUES == 8) {
        v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[u], scale, 0));
        v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[u], scale, 1));
        v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[u], scale, 2));
        v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[u], scale, 3));
      } else {
        const v2f a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[u], scale, 0);
        const v2f b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[u], scale, 1);
        v = __builtin_bit_cast(v4u, v4f{a[0], a[1], b[0], b[1]});
      }
      char* p = (char*)out.p + ((int64_t)row * out.stride + c) * T::kBytes;
      if (left >= VALUES) {
        stg<true, T::kBytes>(p, v);
      } else {
#pragma unroll
        for (int i = 0; i < VALUES; ++i) {
          if (i >= left) break;
          if constexpr (VALUES == 8) stg<false>(p + 2 * i, (uint16_t)(v[i / 2] >> (16 * (i & 1))));
          else stg<false>(p + 4 * i, (uint32_t)v[i]);
        }
      }
    }
  }
}

unsigned grid_for(int64_t groups, int per_workgroup) {
  const size_t wgs = ceil_div((size_t)groups, per_workgroup);
  return (unsigned)(wgs < (1 << 20) ? wgs : 1 << 20);
}

}  // namespace

hipError_t launch_mx_quantize(Mat x, Elem dtype, int64_t rows, int64_t cols, uint8_t* codes, uint8_t* scales,
                              hipStream_t stream) {
  const int64_t groups = groups_of(cols), total = rows * groups;
  const auto kernel = dtype == Elem::f32 ? quantize_kernel<F32> : quantize_kernel<B16>;
  hipLaunchKernelGGL(kernel, dim3(grid_for(total, 16 * kGroups)), dim3(256), 0, stream, x, (uint32_t)total, cols,
                     Divisor((uint32_t)groups), codes, scales);
  return hipGetLastError();
}

hipError_t launch_mx_dequantize(MxMat q, int64_t rows, int64_t cols, MatOut out, Elem dtype, hipStream_t stream) {
  const int64_t groups = groups_of(cols), total = rows * groups;
  const auto kernel = dtype == Elem::f32 ? dequantize_kernel<F32> : dequantize_kernel<B16>;
  const int side = dtype == Elem::f32 ? 8 : 16;
  hipLaunchKernelGGL(kernel, dim3(grid_for(total, side * kGroups)), dim3(256), 0, stream, q, (uint32_t)total, cols,
                     Divisor((uint32_t)groups), out);
  return hipGetLastError();
}

}  // namespace pat
