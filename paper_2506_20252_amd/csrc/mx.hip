// 4-bit block floating point: quantise and widen.
#include "ops_device.hpp"

namespace pat {
namespace {

// One lane per block of 32 values.
template <typename T>
__global__ __launch_bounds__(256) void quantize_kernel(Mat x, int64_t rows, int64_t cols, uint8_t* codes,
                                                       uint8_t* scales) {
  const int64_t blocks = (cols + 127) / 128 * 4;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * blocks; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / blocks, c = i % blocks * 32;
    float v[32];
    uint32_t high = 0;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      v[j] = c + j < cols ? T::load((const char*)x.p, r * x.stride + c + j) : 0.0f;
      high = max(high, __float_as_uint(v[j]) & 0x7FFFFFFFu);
    }
    const uint32_t s = mx_scale_byte(high);
    const v4u q = mx_codes(v, s);
    stg<false>((char*)codes + i * 16, q);
    stg<false>((char*)scales + i, (uint8_t)s);
  }
}

// The two values of a byte of codes, exact in float32.
__device__ __forceinline__ v2f mx_pair(uint32_t byte, uint32_t s) {
  v2f f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(byte, mx_scale_value(s == 255u ? 0u : s), 0);
  if (s == 255u) f = v2f{__uint_as_float(0x7FC00000u), __uint_as_float(0x7FC00000u)};
  return f;
}

// One lane per byte of codes that stands for columns.
template <typename T>
__global__ __launch_bounds__(256) void dequantize_kernel(MxMat q, int64_t rows, int64_t cols, MatOut out) {
  const int64_t pairs = (cols + 1) / 2, pitch = (cols + 127) / 128 * 64;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * pairs; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / pairs, b = i % pairs;
    const v2f f = mx_pair(q.codes[r * pitch + b], q.scales[r * (pitch / 16) + b / 16]);
    T::store((char*)out.p, r * out.stride + 2 * b, f[0]);
    if (2 * b + 1 < cols) T::store((char*)out.p, r * out.stride + 2 * b + 1, f[1]);
  }
}

unsigned grid_for(int64_t items) {
  const size_t wgs = ceil_div((size_t)items, 256);
  return (unsigned)(wgs < (1 << 20) ? wgs : 1 << 20);
}

}  // namespace

hipError_t launch_mx_quantize(Mat x, Elem dtype, int64_t rows, int64_t cols, uint8_t* codes, uint8_t* scales,
                              hipStream_t stream) {
  const auto kernel = dtype == Elem::f32 ? quantize_kernel<F32> : quantize_kernel<B16>;
  hipLaunchKernelGGL(kernel, dim3(grid_for(rows * groups_of(cols) * 4)), dim3(256), 0, stream, x, rows, cols, codes,
                     scales);
  return hipGetLastError();
}

hipError_t launch_mx_dequantize(MxMat q, int64_t rows, int64_t cols, MatOut out, Elem dtype, hipStream_t stream) {
  const auto kernel = dtype == Elem::f32 ? dequantize_kernel<F32> : dequantize_kernel<B16>;
  hipLaunchKernelGGL(kernel, dim3(grid_for(rows * ((cols + 1) / 2))), dim3(256), 0, stream, q, rows, cols, out);
  return hipGetLastError();
}

}  // namespace pat
