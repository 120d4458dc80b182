// 4-bit block floating point: quantise, widen, and the product of two stored forms.
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
    v4u q = {0, 0, 0, 0};
    if (s != 255u) {
      const float scale = mx_scale_value(s);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t word = 0;
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[8 * w], v[8 * w + 1], scale, 0);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[8 * w + 2], v[8 * w + 3], scale, 1);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[8 * w + 4], v[8 * w + 5], scale, 2);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[8 * w + 6], v[8 * w + 7], scale, 3);
        q[w] = word;
      }
    }
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

// One wave per 16 x 16 tile of the output.  A matrix instruction takes a group of 128 values of 16 rows on either
// side: lane l holds block l / 16 of row l % 16 and the block's scale, and gets output rows 4 * (l / 16) ... + 3 of
// column l % 16.  Lanes of rows beyond the matrix hold the last row; what they give is not stored.
template <typename T>
__global__ __launch_bounds__(64) void matmul_kernel(MxMat a, MxMat b, int64_t m, int64_t n, int64_t groups, MatOut out) {
  const int64_t tiles_n = (n + 15) / 16, i0 = blockIdx.x / tiles_n * 16, j0 = blockIdx.x % tiles_n * 16;
  const int lane = threadIdx.x, block = lane / 16;
  const int64_t i = min(i0 + lane % 16, m - 1), j = min(j0 + lane % 16, n - 1);
  v4f sum = {0, 0, 0, 0};
  for (int64_t g = 0; g < groups; ++g) {
    const v4i ca = ldg<v4i, false>((const char*)a.codes + (i * groups + g) * 64 + block * 16);
    const v4i cb = ldg<v4i, false>((const char*)b.codes + (j * groups + g) * 64 + block * 16);
    const int sa = a.scales[(i * groups + g) * 4 + block], sb = b.scales[(j * groups + g) * 4 + block];
    const v8i fa = {ca[0], ca[1], ca[2], ca[3], 0, 0, 0, 0}, fb = {cb[0], cb[1], cb[2], cb[3], 0, 0, 0, 0};
    sum = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa, fb, sum, 4, 4, 0, sa, 0, sb);
  }
  if (j0 + lane % 16 >= n) return;
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (i0 + 4 * block + r < m) T::store((char*)out.p, (i0 + 4 * block + r) * out.stride + j, sum[r]);
}

unsigned grid_for(int64_t items) {
  const size_t wgs = ceil_div((size_t)items, 256);
  return (unsigned)(wgs < (1 << 20) ? wgs : 1 << 20);
}

int64_t groups_of(int64_t cols) { return (cols + 127) / 128; }

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

size_t mx_matmul_workspace(int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_mx_matmul(MxMat a, MxMat b, int64_t m, int64_t n, int64_t k, MatOut out, Elem dtype, void*,
                            hipStream_t stream) {
  const auto kernel = dtype == Elem::f32 ? matmul_kernel<F32> : matmul_kernel<B16>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(ceil_div(m, 16) * ceil_div(n, 16))), dim3(64), 0, stream, a, b, m, n,
                     groups_of(k), out);
  return hipGetLastError();
}

// Workspace of a linear: the quantised rows, codes before scales.
size_t mx_linear_workspace(int64_t m, int64_t, int64_t k) { return (size_t)(m * groups_of(k)) * 68; }

hipError_t launch_mx_linear(Mat x, Elem x_dtype, MxMat w, int64_t m, int64_t n, int64_t k, MatOut out, Elem dtype,
                            void* workspace, hipStream_t stream) {
  uint8_t* codes = (uint8_t*)workspace;
  uint8_t* scales = codes + m * groups_of(k) * 64;
  if (k > 0) {
    const hipError_t e = launch_mx_quantize(x, x_dtype, m, k, codes, scales, stream);
    if (e != hipSuccess) return e;
  }
  return launch_mx_matmul({codes, scales}, w, m, n, k, out, dtype, nullptr, stream);
}

}  // namespace pat
