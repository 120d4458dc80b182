// Dropout from a counter-based generator; the mask is never stored.
#include "ops_device.hpp"

namespace pat {
namespace {

// Philox4x32-10 of counter (block, 0) under a 64-bit key.
__device__ __forceinline__ v4u philox(uint64_t block, uint64_t key) {
  uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = 0, c3 = 0;
  uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)b;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return v4u{c0, c1, c2, c3};
}

// One lane per element, a grid row of workgroups per matrix row (in turn).
template <typename T>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a) {
  const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= a.cols) return;
  for (int64_t r = blockIdx.y; r < a.rows; r += gridDim.y) {
    const uint64_t i = a.index + (uint64_t)r * a.index_stride + (uint64_t)c;
    const v4u w = philox(i >> 3, a.seed);
    const uint32_t u = w[(i >> 1) & 3] >> (16 * (i & 1)) & 0xFFFFu;
    float y = u >= a.drop ? T::load((const char*)a.x.p, r * a.x.stride + c) * a.scale : 0.0f;
    if (a.residual.p) y += T::load((const char*)a.residual.p, r * a.residual.stride + c);
    T::store((char*)a.out.p, r * a.out.stride + c, y);
  }
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, Elem dtype, hipStream_t stream) {
  const dim3 grid((unsigned)ceil_div(a.cols, 256), (unsigned)(a.rows < 65535 ? a.rows : 65535));
  if (dtype == Elem::f32) hipLaunchKernelGGL(dropout_kernel<F32>, grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL(dropout_kernel<B16>, grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace pat
