// Products of a bfloat16 gradient with a 4-bit matrix: both gradients of the 4-bit product.
#include "ops_device.hpp"

namespace pat {
namespace {

// One wave per 16 x 16 tile of out[i][c] = sum over j of g[i][j] q[j][c].  A matrix instruction takes 32 values of j:
// lane l holds j = 8 * (l / 16) ... + 7 of row l % 16 of g and of column l % 16 of q, and gets output rows
// 4 * (l / 16) ... + 3 of column l % 16.  Values of q are widened one by one; they are exact in bfloat16.
template <bool TRANSPOSED, typename T>
__global__ __launch_bounds__(64) void grad_kernel(Mat g, MxMat q, int64_t rows, int64_t inner, int64_t cols, MatOut out) {
  const int64_t pitch = (cols + 127) / 128 * 64;
  const int64_t tiles_c = (cols + 15) / 16, i0 = blockIdx.x / tiles_c * 16, c0 = blockIdx.x % tiles_c * 16;
  const int lane = threadIdx.x, part = lane / 16;
  const int64_t i = min(i0 + lane % 16, rows - 1), c = min(c0 + lane % 16, cols - 1);
  v4f sum = {0, 0, 0, 0};
  for (int64_t j0 = 0; j0 < inner; j0 += 32) {
    uint32_t fg[4], fq[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) fg[w] = fq[w] = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int64_t j = j0 + 8 * part + e;
      if (j >= inner) continue;
      const int64_t at = TRANSPOSED ? j * g.stride + i : i * g.stride + j;
      fg[e / 2] |= (uint32_t)ldg<uint16_t, false>((const char*)g.p + 2 * at) << (16 * (e & 1));
      const uint32_t code = q.codes[j * pitch + c / 2] >> (4 * (c & 1)) & 15u, s = q.scales[j * (pitch / 16) + c / 32];
      const float v = s == 255u ? __uint_as_float(0x7FC00000u)
                                : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, mx_scale_value(s), 0)[0];
      fq[e / 2] |= (__float_as_uint(v) >> 16) << (16 * (e & 1));
    }
    const v4u wg = {fg[0], fg[1], fg[2], fg[3]}, wq = {fq[0], fq[1], fq[2], fq[3]};
    sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, wg), __builtin_bit_cast(v8bf, wq), sum, 0, 0,
                                                  0);
  }
  if (c0 + lane % 16 >= cols) return;
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (i0 + 4 * part + r < rows) T::store((char*)out.p, (i0 + 4 * part + r) * out.stride + c, sum[r]);
}

template <bool TRANSPOSED>
auto grad_of(Elem dtype) {
  return dtype == Elem::f32 ? grad_kernel<TRANSPOSED, F32> : grad_kernel<TRANSPOSED, B16>;
}

}  // namespace

size_t mx_grad_workspace(int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_mx_grad(Mat g, bool transposed, MxMat q, int64_t rows, int64_t inner, int64_t cols, MatOut out,
                          Elem dtype, void*, hipStream_t stream) {
  const auto kernel = transposed ? grad_of<true>(dtype) : grad_of<false>(dtype);
  hipLaunchKernelGGL(kernel, dim3((unsigned)(ceil_div(rows, 16) * ceil_div(cols, 16))), dim3(64), 0, stream, g, q, rows,
                     inner, cols, out);
  return hipGetLastError();
}

}  // namespace pat
