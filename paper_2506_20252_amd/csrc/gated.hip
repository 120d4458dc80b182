// The gradient of the gated block's activation and product, from its 8-bit checkpoint.
#include "layer_device.hpp"

namespace pat {
namespace {

// A lane takes 8 columns of a row, 16 lanes a group of 128, as the casts do.  Bound by memory: 8192 x 8192 bfloat16 (541 MB) in
// 81 us, 6.7 TB/s, by nontemporal loads (95 with cached ones, 87 with nontemporal stores too); two groups a lane at once: 97.
// From a float32 gradient (675 MB) 105, 6.4.
template <typename G>
__global__ __launch_bounds__(256) void gated_grad_kernel(Mat g, MxbMat a, MxbMat b, uint32_t total, int64_t n, Divisor groups, Act act,
                                                         MatOut out) {
  const uint32_t sub = threadIdx.x % 16;
  for (uint32_t at = blockIdx.x * 16 + threadIdx.x / 16; at < total; at += gridDim.x * 16) {
    const uint32_t row = groups.divide(at);
    const int64_t c = (int64_t)(at - row * groups.d) * 128 + sub * 8;
    auto take = [&](auto cover) {
      constexpr Cover C = decltype(cover)::value;
      Raw8<G> r = load_raw8<G, C, true>((const char*)g.p + (int64_t)row * g.stride * G::kBytes, c, n);
      const v2u ca = ldg<v2u, true>((const char*)a.codes + (int64_t)at * 128 + sub * 8);
      const v2u cb = ldg<v2u, true>((const char*)b.codes + (int64_t)at * 128 + sub * 8);
      const uint32_t sa = ldg<uint8_t, false>((const char*)a.scales + (int64_t)at * 4 + sub / 4);
      const uint32_t sb = ldg<uint8_t, false>((const char*)b.scales + (int64_t)at * 4 + sub / 4);
      settle<C>(r, c, n);
      if (c >= n) return;
      float va[8], vb[8], da[8], db[8];
      mxb_values(ca[0], sa, va), mxb_values(ca[1], sa, va + 4);
      mxb_values(cb[0], sb, vb), mxb_values(cb[1], sb, vb + 4);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float gv;
        if constexpr (G::kBytes == 4) gv = __uint_as_float(r.w[i / 4][i % 4]);
        else gv = i & 1 ? bf16_hi(r.w[0][i / 2]) : bf16_lo(r.w[0][i / 2]);
        float slope;
        db[i] = gv * activate(act, va[i], &slope);
        da[i] = gv * vb[i] * slope;
      }
      char* p = (char*)out.p + ((int64_t)row * out.stride + c) * 2;
      if (n - c >= 8) {
        store8<B16, false, false, kWhole>(p, 8, 4, da);
        store8<B16, false, false, kWhole>(p + 2 * n, 8, 4, db);
      } else {
        store8<B16, false, false, kEnd>(p, n - c, 4, da);
        store8<B16, false, false, kEnd>(p + 2 * n, n - c, 4, db);
      }
    };
    if (n % 8 == 0) take(CoverOf<kWhole>{});
    else if (n >= 8) take(CoverOf<kEnd>{});
    else take(CoverOf<kFew>{});
  }
}

}  // namespace

hipError_t launch_gated_grad(Mat g, Elem dtype, MxbMat a, MxbMat b, int64_t m, int64_t n, Act act, MatOut out,
                             hipStream_t stream) {
  const int64_t groups = groups_of(n), total = m * groups;
  const size_t wgs = ceil_div((size_t)total, 16);
  const auto kernel = dtype == Elem::f32 ? gated_grad_kernel<F32> : gated_grad_kernel<B16>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(wgs < (1 << 20) ? wgs : 1 << 20)), dim3(256), 0, stream, g, a, b, (uint32_t)total, n,
                     Divisor((uint32_t)groups), act, out);
  return hipGetLastError();
}

}  // namespace pat
