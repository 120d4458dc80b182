// Products of 8-bit activations with 4-bit weights, x w^T, on the scaled matrix instructions, and what follows them: a
// residual's addition, or the gated block's activation and product.
//
// A matrix instruction multiplies codes as they are stored and applies both blocks' scales.  Its first operand is the
// weight, its second the activations: a lane's results are then 4 consecutive columns of the output of one token.
#include <algorithm>

#include "layer_device.hpp"
#include "layer_shape.hpp"

namespace pat {
namespace {

template <int I>
struct Int {
  static constexpr int value = I;
};

// 4 and 8 bits a value: 32 values of a row.
__device__ __forceinline__ v8i frag(v4i c) { return v8i{c[0], c[1], c[2], c[3], 0, 0, 0, 0}; }
__device__ __forceinline__ v8i frag(v4i lo, v4i hi) { return v8i{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}; }

// Largest magnitude of four values, as float32 bits.
__device__ __forceinline__ uint32_t high_bits(const v4f& v) {
  uint32_t h = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) h = max(h, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  return h;
}
__device__ __forceinline__ uint32_t max_of_8(uint32_t v) {
  v = max_of_4(v);
  return max(v, dpp<0x141>(v));  // the other four of eight, mirrored
}

// Four columns at p of which `left` are there.
template <typename T>
__device__ __forceinline__ v4f load4(const char* p, int64_t left) {
  float v[4] = {0, 0, 0, 0};
  if (left >= 4) T::widen(ldg<typename T::vec4, false, T::kBytes>(p), v);
  else
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < left ? T::load(p, i) : 0.0f;
  return v4f{v[0], v[1], v[2], v[3]};
}
template <typename T>
__device__ __forceinline__ void store4(char* p, int64_t left, const v4f& f) {
  const float v[4] = {f[0], f[1], f[2], f[3]};
  if (left >= 4) stg<false, T::kBytes>(p, T::narrow(v));
  else
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) T::store(p, i, v[i]);
}

// ---- few tokens ----------------------------------------------------------------------------------------------
//
// A workgroup computes 16 * MT tokens by 16 * H columns (gated: 16 * 2 H rows of the weight); its waves take 512 terms (four
// groups) in turn.  An instruction of 16 x 16 x 128 takes four blocks of 16 rows: lane l has row l mod 16 of either
// side, of the weight all of block l / 16, of the activations 16 values of block l / 32 and 16 of block 2 + l / 32.  The j-th
// instruction takes the j-th block of each of the four groups, so that a lane's four loads of the weight are 64 bytes in a
// row; both sides' scales are those of block l / 16, a byte of one word.
constexpr int kFewWaves = 8;

template <int MT, int H, bool GATED, typename O>
__global__ __launch_bounds__(64 * kFewWaves) void few_kernel(MxbMat x, MxMat w, int64_t m, int64_t n, int groups, int64_t tiles_n,
                                                             Epilogue e) {
  constexpr int NT = GATED ? 2 * H : H;
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, quarter = lane / 16;
  const int64_t i0 = blockIdx.x / tiles_n * (16 * MT), j0 = blockIdx.x % tiles_n * (16 * H);
  const int64_t pitch = (int64_t)groups * 64;

  const uint8_t *px[MT], *qx[MT], *pw[NT], *qw[NT];
#pragma unroll
  for (int y = 0; y < MT; ++y) {
    const int64_t i = min(i0 + 16 * y + lane % 16, m - 1);
    px[y] = x.codes + i * 2 * pitch + lane / 16 % 2 * 16;
    qx[y] = x.scales + i * (pitch / 16);
  }
#pragma unroll
  for (int z = 0; z < NT; ++z) {
    const int64_t j = min(j0 + 16 * (z % H) + lane % 16, n - 1) + (z < H ? 0 : n);
    pw[z] = w.codes + j * pitch;
    qw[z] = w.scales + j * (pitch / 16);
  }

  v4f acc[MT][NT];
#pragma unroll
  for (int y = 0; y < MT; ++y)
#pragma unroll
    for (int z = 0; z < NT; ++z) acc[y][z] = v4f{0, 0, 0, 0};

  for (int g0 = 4 * wave; g0 < groups; g0 += 4 * kFewWaves) {
    // What is beyond the last group is that one again, and counts as zeros.
    const bool in = g0 + quarter < groups, lo_in = g0 + quarter / 2 < groups, hi_in = g0 + 2 + quarter / 2 < groups;
    const int g = min(g0 + quarter, groups - 1), lo = min(g0 + quarter / 2, groups - 1), hi = min(g0 + 2 + quarter / 2, groups - 1);
    v4i cw[NT][4];
    int sw[NT], sx[MT];
#pragma unroll
    for (int z = 0; z < NT; ++z) {
#pragma unroll
      for (int j = 0; j < 4; ++j) cw[z][j] = ldg<v4i, false>((const char*)pw[z] + (int64_t)g * 64 + j * 16);
      sw[z] = ldg<int, false>((const char*)qw[z] + (int64_t)g * 4);
      if (!in) sw[z] = 0;
    }
#pragma unroll
    for (int y = 0; y < MT; ++y) {
      sx[y] = ldg<int, false>((const char*)qx[y] + (int64_t)g * 4);
      if (!in) sx[y] = 0;
    }
    auto step = [&](auto which) {
      constexpr int J = decltype(which)::value;
#pragma unroll
      for (int y = 0; y < MT; ++y) {
        v4i a = ldg<v4i, false>((const char*)px[y] + (int64_t)lo * 128 + J * 32);
        v4i b = ldg<v4i, false>((const char*)px[y] + (int64_t)hi * 128 + J * 32);
        if (!lo_in) a = v4i{0, 0, 0, 0};
        if (!hi_in) b = v4i{0, 0, 0, 0};
#pragma unroll
        for (int z = 0; z < NT; ++z)
          acc[y][z] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(frag(cw[z][J]), frag(a, b), acc[y][z], 4, 0, J, sw[z], J,
                                                                      sx[y]);
      }
    };
    step(Int<0>{});
    step(Int<1>{});
    step(Int<2>{});
    step(Int<3>{});
  }

  // The waves' sums in order.  Lane l has rows 4 * (l / 16) ... + 3 of the weight and token l mod 16 of each 16 x 16.
  v4f* sums = (v4f*)lds;
#pragma unroll
  for (int y = 0; y < MT; ++y)
#pragma unroll
    for (int z = 0; z < NT; ++z) sums[((wave * MT + y) * NT + z) * 64 + lane] = acc[y][z];
  __syncthreads();
  for (int u = threadIdx.x; u < 64 * MT * H; u += 64 * kFewWaves) {  // whole waves: four columns of a token each
    const int quad = u % (4 * H), token = u / (4 * H);
    const int at = (token / 16 * NT + quad / 4) * 64 + quad % 4 * 16 + token % 16;
    v4f a = sums[at], b = {0, 0, 0, 0};
#pragma unroll
    for (int v = 1; v < kFewWaves; ++v) a += sums[v * MT * NT * 64 + at];
    if constexpr (GATED) {
      b = sums[at + H * 64];
#pragma unroll
      for (int v = 1; v < kFewWaves; ++v) b += sums[v * MT * NT * 64 + at + H * 64];
    }
    const int64_t i = i0 + token, j = j0 + 4 * quad, left = n - j;
    if constexpr (!GATED) {
      if (i >= m || left <= 0) continue;
      if (e.residual.p) a += load4<O>((const char*)e.residual.p + (i * e.residual.stride + j) * O::kBytes, left);
      store4<O>((char*)e.out.p + (i * e.out.stride + j) * O::kBytes, left, a);
    } else {
      v4f h;
#pragma unroll
      for (int c = 0; c < 4; ++c) h[c] = activate(e.act, a[c]) * b[c];
      const int64_t row = i * ((n + 127) / 128);
      auto keep = [&](MxbOut to, v4f v) {  // eight lanes have a block
#pragma unroll
        for (int c = 0; c < 4; ++c) v[c] = c < left ? v[c] : 0.0f;
        const uint32_t s = mxb_scale_byte(max_of_8(high_bits(v)));
        if (i >= m) return;
        stg<false>((char*)to.codes + row * 128 + j, mxb_codes(v[0], v[1], v[2], v[3], s));
        if (quad % 8 == 0) stg<false>((char*)to.scales + row * 4 + j / 32, (uint8_t)s);
      };
      if (e.saved_a.codes) keep(e.saved_a, a), keep(e.saved_b, b);
      if constexpr (O::kBytes == 1) keep(e.blocks, h);
      else if (i < m && left > 0) store4<O>((char*)e.out.p + (i * e.out.stride + j) * O::kBytes, left, h);
    }
  }
}

template <int MT, int H, bool GATED, typename O>
hipError_t run_few(MxbMat x, MxMat w, int64_t m, int64_t n, int64_t k, Epilogue e, hipStream_t stream) {
  const bool blocks = GATED && (O::kBytes == 1 || e.saved_a.codes);
  const int64_t groups = groups_of(k), out_groups = groups_of(n);
  const int64_t tiles_n = (int64_t)ceil_div(blocks ? out_groups * 128 : n, 16 * H);
  const int64_t band = few_band(m, tiles_n, 16 * MT);
  for (int64_t i = 0; i < m; i += band) {  // as many rows as a launch holds
    const int64_t here = std::min(band, m - i);
    hipLaunchKernelGGL((few_kernel<MT, H, GATED, O>), dim3((unsigned)(ceil_div(here, 16 * MT) * tiles_n)), dim3(64 * kFewWaves),
                       (size_t)kFewWaves * MT * H * (GATED ? 2 : 1) * 1024, stream, x, w, here, n, (int)groups, tiles_n, e);
    x.codes += band * groups * 128, x.scales += band * groups * 4;
    for (MxbOut* q : {&e.blocks, &e.saved_a, &e.saved_b})
      if (q->codes) q->codes += band * out_groups * 128, q->scales += band * out_groups * 4;
    if (e.out.p) e.out.p = (char*)e.out.p + band * e.out.stride * O::kBytes;
    if (e.residual.p) e.residual.p = (const char*)e.residual.p + band * e.residual.stride * O::kBytes;
  }
  return hipGetLastError();
}

template <int MT, typename O>
hipError_t pick_few(MxbMat x, MxMat w, int64_t m, int64_t n, int64_t k, const Epilogue& e, hipStream_t stream) {
  if (e.gated) return run_few<MT, 2, true, O>(x, w, m, n, k, e, stream);
  if constexpr (O::kBytes == 1) return hipErrorInvalidValue;
  else
    switch (few_columns_sixteens(n)) {
      case 1: return run_few<MT, 1, false, O>(x, w, m, n, k, e, stream);
      case 2: return run_few<MT, 2, false, O>(x, w, m, n, k, e, stream);
      default: return run_few<MT, 4, false, O>(x, w, m, n, k, e, stream);
    }
}

template <typename O>
hipError_t pick(MxbMat x, MxMat w, int64_t m, int64_t n, int64_t k, const Epilogue& e, hipStream_t stream) {
  switch (few_tokens_sixteens(m)) {
    case 1: return pick_few<1, O>(x, w, m, n, k, e, stream);
    case 2: return pick_few<2, O>(x, w, m, n, k, e, stream);
    default: return pick_few<3, O>(x, w, m, n, k, e, stream);
  }
}

}  // namespace

hipError_t launch_mxb_product(MxbMat x, MxMat w, int64_t m, int64_t n, int64_t k, const Epilogue& e, hipStream_t stream) {
  if (e.gated && !e.out.p) return pick<Q8>(x, w, m, n, k, e, stream);
  return e.dtype == Elem::f32 ? pick<F32>(x, w, m, n, k, e, stream) : pick<B16>(x, w, m, n, k, e, stream);
}

}  // namespace pat
