// Device-side building blocks of a layer's operators: the 8-bit blocks' arithmetic, activations, sums over lanes.
#pragma once

#include "ops_device.hpp"

namespace pat {
namespace {

typedef short v2s __attribute__((ext_vector_type(2)));

// Values that leave in 8-bit blocks, beside F32 and B16.
struct Q8 {
  static constexpr int kBytes = 1;
};

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float round_to(F32, float v) { return v; }
__device__ __forceinline__ float round_to(B16, float v) { return (float)(__bf16)v; }

// ---- 8-bit blocks

// Scale byte of a block's largest magnitude (as float32 bits): exponent less 1, one more above 1.875 times a power of two.
__device__ __forceinline__ uint32_t mxb_scale_byte(uint32_t high_bits) {
  const uint32_t up = (high_bits + 0x0FFFFFu) >> 23;
  return high_bits >= 0x7F800000u ? 255u : up > 1u ? up - 1u : 0u;
}
// The codes of four values under scale byte s, one word; no magnitude is above 3.75 times the scale.
__device__ __forceinline__ uint32_t mxb_codes(float a, float b, float c, float d, uint32_t s) {
  const float scale = mx_scale_operand(s);
  v2s w = {0, 0};
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, scale, false);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, scale, true);
  return s == 255u ? 0u : __builtin_bit_cast(uint32_t, w);
}
// The codes of eight elements as they are in memory.
__device__ __forceinline__ v2u mxb_codes(const Raw8<F32>& r, uint32_t s) {
  auto f = [&](int i) { return __uint_as_float(r.w[i / 4][i % 4]); };
  return v2u{mxb_codes(f(0), f(1), f(2), f(3), s), mxb_codes(f(4), f(5), f(6), f(7), s)};
}
__device__ __forceinline__ v2u mxb_codes(const Raw8<B16>& r, uint32_t s) {
  const float scale = mx_scale_operand(s);
  auto f = [&](int i) {
    const uint32_t w = r.w[0][i];
    return __builtin_bit_cast(v2bf, w);
  };
  v2s lo = {0, 0}, hi = {0, 0};
  lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, f(0), scale, false);
  lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, f(1), scale, true);
  hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, f(2), scale, false);
  hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, f(3), scale, true);
  if (s == 255u) return v2u{0, 0};
  return v2u{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}
// What four codes stand for.
__device__ __forceinline__ void mxb_values(uint32_t codes, uint32_t s, float* v) {
  const float scale = mx_scale_operand(s);
  const v2f lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, scale, false);
  const v2f hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, scale, true);
  v[0] = lo[0], v[1] = lo[1], v[2] = hi[0], v[3] = hi[1];
}

// ---- activations
//
// By the hardware's 2^x and 1 / x, each within a unit in the last place: the exponential's relative error grows with that of
// a log2 e, 1.23 |a| 2^-24 (0.23 of it the constant's).  Where it overflows, from a = -88.7 down, 1 / inf = 0 stands for a e^a
// of up to 2^-121.

constexpr float kLog2e = 1.44269504088896341f;

__device__ __forceinline__ float sigmoid(float a) { return __builtin_amdgcn_rcpf(1.0f + exp2_of(-kLog2e * a)); }

// P(a) = (1 + erf(a / sqrt 2)) / 2, and e^(-a^2 / 2).  For x = |a| / sqrt 2, erfc(x) e^(x^2) is a polynomial in t = 1 / (1 + 0.36 x)
// (the form of Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26; degree and coefficients by a minimax fit):
// P is off by 9e-9 for that, and by 3.9 * 2^-24 with float32's roundings (near zero, where t is off most), 5.9 * 2^-24 where the
// hardware's 1 / x and 2^x are a unit off; of itself by 4e-5 down to -5, 1e-4 down to -13.  A third of erff's
// instructions, and the bell is there already: 5.1 us instead of 5.9 for the gated block's gradient of 300 x 4096.
__device__ __forceinline__ float normal_below(float a, float* bell) {
  const float t = __builtin_amdgcn_rcpf(1.0f + 0.254558441f * fabsf(a));
  float p = -0.157440618f;
  p = fmaf(p, t, 0.535437644f);
  p = fmaf(p, t, -0.301273644f);
  p = fmaf(p, t, 0.375326842f);
  p = fmaf(p, t, 0.136009216f);
  p = fmaf(p, t, 0.208934069f);
  p = fmaf(p, t, 0.203006476f);
  *bell = exp2_of(-0.5f * kLog2e * a * a);
  const float q = 0.5f * (p * t) * *bell;
  return a >= 0.0f ? 1.0f - q : q;
}

__device__ __forceinline__ float activate(Act act, float a) {
  if (act == Act::silu) return a * sigmoid(a);
  float bell;
  return a * normal_below(a, &bell);
}
// The activation, and its derivative.
__device__ __forceinline__ float activate(Act act, float a, float* slope) {
  if (act == Act::silu) {
    const float s = sigmoid(a);
    *slope = s * (1.0f + a * (1.0f - s));
    return a * s;
  }
  float bell;
  const float p = normal_below(a, &bell);
  *slope = p + a * (0.398942280401432678f * bell);
  return a * p;
}

// ---- sums

// The sum over each `lanes` consecutive lanes (a power of two up to 64), in every one of them and the same bits in all;
// every lane of the wave has to be active.
__device__ __forceinline__ float sum_of_lanes(float v, int lanes) {
  auto add = [&](uint32_t other) { v += __uint_as_float(other); };
  if (lanes > 1) add(dpp<0xB1>(__float_as_uint(v)));   // quad_perm 1, 0, 3, 2
  if (lanes > 2) add(dpp<0x4E>(__float_as_uint(v)));   // quad_perm 2, 3, 0, 1
  if (lanes > 4) add(dpp<0x141>(__float_as_uint(v)));  // the other four of eight, mirrored
  if (lanes > 8) add(dpp<0x140>(__float_as_uint(v)));  // the other eight of sixteen, mirrored
  if (lanes > 16) v += __shfl_xor(v, 16);
  if (lanes > 32) v += __shfl_xor(v, 32);
  return v;
}

}  // namespace
}  // namespace pat
