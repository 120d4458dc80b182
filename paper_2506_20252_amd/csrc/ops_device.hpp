// Device-side building blocks of the operators: element types, short vectors,
// the 4-bit format's scale arithmetic and division by a launch constant.
#pragma once

#include <hip/hip_runtime.h>

#include "device_access.hpp"
#include "ops.hpp"

namespace pat {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

// Two float32 to bfloat16 (nearest even, NaN stays NaN), the first in the low half: one instruction.
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  const v2bf v = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, v);
}

// An element type in memory: single elements, and 8 consecutive ones as vectors at element-aligned addresses, of
// which the first n count (the others read as 0 and are not written).  NT: nontemporal.
struct F32 {
  static constexpr int kBytes = 4;
  __device__ static float load(const char* p, int64_t i) { return ldg<float, false>(p + i * 4); }
  __device__ static void store(char* p, int64_t i, float v) { stg<false>(p + i * 4, v); }
  template <bool NT>
  __device__ static void load8(const char* p, int64_t n, float (&v)[8]) {
    if (n >= 8) {
      const v4f a = ldg<v4f, NT, 4>(p), b = ldg<v4f, NT, 4>(p + 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < n ? ldg<float, false>(p + 4 * i) : 0.0f;
    }
  }
  template <bool NT>
  __device__ static void store8(char* p, int64_t n, const float (&v)[8]) {
    if (n >= 8) {
      stg<NT, 4>(p, v4f{v[0], v[1], v[2], v[3]});
      stg<NT, 4>(p + 16, v4f{v[4], v[5], v[6], v[7]});
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < n) stg<false>(p + 4 * i, v[i]);
    }
  }
};
struct B16 {
  static constexpr int kBytes = 2;
  __device__ static float load(const char* p, int64_t i) { return bf16_lo(ldg<uint16_t, false>(p + i * 2)); }
  __device__ static void store(char* p, int64_t i, float v) { stg<false>(p + i * 2, (uint16_t)bf16_rne(v)); }
  template <bool NT>
  __device__ static void load8(const char* p, int64_t n, float (&v)[8]) {
    if (n >= 8) {
      const v4u a = ldg<v4u, NT, 2>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[2 * i] = bf16_lo(a[i]), v[2 * i + 1] = bf16_hi(a[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < n ? bf16_lo(ldg<uint16_t, false>(p + 2 * i)) : 0.0f;
    }
  }
  template <bool NT>
  __device__ static void store8(char* p, int64_t n, const float (&v)[8]) {
    if (n >= 8) {
      v4u a;
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
      stg<NT, 2>(p, a);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < n) stg<false>(p + 2 * i, (uint16_t)bf16_rne(v[i]));
    }
  }
};

// Lanes of a power of two that take a row of `vectors` vectors, at most a workgroup of `threads`.
inline int row_lanes(int64_t vectors, int threads) {
  int lanes = 1;
  while (lanes < vectors && lanes < threads) lanes *= 2;
  return lanes;
}

// 4-bit blocks: scale byte of the block's largest magnitude (as float32 bits), and the powers of two around it.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t high_bits) {
  const uint32_t field = high_bits >> 23;
  return field == 255u ? 255u : (field > 2u ? field - 2u : 0u);
}
// 2^(s - 127); s = 0 is the subnormal 2^-127, s = 255 NaN.
__device__ __forceinline__ float mx_scale_value(uint32_t s) {
  return __uint_as_float(s == 0u ? 0x00400000u : s == 255u ? 0x7FC00000u : s << 23);
}

}  // namespace
}  // namespace pat
