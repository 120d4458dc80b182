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

// An element type in memory, and its 16-byte-or-wider vector of 8 elements.
struct F32 {
  static constexpr int kBytes = 4;
  __device__ static float load(const char* p, int64_t i) { return ldg<float, false>(p + i * 4); }
  __device__ static void store(char* p, int64_t i, float v) { stg<false>(p + i * 4, v); }
};
struct B16 {
  static constexpr int kBytes = 2;
  __device__ static float load(const char* p, int64_t i) { return bf16_lo(ldg<uint16_t, false>(p + i * 2)); }
  __device__ static void store(char* p, int64_t i, float v) { stg<false>(p + i * 2, (uint16_t)bf16_rne(v)); }
};

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
