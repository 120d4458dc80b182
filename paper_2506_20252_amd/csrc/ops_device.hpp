// Device-side building blocks of the operators: element types, short vectors,
// the 4-bit format's scale arithmetic and division by a launch constant.
#pragma once

#include <hip/hip_runtime.h>

#include "device_access.hpp"
#include "ops.hpp"
#include "ops_shape.hpp"

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

// A compile-time truth value as an argument.
template <bool B>
struct Bool {
  static constexpr bool value = B;
};

// Element types in memory: single elements, and a lane's 8 columns as vectors at element-aligned addresses.
struct F32 {
  static constexpr int kBytes = 4;
  typedef v4f vec4;
  __device__ static float load(const char* p, int64_t i) { return ldg<float, false>(p + i * 4); }
  __device__ static void store(char* p, int64_t i, float v) { stg<false>(p + i * 4, v); }
  __device__ static void widen(const vec4& a, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i];
  }
  __device__ static vec4 narrow(const float* v) { return vec4{v[0], v[1], v[2], v[3]}; }
};
struct B16 {
  static constexpr int kBytes = 2;
  typedef v2u vec4;
  __device__ static float load(const char* p, int64_t i) { return bf16_lo(ldg<uint16_t, false>(p + i * 2)); }
  __device__ static void store(char* p, int64_t i, float v) { stg<false>(p + i * 2, (uint16_t)bf16_rne(v)); }
  __device__ static void widen(const vec4& a, float* v) {
#pragma unroll
    for (int i = 0; i < 2; ++i) v[2 * i] = bf16_lo(a[i]), v[2 * i + 1] = bf16_hi(a[i]);
  }
  __device__ static vec4 narrow(const float* v) { return vec4{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])}; }
};

// The 8 columns that a lane takes at a time out of `lanes` lanes' 8 * lanes: one vector of 16 bytes where every type
// is bfloat16, else two vectors of 4 columns, `lanes` vectors apart.  Either way the lanes of a wave read and write
// consecutive bytes with each instruction; float32 columns taken 8 in a row would be written in alternate
// 16-byte pieces.
template <typename A, typename B>
struct Split {
  static constexpr bool value = A::kBytes == 4 || B::kBytes == 4;
};
// First of a lane's columns, and from there to the first of its second four.
template <bool SPLIT>
__device__ __forceinline__ int64_t lane_column(int lane) {
  return SPLIT ? 4 * lane : 8 * lane;
}
template <bool SPLIT>
__device__ __forceinline__ int64_t lane_gap(int lanes) {
  return SPLIT ? 4 * lanes : 4;
}

// Loads and stores of such columns at p, of which those below n (counted from p) exist: others read as 0 and are not
// written.  Whether all exist is decided for a whole wave, and no load hides behind a branch of a lane's own, so the
// loads of several rows are in flight together:
//   kWhole  all exist;
//   kEnd    a vector that would go over the row's end ends there and is moved down (rows of 4 columns and more);
//   kFew    columns one by one.
enum Cover { kWhole, kEnd, kFew };
template <Cover C>
struct CoverOf {
  static constexpr Cover value = C;
};
__device__ __forceinline__ Cover cover_of(int64_t n, int64_t gap, int64_t cols) {
  return __all(n >= gap + 4) ? kWhole : cols >= 4 ? kEnd : kFew;
}

// Four values moved down by d places, zeros behind them.
__device__ __forceinline__ void move_down(float* v, int64_t d) {
  const float t0 = d & 1 ? v[1] : v[0], t1 = d & 1 ? v[2] : v[1], t2 = d & 1 ? v[3] : v[2], t3 = d & 1 ? 0.0f : v[3];
  v[0] = d >= 4 ? 0.0f : d & 2 ? t2 : t0;
  v[1] = d >= 4 ? 0.0f : d & 2 ? t3 : t1;
  v[2] = d >= 2 ? 0.0f : t2;
  v[3] = d >= 2 ? 0.0f : t3;
}

template <typename T, bool SPLIT, bool NT, Cover C>
__device__ __forceinline__ void load8(const char* p, int64_t n, int64_t gap, float (&v)[8]) {
  typedef typename T::vec4 V;
  if constexpr (C == kWhole && !SPLIT && T::kBytes == 2) {
    const v4u a = ldg<v4u, NT, 2>(p);
    T::widen({a[0], a[1]}, v);
    T::widen({a[2], a[3]}, v + 4);
  } else if constexpr (C == kWhole) {
    const V a = ldg<V, NT, T::kBytes>(p), b = ldg<V, NT, T::kBytes>(p + gap * T::kBytes);
    T::widen(a, v);
    T::widen(b, v + 4);
  } else if constexpr (C == kEnd) {
    const int64_t at = min((int64_t)0, n - 4), to = min(gap, n - 4);
    const V a = ldg<V, NT, T::kBytes>(p + at * T::kBytes), b = ldg<V, NT, T::kBytes>(p + to * T::kBytes);
    T::widen(a, v);
    T::widen(b, v + 4);
    move_down(v, -at);
    move_down(v + 4, gap - to);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t at = i < 4 ? i : gap + i - 4;
      v[i] = at < n ? T::load(p, at) : 0.0f;
    }
  }
}
template <typename T, bool SPLIT, bool NT, Cover C>
__device__ __forceinline__ void store8(char* p, int64_t n, int64_t gap, const float (&v)[8]) {
  if constexpr (C == kWhole && !SPLIT && T::kBytes == 2) {
    const v2u a = T::narrow(v), b = T::narrow(v + 4);
    stg<NT, 2>(p, v4u{a[0], a[1], b[0], b[1]});
  } else if constexpr (C == kWhole) {
    stg<NT, T::kBytes>(p, T::narrow(v));
    stg<NT, T::kBytes>(p + gap * T::kBytes, T::narrow(v + 4));
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t at = h * gap;
      if (n - at >= 4) {
        stg<NT, T::kBytes>(p + at * T::kBytes, T::narrow(v + 4 * h));
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (at + i < n) T::store(p, at + i, v[4 * h + i]);
      }
    }
  }
}

// 4-bit blocks: scale byte of the block's largest magnitude (as float32 bits), and the powers of two around it.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t high_bits) {
  const uint32_t field = high_bits >> 23;
  return field == 255u ? 255u : (field > 2u ? field - 2u : 0u);
}
// The scale operand of the conversion instructions, of which they take the exponent field alone: 2^(s - 127), 0 being
// 2^-127 and 255 NaN.
__device__ __forceinline__ float mx_scale_operand(uint32_t s) { return __uint_as_float(s << 23); }

// Eight consecutive elements as they are in memory; nothing is done with what is loaded, so that several are in flight
// together.
template <typename T>
struct Raw8 {
  v4u w[T::kBytes / 2];
};

// The eight elements from column c of a row of `cols`, those behind it zero, as above: kWhole where eight exist or none,
// kEnd for rows of 8 columns and more (settle() moves them once they are there), kFew else.
__device__ __forceinline__ void move_down(Raw8<B16>& r, int d) {
  uint64_t lo = r.w[0][0] | (uint64_t)r.w[0][1] << 32, hi = r.w[0][2] | (uint64_t)r.w[0][3] << 32;
  if (d >= 4) lo = hi, hi = 0, d -= 4;
  if (d >= 4) lo = 0, d = 0;
  if (d > 0) lo = lo >> 16 * d | hi << (64 - 16 * d), hi >>= 16 * d;
  r.w[0] = v4u{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}
__device__ __forceinline__ void move_down(Raw8<F32>& r, int d) {
#pragma unroll
  for (int s = 1; s <= 8; s *= 2) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t from = i + s < 8 ? r.w[(i + s) / 4 % 2][(i + s) % 4] : 0u;
      r.w[i / 4][i % 4] = d & s ? from : r.w[i / 4][i % 4];
    }
  }
}
template <typename T, Cover C, bool NT = false>
__device__ __forceinline__ Raw8<T> load_raw8(const char* row, int64_t c, int64_t cols) {
  Raw8<T> r;
  if constexpr (C == kEnd) {
    const int64_t at = min(c, cols - 8);
#pragma unroll
    for (int i = 0; i < T::kBytes / 2; ++i) r.w[i] = ldg<v4u, NT, T::kBytes>(row + at * T::kBytes + 16 * i);
    return r;
  }
#pragma unroll
  for (int i = 0; i < T::kBytes / 2; ++i) r.w[i] = v4u{0, 0, 0, 0};
  if constexpr (C == kWhole) {
    if (c < cols) {
#pragma unroll
      for (int i = 0; i < T::kBytes / 2; ++i) r.w[i] = ldg<v4u, NT, T::kBytes>(row + c * T::kBytes + 16 * i);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (c + i >= cols) break;
      if constexpr (T::kBytes == 4) r.w[i / 4][i % 4] = ldg<uint32_t, false>(row + 4 * (c + i));
      else r.w[0][i / 2] |= (uint32_t)ldg<uint16_t, false>(row + 2 * (c + i)) << (16 * (i & 1));
    }
  }
  return r;
}
template <Cover C, typename T>
__device__ __forceinline__ void settle(Raw8<T>& r, int64_t c, int64_t cols) {
  if constexpr (C == kEnd) move_down(r, (int)min(max(c - (cols - 8), (int64_t)0), (int64_t)8));
}

// Largest magnitude of 8 elements, as float32 bits.
__device__ __forceinline__ uint32_t high_bits(const Raw8<F32>& r) {
  uint32_t h = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) h = max(h, r.w[i / 4][i % 4] & 0x7FFFFFFFu);
  return h;
}
__device__ __forceinline__ uint32_t high_bits(const Raw8<B16>& r) {
  typedef unsigned short v2h __attribute__((ext_vector_type(2)));
  v2h h = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) h = __builtin_elementwise_max(h, __builtin_bit_cast(v2h, r.w[0][i] & 0x7FFF7FFFu));
  return (uint32_t)(h[0] > h[1] ? h[0] : h[1]) << 16;
}

// The codes of 8 elements under scale byte s, one word.
__device__ __forceinline__ uint32_t mx_codes(const Raw8<F32>& r, uint32_t s) {
  const float scale = mx_scale_operand(s);
  auto f = [&](int i) { return __uint_as_float(r.w[i / 4][i % 4]); };
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f(0), f(1), scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f(2), f(3), scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f(4), f(5), scale, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f(6), f(7), scale, 3);
  return s == 255u ? 0u : c;
}
__device__ __forceinline__ uint32_t mx_codes(const Raw8<B16>& r, uint32_t s) {
  const float scale = mx_scale_operand(s);
  auto f = [&](int i) {
    const uint32_t w = r.w[0][i];  // __builtin_bit_cast of a vector's element itself takes its first one
    return __builtin_bit_cast(v2bf, w);
  };
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, f(0), scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, f(1), scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, f(2), scale, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, f(3), scale, 3);
  return s == 255u ? 0u : c;
}

// Division of numbers below 2^31 by a launch constant d < 2^31: with 2^(s - 1) < d <= 2^s and
// m = ceil(2^(31 + s) / d) < 2^32, n / d = n * m >> (31 + s), since n * (m * d - 2^(31 + s)) < 2^(31 + s).
struct Divisor {
  uint32_t d, m;
  int shift;
  explicit Divisor(uint32_t divisor) : d(divisor), m(0), shift(31) {
    while (((uint64_t)1 << (shift - 31)) < d) ++shift;
    m = (uint32_t)((((__uint128_t)1 << shift) + d - 1) / d);
  }
  __device__ __forceinline__ uint32_t divide(uint32_t n) const { return (uint32_t)((uint64_t)n * m >> shift); }
};

// Lane exchange inside groups of 4 and 16 lanes; every lane of the wave has to be active.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
__device__ __forceinline__ uint32_t max_of_4(uint32_t v) {
  v = max(v, dpp<0xB1>(v));         // quad_perm 1, 0, 3, 2
  return max(v, dpp<0x4E>(v));      // quad_perm 2, 3, 0, 1
}
__device__ __forceinline__ uint32_t or_of_16_by_4(uint32_t v) {
  v |= dpp<0x124>(v);               // row_ror 4
  return v | dpp<0x128>(v);         // row_ror 8
}

// Where a tile of the output is; neighbours in `t` share rows of a or b.
struct TilePlace {
  int64_t i, j;
};
// Workgroups go to the 8 XCDs in turn; each XCD gets consecutive tiles, in bands of 6 tile rows, so that the 32 tiles that
// it works on together are nearly square and what they read stays in its L2 (us with bands of 4, 6, 8, 16: 297, 294, 300,
// 300 for 8192 x 8192 x 8192 with its quantisation, 445, 447, 455, 470 for both gradients of 8192 x 4096 x 4096;
// timed at these two sizes alone).
__device__ __forceinline__ bool tile_place(int64_t tiles_m, int64_t tiles_n, TilePlace* p) {
  constexpr int kBand = 6;
  const int64_t total = tiles_m * tiles_n, per = (total + 7) / 8;
  const int64_t t = blockIdx.x % 8 * per + blockIdx.x / 8;
  if (blockIdx.x / 8 >= per || t >= total) return false;
  const int64_t band = t / (kBand * tiles_n), in_band = t % (kBand * tiles_n);
  const int64_t high = min((int64_t)kBand, tiles_m - band * kBand);
  p->i = band * kBand + in_band % high;
  p->j = in_band / high;
  return true;
}

// Writes a wave's FA x FB blocks of 32 x 32, as the 32 x 32 matrix instructions leave them (lane l: column l mod 32, rows
// 8 * (e / 4) + 4 * (l / 32) + e mod 4), to rows wave_row ... and columns wave_col ... of the tile at (i0, j0).  The wave
// turns 32 rows at a time round in a part of LDS of its own, the `slot`-th at `lds` (tile_part floats each), and writes
// them as vectors.  Nobody may still be reading that LDS when the last wave comes here: the barrier is in here.
constexpr int tile_part(int fb) { return 32 * (32 * fb + 8); }  // rows 8 banks apart, for the halves' rows of 4 apart

template <int FA, int FB, typename T, bool NT>
__device__ __forceinline__ void write_tile(const v16f (&acc)[FA][FB], float* lds, int slot, int wave_row, int wave_col,
                                           int64_t i0, int64_t j0, int64_t rows, int64_t cols, MatOut out) {
  constexpr int C = 32 * FB, P = C + 8, LANES = C / 8;  // columns, their pitch, lanes a row with 8 columns each
  const int lane = threadIdx.x % 64, half = lane / 32;
  __syncthreads();
  float* part = lds + slot * tile_part(FB);
#pragma unroll
  for (int x = 0; x < FA; ++x) {
#pragma unroll
    for (int y = 0; y < FB; ++y)
#pragma unroll
      for (int e = 0; e < 16; ++e) part[(8 * (e / 4) + 4 * half + e % 4) * P + 32 * y + lane % 32] = acc[x][y][e];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int u = 0; u < 32 * LANES / 64; ++u) {
      const int r = u * (64 / LANES) + lane / LANES, c = lane % LANES * 8;
      const int64_t i = i0 + wave_row + 32 * x + r, j = j0 + wave_col + c;
      const v4f lo = *(const v4f*)(part + r * P + c), hi = *(const v4f*)(part + r * P + c + 4);
      const float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      char* p = (char*)out.p + (i * out.stride + j) * T::kBytes;
      if (i < rows && cols - j >= 8) store8<T, false, NT, kWhole>(p, 8, 4, v);
      else if (i < rows && cols > j) store8<T, false, NT, kEnd>(p, cols - j, 4, v);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

}  // namespace
}  // namespace pat
