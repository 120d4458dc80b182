// Dropout from a counter-based generator; the mask is never stored.
//
// One Philox4x32-10 call gives the 16-bit numbers of 8 consecutive elements (numbered over the whole tensor), so a lane
// takes the 8 elements of a generator block.  16 bits instead of 32 halve the generator's work, whose 20 wide
// multiplications otherwise cost more than the memory; p is met to 2^-17, and the scale belongs to the p that is.
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

// The elements of generator block b that a row of `cols` elements numbered from `start` has: columns c ... c + 7 less
// what is before 0 and behind the row.  Blocks of a row are numbered from the one of its first element.
//
// A row takes `lanes` lanes and kBlocks blocks a lane in turn; a workgroup holds 256 / lanes rows side by side.  Rows
// without gaps in memory and in numbering come as one row.  Whole blocks are read and written as vectors at
// element-aligned addresses.
//
// Bound by memory: 16384 x 4096 bfloat16 with a residual (403 MB) in 60 us, 6.7 TB/s, with the generator's
// multiplications under the loads.  Two blocks a lane, both read before either is numbered.  Loads are nontemporal, stores
// are not (us: 60; both 63, neither 71).
constexpr int kBlocks = kDropoutBlocks;

struct RowSplit {
  int lanes;
  uint32_t tiles;  // workgroups along a row
};

// Elements lo ... hi - 1 of the 8 at p, which may begin before the row.
template <typename T, bool WHOLE>
__device__ __forceinline__ Raw8<T> load_part(const char* p, int lo, int hi) {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < T::kBytes / 2; ++i) r.w[i] = v4u{0, 0, 0, 0};
  if (WHOLE || (lo == 0 && hi == 8)) {
#pragma unroll
    for (int i = 0; i < T::kBytes / 2; ++i) r.w[i] = ldg<v4u, true, T::kBytes>(p + 16 * i);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i < lo || i >= hi) continue;
      if constexpr (T::kBytes == 4) r.w[i / 4][i % 4] = ldg<uint32_t, false>(p + 4 * i);
      else r.w[0][i / 2] |= (uint32_t)ldg<uint16_t, false>(p + 2 * i) << (16 * (i & 1));
    }
  }
  return r;
}
__device__ __forceinline__ float value_of(const Raw8<F32>& r, int i) {
  const uint32_t w = r.w[i / 4][i % 4];
  return __uint_as_float(w);
}
__device__ __forceinline__ float value_of(const Raw8<B16>& r, int i) {
  const uint32_t w = r.w[0][i / 2];
  return i & 1 ? bf16_hi(w) : bf16_lo(w);
}

template <typename T, bool RESIDUAL>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a, RowSplit split) {
  const int side = 256 / split.lanes, lane = threadIdx.x % split.lanes;
  const int64_t step = (int64_t)(gridDim.x / split.tiles) * side;
  const uint32_t tile = blockIdx.x % split.tiles;
  for (int64_t r = (int64_t)(blockIdx.x / split.tiles) * side + threadIdx.x / split.lanes; r < a.rows; r += step) {
    const uint64_t start = a.index + (uint64_t)r * a.index_stride;
    const int64_t behind = (int64_t)(start & 7);  // elements of the row's first block that are before the row
    const int64_t b0 = (int64_t)tile * split.lanes * kBlocks + lane;
    auto blocks = [&](auto whole) {
      constexpr bool WHOLE = decltype(whole)::value;
      Raw8<T> x[kBlocks], res[kBlocks];
#pragma unroll
      for (int u = 0; u < kBlocks; ++u) {
        const int64_t c = 8 * (b0 + u * split.lanes) - behind, left = a.cols - c;
        const int lo = WHOLE ? 0 : (int)max(-c, (int64_t)0), hi = WHOLE ? 8 : (int)min(max(left, (int64_t)0), (int64_t)8);
        x[u] = load_part<T, WHOLE>((const char*)a.x.p + (r * a.x.stride + c) * T::kBytes, lo, hi);
        if constexpr (RESIDUAL)
          res[u] = load_part<T, WHOLE>((const char*)a.residual.p + (r * a.residual.stride + c) * T::kBytes, lo, hi);
      }
#pragma unroll
      for (int u = 0; u < kBlocks; ++u) {
        const int64_t b = b0 + u * split.lanes, c = 8 * b - behind, left = a.cols - c;
        if (!WHOLE && left <= 0) continue;
        // blocks are consecutive modulo 2^61, as element numbers are modulo 2^64
        const v4u w = philox(((start >> 3) + (uint64_t)b) & (~(uint64_t)0 >> 3), a.seed);
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t number = i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xFFFFu;
          y[i] = number >= a.drop ? value_of(x[u], i) * a.scale : 0.0f;
          if constexpr (RESIDUAL) y[i] += value_of(res[u], i);
        }
        char* p = (char*)a.out.p + (r * a.out.stride + c) * T::kBytes;
        if (WHOLE || (c >= 0 && left >= 8)) {
          store8<T, false, false, kWhole>(p, 8, 4, y);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (c + i >= 0 && i < left) T::store(p, i, y[i]);
        }
      }
    };
    const int64_t c_first = 8 * b0 - behind, c_last = c_first + 8 * (kBlocks - 1) * split.lanes;
    if (__all(c_first >= 0 && a.cols - c_last >= 8)) blocks(Bool<true>{});
    else blocks(Bool<false>{});
  }
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& given, Elem dtype, hipStream_t stream) {
  DropoutArgs a = given;
  const DropoutPlan plan = dropout_plan(a.rows, a.cols,
                                        a.x.stride == a.cols && a.out.stride == a.cols && a.index_stride == (uint64_t)a.cols &&
                                            (!a.residual.p || a.residual.stride == a.cols));
  if (plan.flat) {
    a.cols *= a.rows;
    a.rows = 1;
  }
  const RowSplit split{plan.lanes, (uint32_t)plan.tiles};
  const dim3 grid((unsigned)plan.wgs);
  const auto kernel = dtype == Elem::f32 ? (a.residual.p ? dropout_kernel<F32, true> : dropout_kernel<F32, false>)
                                         : (a.residual.p ? dropout_kernel<B16, true> : dropout_kernel<B16, false>);
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a, split);
  return hipGetLastError();
}

}  // namespace pat
