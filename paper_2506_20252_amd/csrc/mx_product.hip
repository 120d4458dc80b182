// Products of two 4-bit matrices, out = a b^T, on the scaled matrix instructions.
//
// A matrix instruction multiplies codes as they are stored and applies both blocks' scales: nothing is widened.
// Two kernels:
//   tile_kernel   many rows on both sides: tiles of both matrices go through LDS;
//   split_kernel  few rows or few tiles: every wave of a workgroup takes its part of the columns straight from
//                 memory, and the waves' sums are added in order.
#include <algorithm>

#include "ops_device.hpp"

namespace pat {
namespace {

typedef __attribute__((address_space(1))) const uint32_t* GlobalWords;
typedef __attribute__((address_space(3))) uint32_t* LdsWords;

template <int I>
struct Int {
  static constexpr int value = I;
};

__device__ __forceinline__ v8i frag(v4i c) { return v8i{c[0], c[1], c[2], c[3], 0, 0, 0, 0}; }

// ---- tiles through LDS ---------------------------------------------------------------------------------------
//
// A workgroup of 2 x 2 waves computes a tile of 2 * 32 * F rows and columns, a wave F x F blocks of 32 x 32.  It goes
// through the columns 256 at a time (two groups, 128 bytes of codes a row).  The next 256 columns of both sides are
// on their way into the other half of LDS, written there by the loads themselves, while these are multiplied.
//
// LDS holds a row's eight 16-byte blocks of codes at place block ^ (row mod 8), so that lanes reading one block of
// consecutive rows hit different banks; the loads write lane after lane, so each lane fetches the block that
// belongs at its place.  An instruction of 32 x 32 x 64 takes two blocks of 32 rows: lane l has row l mod 32 and one
// block, and any two blocks will do as long as both sides take the same.  Lane half h takes blocks 2h and 2h + 1 of a
// group in turn, whose scales are two neighbouring bytes: the instruction picks the byte.

constexpr int kTileThreads = 256;

template <int F>
struct TileLds {
  static constexpr int kRows = 64 * F;
  uint8_t codes[2][kRows * 128];  // [a, b]
  uint8_t scales[2][kRows * 8];
};

template <int F, typename T>
__global__ __launch_bounds__(kTileThreads, F == 4 ? 1 : 2) void tile_kernel(MxMat a, MxMat b, int64_t m, int64_t n,
                                                                             int groups, MatOut out) {
  constexpr int R = 64 * F;
  __shared__ __attribute__((aligned(16))) TileLds<F> lds0;
  __shared__ __attribute__((aligned(16))) TileLds<F> lds1;
  TilePlace place;
  if (!tile_place((m + R - 1) / R, (n + R - 1) / R, &place)) return;
  const int64_t i0 = place.i * R, j0 = place.j * R;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint32_t pitch = groups * 64, spitch = groups * 4;

  // Rows beyond a matrix are its last row again; what they give is not stored.
  const int rows_a = (int)min((int64_t)R, m - i0), rows_b = (int)min((int64_t)R, n - j0);
  uint32_t at_a[F * 2], at_b[F * 2];  // of this lane's block, in the rows' codes
  const int block = lane % 8 ^ lane / 8;
#pragma unroll
  for (int u = 0; u < F * 2; ++u) {
    const int row = (u * 4 + wave) * 8 + lane / 8;
    at_a[u] = (uint32_t)min(row, rows_a - 1) * pitch + block * 16;
    at_b[u] = (uint32_t)min(row, rows_b - 1) * pitch + block * 16;
  }
  constexpr int SU = (F + 1) / 2;  // loads of scales: 32 rows of 8 bytes a wave
  uint32_t sat_a[SU], sat_b[SU];
#pragma unroll
  for (int u = 0; u < SU; ++u) {
    const int row = (u * 4 + wave) * 32 + lane / 2;
    sat_a[u] = (uint32_t)min(row, rows_a - 1) * spitch + lane % 2 * 4;
    sat_b[u] = (uint32_t)min(row, rows_b - 1) * spitch + lane % 2 * 4;
  }
  const uint8_t *codes_a = a.codes + i0 * pitch, *codes_b = b.codes + j0 * pitch;
  const uint8_t *scales_a = a.scales + i0 * spitch, *scales_b = b.scales + j0 * spitch;

  auto fetch = [&](TileLds<F>& l, int g) {
    // the second group of the last 256 columns may not exist: the first again, not multiplied
    const uint32_t back = g + 1 < groups ? 0 : (block >= 4 ? 64 : 0), sback = g + 1 < groups ? 0 : lane % 2 * 4;
    const uint8_t *pa = codes_a + (int64_t)g * 64, *pb = codes_b + (int64_t)g * 64;
#pragma unroll
    for (int u = 0; u < F * 2; ++u) {
      __builtin_amdgcn_global_load_lds((GlobalWords)(pa + (at_a[u] - back)), (LdsWords)(l.codes[0] + (u * 4 + wave) * 1024),
                                       16, 0, 0);
      __builtin_amdgcn_global_load_lds((GlobalWords)(pb + (at_b[u] - back)), (LdsWords)(l.codes[1] + (u * 4 + wave) * 1024),
                                       16, 0, 0);
    }
    const uint8_t *qa = scales_a + (int64_t)g * 4, *qb = scales_b + (int64_t)g * 4;
#pragma unroll
    for (int u = 0; u < SU; ++u) {
      if ((u * 4 + wave) * 32 >= R) continue;
      __builtin_amdgcn_global_load_lds((GlobalWords)(qa + (sat_a[u] - sback)), (LdsWords)(l.scales[0] + (u * 4 + wave) * 256),
                                       4, 0, 0);
      __builtin_amdgcn_global_load_lds((GlobalWords)(qb + (sat_b[u] - sback)), (LdsWords)(l.scales[1] + (u * 4 + wave) * 256),
                                       4, 0, 0);
    }
  };

  const int row_a = wave / 2 * 32 * F + lane % 32, row_b = wave % 2 * 32 * F + lane % 32, half = lane / 32;
  v16f acc[F][F];
#pragma unroll
  for (int x = 0; x < F; ++x)
#pragma unroll
    for (int y = 0; y < F; ++y)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[x][y][e] = 0.0f;

  auto multiply = [&](const TileLds<F>& l, int g) {
    v2u sa[F], sb[F];
#pragma unroll
    for (int x = 0; x < F; ++x) {
      sa[x] = *(const v2u*)(l.scales[0] + (row_a + 32 * x) * 8);
      sb[x] = *(const v2u*)(l.scales[1] + (row_b + 32 * x) * 8);
    }
    auto group = [&](int e) {
      int fa[F], fb[F];
#pragma unroll
      for (int x = 0; x < F; ++x) fa[x] = sa[x][e] >> (16 * half), fb[x] = sb[x][e] >> (16 * half);
      auto step = [&](auto which) {
        constexpr int J = decltype(which)::value;
        const int at = ((e * 4 + half * 2 + J) ^ (lane & 7)) * 16;
        v4i ca[F], cb[F];
#pragma unroll
        for (int x = 0; x < F; ++x) {
          ca[x] = *(const v4i*)(l.codes[0] + (row_a + 32 * x) * 128 + at);
          cb[x] = *(const v4i*)(l.codes[1] + (row_b + 32 * x) * 128 + at);
        }
#pragma unroll
        for (int x = 0; x < F; ++x)
#pragma unroll
          for (int y = 0; y < F; ++y)
            acc[x][y] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(frag(ca[x]), frag(cb[y]), acc[x][y], 4, 4, J, fa[x], J,
                                                                       fb[y]);
      };
      step(Int<0>{});
      step(Int<1>{});
    };
    group(0);
    if (g + 1 < groups) group(1);
  };

  fetch(lds0, 0);
  for (int g = 0; g < groups; g += 4) {
    __syncthreads();  // these columns have arrived, and nobody reads the other half any more
    if (g + 2 < groups) fetch(lds1, g + 2);
    multiply(lds0, g);
    if (g + 2 >= groups) break;
    __syncthreads();
    if (g + 4 < groups) fetch(lds0, g + 4);
    multiply(lds1, g + 2);
  }

  // Lane l has column l mod 32 of a block and rows 8 * (e / 4) + 4 * (l / 32) + e mod 4.
#pragma unroll
  for (int x = 0; x < F; ++x) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int row = wave / 2 * 32 * F + 32 * x + 8 * (e / 4) + 4 * half + e % 4;
      if (row >= rows_a) continue;
      char* p = (char*)out.p + ((i0 + row) * out.stride + j0) * T::kBytes;
#pragma unroll
      for (int y = 0; y < F; ++y)
        if (row_b + 32 * y < rows_b) T::store(p, row_b + 32 * y, acc[x][y][e]);
    }
  }
}

// ---- few rows ------------------------------------------------------------------------------------------------
//
// A workgroup computes 16 * MT rows by 16 * NT columns; its waves take 512 columns (four groups) in turn.  An
// instruction of 16 x 16 x 128 takes four blocks of 16 rows; lane l takes row l mod 16 and, of the four groups, group
// l / 16: 64 consecutive bytes of codes in four instructions, whose four scales are one word.
//
// FUSED: the rows of a are still x, float32 or bfloat16.  The workgroup quantises all of them into LDS first; every
// workgroup repeats that, which is little beside its part of b as long as the rows are few.

constexpr int kSplitWaves = 8;

template <int MT, int NT, bool FUSED, typename X, typename T>
__global__ __launch_bounds__(64 * kSplitWaves) void split_kernel(MxMat a, Mat x, MxMat b, int64_t m, int64_t n, int64_t k,
                                                                  int groups, MatOut out) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int64_t tiles_n = (n + 16 * NT - 1) / (16 * NT);
  const int64_t i0 = blockIdx.x / tiles_n * (16 * MT), j0 = blockIdx.x % tiles_n * (16 * NT);
  const int64_t pitch = (int64_t)groups * 64;

  const uint8_t *pa[MT], *pb[NT], *qa[MT], *qb[NT];
  const int lds_pitch = groups * 64 + 16;  // the extra block spreads rows over the banks
  uint8_t* lds_scales = lds + m * lds_pitch;
#pragma unroll
  for (int y = 0; y < MT; ++y) {
    const int64_t i = min(i0 + 16 * y + lane % 16, m - 1);
    pa[y] = FUSED ? lds + i * lds_pitch : a.codes + i * pitch;
    qa[y] = FUSED ? lds_scales + i * groups * 4 : a.scales + i * (pitch / 16);
  }
#pragma unroll
  for (int y = 0; y < NT; ++y) {
    const int64_t j = min(j0 + 16 * y + lane % 16, n - 1);
    pb[y] = b.codes + j * pitch;
    qb[y] = b.scales + j * (pitch / 16);
  }

  if constexpr (FUSED) {
    const int blocks = groups * 4;
    for (int i = threadIdx.x; i < (int)m * blocks; i += 64 * kSplitWaves) {
      const int r = i / blocks, c = i % blocks * 32;
      const char* p = (const char*)x.p + (r * x.stride + c) * X::kBytes;
      float v[32];
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        float part[8];
        if (k - c >= 8 * w + 8) load8<X, false, false, true>(p + 8 * w * X::kBytes, 8, 4, part);
        else load8<X, false, false, false>(p + 8 * w * X::kBytes, k - c - 8 * w, 4, part);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[8 * w + e] = part[e];
      }
      uint32_t high = 0;
#pragma unroll
      for (int e = 0; e < 32; ++e) high = max(high, __float_as_uint(v[e]) & 0x7FFFFFFFu);
      const uint32_t s = mx_scale_byte(high);
      *(v4u*)(lds + r * lds_pitch + c / 2) = mx_codes(v, s);
      lds_scales[r * blocks + c / 32] = (uint8_t)s;
    }
    __syncthreads();
  }

  v4f acc[MT][NT];
#pragma unroll
  for (int y = 0; y < MT; ++y)
#pragma unroll
    for (int z = 0; z < NT; ++z) acc[y][z] = v4f{0, 0, 0, 0};

  for (int g0 = 4 * wave; g0 < groups; g0 += 4 * kSplitWaves) {
    const int g = min(g0 + lane / 16, groups - 1);
    const bool in = g0 + lane / 16 < groups;  // what is beyond the last group counts as zeros
    v4i ca[MT][4], cb[NT][4];
    int sa[MT], sb[NT];
#pragma unroll
    for (int z = 0; z < NT; ++z) {
#pragma unroll
      for (int j = 0; j < 4; ++j) cb[z][j] = ldg<v4i, false>((const char*)pb[z] + (int64_t)g * 64 + j * 16);
      sb[z] = in ? ldg<int, false>((const char*)qb[z] + (int64_t)g * 4) : 0;
    }
#pragma unroll
    for (int y = 0; y < MT; ++y) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (FUSED) ca[y][j] = *(const v4i*)(pa[y] + g * 64 + j * 16);
        else ca[y][j] = ldg<v4i, false>((const char*)pa[y] + (int64_t)g * 64 + j * 16);
        if (!in) ca[y][j] = v4i{0, 0, 0, 0};
      }
      if constexpr (FUSED) sa[y] = *(const int*)(qa[y] + g * 4);
      else sa[y] = ldg<int, false>((const char*)qa[y] + (int64_t)g * 4);
      if (!in) sa[y] = 0;
    }
    auto step = [&](auto which) {
      constexpr int J = decltype(which)::value;
#pragma unroll
      for (int y = 0; y < MT; ++y)
#pragma unroll
        for (int z = 0; z < NT; ++z)
          acc[y][z] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(frag(ca[y][J]), frag(cb[z][J]), acc[y][z], 4, 4, J, sa[y],
                                                                      J, sb[z]);
    };
    step(Int<0>{});
    step(Int<1>{});
    step(Int<2>{});
    step(Int<3>{});
  }

  // The waves' sums in order.  Lane l has column l mod 16 and rows 4 * (l / 16) ... + 3 of each 16 x 16.
  if constexpr (FUSED) __syncthreads();  // the sums go where the quantised rows were
  v4f* sums = (v4f*)lds;
#pragma unroll
  for (int y = 0; y < MT; ++y)
#pragma unroll
    for (int z = 0; z < NT; ++z) sums[((wave * MT + y) * NT + z) * 64 + lane] = acc[y][z];
  __syncthreads();
  for (int t = wave; t < MT * NT; t += kSplitWaves) {
    v4f sum = sums[t * 64 + lane];
#pragma unroll
    for (int w = 1; w < kSplitWaves; ++w) sum += sums[(w * MT * NT + t) * 64 + lane];
    const int64_t i = i0 + t / NT * 16 + 4 * (lane / 16), j = j0 + t % NT * 16 + lane % 16;
    if (j >= n) continue;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < m) T::store((char*)out.p, (i + e) * out.stride + j, sum[e]);
  }
}

template <int MT, int NT, bool FUSED, typename X>
hipError_t run_split(MxMat a, Mat x, MxMat b, int64_t m, int64_t n, int64_t k, MatOut out, Elem dtype, hipStream_t stream) {
  const int groups = (int)groups_of(k);
  const size_t sums = (size_t)kSplitWaves * MT * NT * 1024, rows = FUSED ? (size_t)m * (groups * 68 + 16) : 0;
  const dim3 grid((unsigned)(ceil_div(m, 16 * MT) * ceil_div(n, 16 * NT))), block(64 * kSplitWaves);
  const auto kernel = dtype == Elem::f32 ? split_kernel<MT, NT, FUSED, X, F32> : split_kernel<MT, NT, FUSED, X, B16>;
  hipLaunchKernelGGL(kernel, grid, block, std::max(sums, rows), stream, a, x, b, m, n, k, groups, out);
  return hipGetLastError();
}

template <bool FUSED, typename X>
hipError_t pick_split(MxMat a, Mat x, MxMat b, int64_t m, int64_t n, int64_t k, MatOut out, Elem dtype, hipStream_t stream) {
  if (m <= 16) return run_split<1, 1, FUSED, X>(a, x, b, m, n, k, out, dtype, stream);
  if (m <= 32) return run_split<2, 1, FUSED, X>(a, x, b, m, n, k, out, dtype, stream);
  return run_split<4, 1, FUSED, X>(a, x, b, m, n, k, out, dtype, stream);
}

template <int F>
hipError_t run_tile(MxMat a, MxMat b, int64_t m, int64_t n, int64_t k, MatOut out, Elem dtype, hipStream_t stream) {
  const size_t tiles = ceil_div(m, 64 * F) * ceil_div(n, 64 * F);
  const auto kernel = dtype == Elem::f32 ? tile_kernel<F, F32> : tile_kernel<F, B16>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(ceil_div(tiles, 8) * 8)), dim3(kTileThreads), 0, stream, a, b, m, n,
                     (int)groups_of(k), out);
  return hipGetLastError();
}

// Rows that the fused form quantises in every workgroup: what 64 KB of LDS hold.
bool fused_fits(int64_t m, int64_t k) { return m <= 64 && m * (groups_of(k) * 68 + 16) <= 64 << 10; }

}  // namespace

size_t mx_matmul_workspace(int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_mx_matmul(MxMat a, MxMat b, int64_t m, int64_t n, int64_t k, MatOut out, Elem dtype, void*,
                            hipStream_t stream) {
  auto wgs = [&](int f) { return ceil_div(m, 64 * f) * ceil_div(n, 64 * f); };
  int pick = 0;
  if (m > 64 && n > 64 && k > 0) pick = wgs(4) >= 192 ? 4 : wgs(2) >= 192 ? 2 : wgs(1) >= 128 ? 1 : 0;
  if (pick == 4) return run_tile<4>(a, b, m, n, k, out, dtype, stream);
  if (pick == 2) return run_tile<2>(a, b, m, n, k, out, dtype, stream);
  if (pick == 1) return run_tile<1>(a, b, m, n, k, out, dtype, stream);
  return pick_split<false, F32>(a, {}, b, m, n, k, out, dtype, stream);
}

// Workspace of a linear that does not quantise on its way: the quantised rows, codes before scales.
size_t mx_linear_workspace(int64_t m, int64_t, int64_t k) { return fused_fits(m, k) ? 0 : (size_t)(m * groups_of(k)) * 68; }

hipError_t launch_mx_linear(Mat x, Elem x_dtype, MxMat w, int64_t m, int64_t n, int64_t k, MatOut out, Elem dtype,
                            void* workspace, hipStream_t stream) {
  if (fused_fits(m, k)) {
    return x_dtype == Elem::f32 ? pick_split<true, F32>({}, x, w, m, n, k, out, dtype, stream)
                                : pick_split<true, B16>({}, x, w, m, n, k, out, dtype, stream);
  }
  uint8_t* codes = (uint8_t*)workspace;
  uint8_t* scales = codes + m * groups_of(k) * 64;
  if (k > 0) {
    const hipError_t e = launch_mx_quantize(x, x_dtype, m, k, codes, scales, stream);
    if (e != hipSuccess) return e;
  }
  return launch_mx_matmul({codes, scales}, w, m, n, k, out, dtype, nullptr, stream);
}

}  // namespace pat
