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
// A workgroup of WA x WB waves computes a tile of R x R of the output, a wave FA x FB blocks of 32 x 32.  It goes
// through the columns 256 at a time (two groups, 128 bytes of codes a row).  The next 256 columns of both sides are
// on their way into the other half of LDS, written there by the loads themselves, while these are multiplied.
//
// LDS holds a row's eight 16-byte blocks of codes at place block ^ (row / 2 mod 8): a row is half of the 64 banks, so
// 16 lanes that read one block of consecutive rows hit all banks once.  The loads write lane after lane, so each lane
// fetches the block that belongs at its place.  An instruction of 32 x 32 x 64 takes two blocks of 32 rows: lane l has
// row l mod 32 and one block, and any two blocks will do as long as both sides take the same.  Lane half h takes blocks
// 2h and 2h + 1 of a group in turn, whose scales are two neighbouring bytes: the instruction picks the byte.
//
// 8192 x 8192 x 8192: 265 us, 4.15 PFLOP/s (the first dozens of calls from an idle card up to 345), where the instructions
// alone take 160 for these columns, the loads alone 190 (45 GB/s a CU: 12 % of what is read from L2 is not there) and the
// reads of LDS nearly the cycles of the instructions; 25 us are each tile's first loads and its stores.  Four waves of 128 x 128 take as long as these eight.
// Slower: four groups of 128 columns in LDS (330: pieces of 64 bytes), a barrier of its own for the release of LDS (290
// beside 277).

template <int FA, int FB, int WA, int WB>
struct Tile {
  static constexpr int kWaves = WA * WB, R = 32 * FA * WA;
  static_assert(R == 32 * FB * WB, "square");
  struct Lds {
    uint8_t codes[2][R * 128];  // [a, b]
    uint8_t scales[2][R * 8];
  };
};

template <int FA, int FB, int WA, int WB, typename T>
__global__ __launch_bounds__(64 * WA * WB, 2) void tile_kernel(MxMat a, MxMat b, int64_t m, int64_t n, int groups,
                                                               MatOut out) {
  typedef Tile<FA, FB, WA, WB> S;
  typedef typename S::Lds Lds;
  constexpr int R = S::R, W = S::kWaves;
  // Two objects, and not an array: the compiler then knows that the loads into one do not touch the other.
  __shared__ __attribute__((aligned(16))) Lds lds0;
  __shared__ __attribute__((aligned(16))) Lds lds1;
  TilePlace place;
  if (!tile_place((m + R - 1) / R, (n + R - 1) / R, &place)) return;
  const int64_t i0 = place.i * R, j0 = place.j * R;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint32_t pitch = groups * 64, spitch = groups * 4;

  // Rows beyond a matrix are its last row again; what they give is not stored.
  const int rows_a = (int)min((int64_t)R, m - i0), rows_b = (int)min((int64_t)R, n - j0);
  constexpr int LOADS = R / 8 / W;  // of codes, 8 rows each, a wave
  uint32_t at_a[LOADS], at_b[LOADS];  // of this lane's block, in the rows' codes
  const int block = (lane ^ (wave * 8 + lane / 8) / 2) % 8;
#pragma unroll
  for (int u = 0; u < LOADS; ++u) {
    const int row = (u * W + wave) * 8 + lane / 8;
    at_a[u] = (uint32_t)min(row, rows_a - 1) * pitch + block * 16;
    at_b[u] = (uint32_t)min(row, rows_b - 1) * pitch + block * 16;
  }
  constexpr bool SCALES_OF_ALL = R / 32 >= W;  // a wave loads the scales of 32 rows; small tiles have fewer than waves
  static_assert(R / 32 <= W, "");
  const int srow = wave * 32 + lane / 2;
  const uint32_t sat_a = (uint32_t)min(srow, rows_a - 1) * spitch + lane % 2 * 4;
  const uint32_t sat_b = (uint32_t)min(srow, rows_b - 1) * spitch + lane % 2 * 4;
  const uint8_t *codes_a = a.codes + i0 * pitch, *codes_b = b.codes + j0 * pitch;
  const uint8_t *scales_a = a.scales + i0 * spitch, *scales_b = b.scales + j0 * spitch;

  auto fetch = [&](Lds& l, int g) {
    // the second group of the last 256 columns may not exist: the first again, not multiplied
    const uint32_t back = g + 1 < groups ? 0 : (block >= 4 ? 64 : 0), sback = g + 1 < groups ? 0 : lane % 2 * 4;
    const uint8_t *pa = codes_a + (int64_t)g * 64, *pb = codes_b + (int64_t)g * 64;
#pragma unroll
    for (int u = 0; u < LOADS; ++u) {
      __builtin_amdgcn_global_load_lds((GlobalWords)(pa + (at_a[u] - back)), (LdsWords)(l.codes[0] + (u * W + wave) * 1024),
                                       16, 0, 0);
      __builtin_amdgcn_global_load_lds((GlobalWords)(pb + (at_b[u] - back)), (LdsWords)(l.codes[1] + (u * W + wave) * 1024),
                                       16, 0, 0);
    }
    if (SCALES_OF_ALL || wave < R / 32) {
      const uint8_t *qa = scales_a + (int64_t)g * 4, *qb = scales_b + (int64_t)g * 4;
      __builtin_amdgcn_global_load_lds((GlobalWords)(qa + (sat_a - sback)), (LdsWords)(l.scales[0] + wave * 256), 4, 0, 0);
      __builtin_amdgcn_global_load_lds((GlobalWords)(qb + (sat_b - sback)), (LdsWords)(l.scales[1] + wave * 256), 4, 0, 0);
    }
  };

  const int half = lane / 32, wave_row = wave / WB * 32 * FA, wave_col = wave % WB * 32 * FB;
  const int row_a = wave_row + lane % 32, row_b = wave_col + lane % 32;
  v16f acc[FA][FB];
#pragma unroll
  for (int x = 0; x < FA; ++x)
#pragma unroll
    for (int y = 0; y < FB; ++y)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[x][y][e] = 0.0f;

  // A step is one block of every row: FA x FB instructions.  What the next step multiplies is read from LDS while these
  // run, from one register set into the other.
  struct Blocks {
    v4i a[FA], b[FB];
  };
  struct Scales {
    v2u a[FA], b[FB];
  };
  auto read_scales = [&](const Lds& l, Scales& s) {
#pragma unroll
    for (int x = 0; x < FA; ++x) s.a[x] = *(const v2u*)(l.scales[0] + (row_a + 32 * x) * 8);
#pragma unroll
    for (int y = 0; y < FB; ++y) s.b[y] = *(const v2u*)(l.scales[1] + (row_b + 32 * y) * 8);
  };
  auto read = [&](const Lds& l, int step, Blocks& c) {  // step: 2 * group + which of the half's two blocks
    const int at = ((step / 2 * 4 + half * 2 + step % 2) ^ (lane >> 1 & 7)) * 16;
#pragma unroll
    for (int x = 0; x < FA; ++x) c.a[x] = *(const v4i*)(l.codes[0] + (row_a + 32 * x) * 128 + at);
#pragma unroll
    for (int y = 0; y < FB; ++y) c.b[y] = *(const v4i*)(l.codes[1] + (row_b + 32 * y) * 128 + at);
  };
  auto multiply = [&](const Blocks& c, const Scales& s, auto which) {
    constexpr int STEP = decltype(which)::value, J = STEP % 2;
    int fa[FA], fb[FB];
#pragma unroll
    for (int x = 0; x < FA; ++x) fa[x] = s.a[x][STEP / 2] >> (16 * half);
#pragma unroll
    for (int y = 0; y < FB; ++y) fb[y] = s.b[y][STEP / 2] >> (16 * half);
#pragma unroll
    for (int x = 0; x < FA; ++x)
#pragma unroll
      for (int y = 0; y < FB; ++y)
        acc[x][y] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(frag(c.a[x]), frag(c.b[y]), acc[x][y], 4, 4, J, fa[x], J,
                                                                   fb[y]);
    // a step's instructions stay together: moved over each other, all steps' blocks would be in registers at once
    __builtin_amdgcn_sched_barrier(0);
  };

  const int tiles = (groups + 1) / 2, pairs = groups / 4;  // 256 columns each; whole ones, two by two
  Blocks c0, c1;
  Scales s0, s1;
  // Tile t out of `l`; the first step's blocks are in c0 and the scales in `s`.  Before the last step's
  // multiplications the next tile has arrived and this half of LDS has been read by all, so both the next first
  // step and the tile after the next come in under them.  No branch: beyond the last tile it is fetched again.
  auto columns = [&](Lds& l, Lds& next, const Scales& s, Scales& s_next, int t) {
    read(l, 1, c1);
    multiply(c0, s, Int<0>{});
    read(l, 2, c0);
    multiply(c1, s, Int<1>{});
    read(l, 3, c1);
    multiply(c0, s, Int<2>{});
    __syncthreads();
    read_scales(next, s_next);
    read(next, 0, c0);
    fetch(l, 2 * min(t + 2, tiles - 1));
    multiply(c1, s, Int<3>{});
  };
  fetch(lds0, 0);
  __syncthreads();
  fetch(lds1, 2 * min(1, tiles - 1));
  read_scales(lds0, s0);
  read(lds0, 0, c0);
  for (int p = 0; p < pairs; ++p) {
    columns(lds0, lds1, s0, s1, 2 * p);
    columns(lds1, lds0, s1, s0, 2 * p + 1);
  }
  // up to three groups are left, in both halves
  if (groups % 4) {
    read(lds0, 1, c1);
    multiply(c0, s0, Int<0>{});
    multiply(c1, s0, Int<1>{});
    if (groups % 4 >= 2) {
      read(lds0, 2, c0);
      read(lds0, 3, c1);
      multiply(c0, s0, Int<2>{});
      multiply(c1, s0, Int<3>{});
    }
    if (groups % 4 == 3) {
      __syncthreads();
      read_scales(lds1, s1);
      read(lds1, 0, c0);
      read(lds1, 1, c1);
      multiply(c0, s1, Int<0>{});
      multiply(c1, s1, Int<1>{});
    }
  }

  // What the large tiles write is more than the caches hold beside the codes: nontemporal, 8192 x 8192 x 8192 takes 299 us
  // with its quantisation and 325 otherwise.
  write_tile<FA, FB, T, R == 256>(acc, wave < W / 2 ? (float*)&lds0 : (float*)&lds1, wave % (W / 2), wave_row, wave_col, i0, j0, m, n, out);
}

// ---- few rows ------------------------------------------------------------------------------------------------
//
// A workgroup computes 16 * MT rows by 16 * NT columns; its waves take 512 columns (four groups) in turn.  An
// instruction of 16 x 16 x 128 takes four blocks of 16 rows; lane l takes row l mod 16 and, of the four groups, group
// l / 16: 64 consecutive bytes of codes in four instructions, whose four scales are one word.
//
// FUSED: the rows of a are still x, float32 or bfloat16.  The workgroup quantises all of them into LDS first; every
// workgroup repeats that, which is little beside its part of b as long as the rows are few.
//
// Bound by the reading of b: one row of 8192 columns by 8192 rows of b (36 MB) in 9.3 us, of which 3 are a launch of
// anything; 24 quantised rows of 4001 by 5000 (11 MB) in 7.

template <int MT, int NT, bool FUSED, typename X, typename T>
__global__ __launch_bounds__(64 * kSplitWaves) void split_kernel(MxMat a, Mat x, MxMat b, int64_t m, int64_t n, int64_t k,
                                                                  int groups, Divisor per_row, MatOut out) {
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

  if constexpr (FUSED) {  // as quantize_kernel does it: 8 values a lane, 4 lanes a block, 16 a group
    constexpr int U = 2, T512 = 64 * kSplitWaves;
    const int total = (int)m * groups * 16, sub = threadIdx.x % 16;
    for (int base = 0; base < total; base += T512 * U) {
      auto take = [&](auto cover) {
        constexpr Cover C = decltype(cover)::value;
        Raw8<X> r[U];
        int row[U], c[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const uint32_t i = min(base + u * T512 + (int)threadIdx.x, total - 1), q = per_row.divide(i);
          row[u] = q;
          c[u] = (i - q * per_row.d) * 8;
          r[u] = load_raw8<X, C>((const char*)x.p + row[u] * x.stride * X::kBytes, c[u], k);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          settle<C>(r[u], c[u], k);
          const uint32_t s = mx_scale_byte(max_of_4(high_bits(r[u])));
          if (base + u * T512 + (int)threadIdx.x >= total) continue;  // whole groups of 16 lanes
          *(uint32_t*)(lds + row[u] * lds_pitch + c[u] / 2) = mx_codes(r[u], s);
          if (sub % 4 == 0) lds_scales[row[u] * groups * 4 + c[u] / 32] = (uint8_t)s;
        }
      };
      if (k % 8 == 0) take(CoverOf<kWhole>{});
      else if (k >= 8) take(CoverOf<kEnd>{});
      else take(CoverOf<kFew>{});
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
  const dim3 grid((unsigned)split_wgs(m, n)), block(64 * kSplitWaves);
  const auto kernel = dtype == Elem::f32 ? split_kernel<MT, NT, FUSED, X, F32> : split_kernel<MT, NT, FUSED, X, B16>;
  hipLaunchKernelGGL(kernel, grid, block, std::max(sums, rows), stream, a, x, b, m, n, k, groups,
                     Divisor((uint32_t)groups * 16), out);
  return hipGetLastError();
}

template <int MT, bool FUSED, typename X>
hipError_t pick_columns(MxMat a, Mat x, MxMat b, int64_t m, int64_t n, int64_t k, MatOut out, Elem dtype, hipStream_t stream) {
  switch (split_columns(n)) {
    case 1: return run_split<MT, 1, FUSED, X>(a, x, b, m, n, k, out, dtype, stream);
    case 2: return run_split<MT, 2, FUSED, X>(a, x, b, m, n, k, out, dtype, stream);
    default: return run_split<MT, 4, FUSED, X>(a, x, b, m, n, k, out, dtype, stream);
  }
}

template <bool FUSED, typename X>
hipError_t pick_split(MxMat a, Mat x, MxMat b, int64_t m, int64_t n, int64_t k, MatOut out, Elem dtype, hipStream_t stream) {
  switch (split_rows(m)) {
    case 1: return pick_columns<1, FUSED, X>(a, x, b, m, n, k, out, dtype, stream);
    case 2: return pick_columns<2, FUSED, X>(a, x, b, m, n, k, out, dtype, stream);
    default: return pick_columns<4, FUSED, X>(a, x, b, m, n, k, out, dtype, stream);
  }
}

template <int FA, int FB, int WA, int WB>
hipError_t run_tile(MxMat a, MxMat b, int64_t m, int64_t n, int64_t k, MatOut out, Elem dtype, hipStream_t stream) {
  constexpr int R = Tile<FA, FB, WA, WB>::R;
  const auto kernel = dtype == Elem::f32 ? tile_kernel<FA, FB, WA, WB, F32> : tile_kernel<FA, FB, WA, WB, B16>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)tile_wgs(m, n, R)), dim3(64 * WA * WB), 0, stream, a, b, m, n,
                     (int)groups_of(k), out);
  return hipGetLastError();
}

// Rows that every workgroup quantises for itself, and not a launch before: m * k up to 32768 values (us fused and not,
// k = 4096: 4.5 and 5.8 for one row, 5.1 and 6.6 for 4, 8.6 and 7.3 for 16; k = 8192: 8.1 and 10.7, 10.4 and 11.6,
// none and 12.6).  What they take in LDS stays below 32 KB.  No more rows than the split takes of a product whose rows
// are quantised before: the sums are then the same either way.
bool fused(int64_t m, int64_t k) { return k > 0 && m <= kSplitRows && m * k <= 32768; }

}  // namespace

hipError_t launch_mx_matmul(MxMat a, MxMat b, int64_t m, int64_t n, int64_t k, MatOut out, Elem dtype, hipStream_t stream) {
  // without columns all are zero: the gradient's sum of no terms, which takes outputs of any size
  if (k == 0) return launch_mx_grad({nullptr, 0}, false, {nullptr, nullptr}, m, 0, n, out, dtype, nullptr, stream);
  switch (product_tile(m, n)) {
    case 256: return run_tile<4, 2, 2, 4>(a, b, m, n, k, out, dtype, stream);
    case 128: return run_tile<2, 2, 2, 2>(a, b, m, n, k, out, dtype, stream);
    case 64: return run_tile<1, 1, 2, 2>(a, b, m, n, k, out, dtype, stream);
  }
  return pick_split<false, F32>(a, {}, b, m, n, k, out, dtype, stream);
}

// Workspace of a linear that does not quantise on its way: the quantised rows, codes before scales.
size_t mx_linear_workspace(int64_t m, int64_t, int64_t k) { return fused(m, k) ? 0 : (size_t)(m * groups_of(k)) * 68; }

hipError_t launch_mx_linear(Mat x, Elem x_dtype, MxMat w, int64_t m, int64_t n, int64_t k, MatOut out, Elem dtype,
                            void* workspace, hipStream_t stream) {
  if (fused(m, k)) {
    return x_dtype == Elem::f32 ? pick_split<true, F32>({}, x, w, m, n, k, out, dtype, stream)
                                : pick_split<true, B16>({}, x, w, m, n, k, out, dtype, stream);
  }
  uint8_t* codes = (uint8_t*)workspace;
  uint8_t* scales = codes + m * groups_of(k) * 64;
  if (k > 0) {
    const hipError_t e = launch_mx_quantize(x, x_dtype, m, k, codes, scales, stream);
    if (e != hipSuccess) return e;
  }
  return launch_mx_matmul({codes, scales}, w, m, n, k, out, dtype, stream);
}

}  // namespace pat
