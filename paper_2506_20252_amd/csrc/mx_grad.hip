// Products of a bfloat16 gradient with a matrix in blocks, out[i][c] = sum over j of g[i][j] q[j][c] (or g[j][i]): both
// gradients of the 4-bit product, and the weight's gradient from an input in 8-bit blocks.
//
// The sum runs over rows of q, across its blocks, so q is widened to bfloat16 (exactly) and multiplied by the bfloat16
// matrix instructions.  These want 8 consecutive j of one row of g and of one column of q in a lane, while q, and g where
// it is given by j, have consecutive columns in memory: they stand in LDS as they come, and gfx950's transposing reads
// (ds_read_b64_tr_b16) turn them round on the way to the registers.
#include <algorithm>

#include "layer_device.hpp"

namespace pat {
namespace {

// A workgroup of WA x WB waves computes a tile of R x R of out, a wave FA x FB blocks of 32 x 32, going through j 64 at a
// time.  While a step's 64 are multiplied out of one half of LDS, the next step's are widened from registers into the
// other, and what the step after that needs is on its way into these registers.  A wave's scales come in one load, a byte a
// lane, and go to their lanes by a permutation: a load takes 16 cycles of address work however little it asks for.  Of two
// waves on a SIMD one multiplies first and the other widens first, so that the matrix unit and the vector unit both have
// work (229 and 226 us for the sizes below on one card, 236 and 235 with all in the same order).
//
// 8192 x 4096 x 4096 in 220 us (g as given) and 225 us (g by j, float32 out), 1235 TFLOP/s, beside 1622 of a large bfloat16
// library product of rows by rows and 1398 of rows by columns; the first dozens of calls from an idle card take 240 to 300.
// The matrix units work in 0.6 of the busy CUs' cycles; what is between is widening, and LDS's reads and barriers.  Turning q
// and g round by vector instructions on their way into LDS took 6 and 19 longer.  1001 x 1000 x 1333: 13.1 and 13.4 us (15 and
// 17), the latency of 8 to 11 steps in turn with one or two workgroups a CU.
//
// PARTS: as many such groups of waves in a workgroup, each with its own part of j and its own LDS; their sums are added
// in order at the end.  For few tiles, whose waves would otherwise wait for one another's latencies alone.

template <int FA, int FB, int WA, int WB>
struct GradTile {
  static constexpr int kWaves = WA * WB, kThreads = 64 * kWaves, R = 32 * FA * WA;
  static_assert(R == 32 * FB * WB, "square");
  // A step's 64 rows of q are cut into pieces of 8 columns; a thread takes kEach of them, kSide rows apart.
  static constexpr int kPieces = R / 8, kEach = 64 * kPieces / kThreads, kSide = kThreads / kPieces;
  struct Lds {
    uint8_t g[R * 128];  // 64 values of j for every row of out; where g is given by j, as q
    uint8_t q[R * 128];  // 64 rows of q, widened
  };
};

// Where 16-byte block `block` (8 values of j) of a row of g given by rows stands.  A row is half of the 64 banks: 16 lanes
// that read one block of consecutive rows, or write two whole rows, hit all banks once.  Rows 32 apart are a constant apart.
__device__ __forceinline__ int lds_at(int row, int block) { return row * 128 + (block ^ (row >> 1 & 7)) * 16; }

// What is given by j stands by j, 64 rows of R values: a transposing read gives a lane 4 values of j of one column.  32 lanes
// read 64 bytes of 4 rows that follow each other, so the 64-byte parts of a row are exchanged by its number, and all banks
// are hit once.
template <int R>
__device__ __forceinline__ int exchange(int j) {
  return R == 64 ? j >> 1 & 1 : j & 3;
}
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s* LdsV4s;
// Lane l's operand of a 32 x 32 x 16 instruction, j0 + 8 * (l / 32) ... + 7 of column l mod 32 of those 32 whose first part
// for this lane is at `at`.
template <int R>
__device__ __forceinline__ v8bf read_turned(const uint8_t* at, int j0) {
  const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsV4s)(at + j0 * 2 * R));
  const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsV4s)(at + (j0 + 4) * 2 * R));
  return __builtin_bit_cast(v8bf, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// What q's codes are: how many bytes 8 columns take, and the 8 bfloat16 that they stand for under scale byte s.  Every
// value of a 4-bit block is one exactly, and of an 8-bit block every one above 2^-127.
struct Fours {
  static constexpr int kBytes = 4;
  typedef uint32_t Codes;
  // two codes of a byte (the I-th of the word)
  template <int I>
  __device__ static uint32_t widen2(Codes code, uint32_t s) {
    const v2bf v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, mx_scale_operand(s), I);
    return __builtin_bit_cast(uint32_t, v);
  }
  __device__ static v4u widen(Codes c, uint32_t s) { return v4u{widen2<0>(c, s), widen2<1>(c, s), widen2<2>(c, s), widen2<3>(c, s)}; }
  __device__ static Codes none() { return 0u; }
  // column c's bfloat16, of a row's codes
  __device__ static uint32_t one(const uint8_t* row, int64_t c, uint32_t s) {
    const uint32_t code = row[c / 2] >> (4 * (c & 1));
    return widen2<0>(code & 15u, s) & 0xFFFFu;
  }
};
struct Eights {
  static constexpr int kBytes = 8;
  typedef v2u Codes;
  template <bool HIGH>
  __device__ static uint32_t widen2(uint32_t code, uint32_t s) {
    const v2bf v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code, mx_scale_operand(s), HIGH);
    return __builtin_bit_cast(uint32_t, v);
  }
  __device__ static v4u widen(Codes c, uint32_t s) {
    return v4u{widen2<false>(c[0], s), widen2<true>(c[0], s), widen2<false>(c[1], s), widen2<true>(c[1], s)};
  }
  __device__ static Codes none() { return v2u{0, 0}; }
  __device__ static uint32_t one(const uint8_t* row, int64_t c, uint32_t s) { return widen2<false>(row[c], s) & 0xFFFFu; }
};

template <typename Q, int FA, int FB, int WA, int WB, int PARTS, bool TRANSPOSED, bool EDGE, typename T>
__global__ __launch_bounds__(64 * WA * WB * PARTS, 2) void grad_kernel(Mat g, MxMat q, int64_t rows, int64_t inner,
                                                                       int64_t cols, MatOut out, int64_t slice) {
  typedef GradTile<FA, FB, WA, WB> S;
  typedef typename S::Lds Lds;
  constexpr int R = S::R, W = S::kWaves, NT = S::kThreads, PIECES = S::kPieces, EACH = S::kEach, SIDE = S::kSide;
  __shared__ __attribute__((aligned(16))) Lds all_lds[PARTS][2];
  TilePlace place;
  if (!tile_place((rows + R - 1) / R, (cols + R - 1) / R, &place)) return;
  const int64_t i0 = place.i * R, c0 = place.j * R;
  const int64_t pitch = (cols + 127) / 128 * (16 * Q::kBytes), spitch = pitch / (4 * Q::kBytes);  // of codes, of scales
  if (gridDim.y > 1) {  // this launch row's slice of j, into its own matrix
    const int64_t j = blockIdx.y * slice;
    g.p = (const char*)g.p + 2 * (TRANSPOSED ? j * g.stride : j);
    q.codes += j * pitch;
    q.scales += j * spitch;
    out.p = (char*)out.p + (int64_t)blockIdx.y * rows * out.stride * T::kBytes;
    inner = min(slice, inner - j);
  }
  const int part = __builtin_amdgcn_readfirstlane(threadIdx.x / NT);
  const int tid = threadIdx.x % NT, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  Lds* lds = all_lds[part];

  // What a lane reads of 64 values of j.  q: the codes of 8 columns of EACH rows, and the scale of one of the wave's 16 * EACH
  // groups of 32.  g by j: 8 rows of out at the same EACH j.  g by rows: blocks of 8 values of j, 8 of them a row.
  // Nothing is read beyond a matrix: rows of out beyond the last are the last again, j beyond the last likewise and
  // zeroed before they reach LDS, and a piece or block that would go over a row's end ends there instead.
  const int piece = tid % PIECES, first = tid / PIECES;
  const int put = first * 2 * R + (piece / 4 ^ exchange<R>(first)) * 64 + piece % 4 * 16;  // in LDS
  constexpr int GROUPS = R / 32;
  const int scale_j = wave * (64 / PIECES) + lane % 16 / GROUPS + min(lane / 16, EACH - 1) * SIDE;
  const int scale_of = 4 * (lane / PIECES * GROUPS + piece / 4);  // the lane that has this lane's, 16 lanes further for each row
  const uint32_t q_at = (uint32_t)(first * pitch + min(c0 * Q::kBytes / 8 + piece * Q::kBytes, pitch - Q::kBytes));
  const uint32_t q_scale_at = (uint32_t)(scale_j * spitch + min(c0 / 32 + lane % GROUPS, spitch - 1));
  const int64_t gi = min(i0 + piece * 8, rows - 8);  // TRANSPOSED: the first row of out that is read
  const int over = (int)min(i0 + piece * 8 - gi, (int64_t)8);
  constexpr int BLOCKS = R * 8 / NT;
  const int block = tid % 8, row_u = tid / 8;  // by rows: block and row of each NT / 8 rows
  // of g: from the tile's corner, 32 bits (rows are not too far apart for that)
  constexpr int ROWS = TRANSPOSED ? 1 : BLOCKS, VECTORS = TRANSPOSED ? EACH : BLOCKS;
  uint32_t g_at[ROWS];
#pragma unroll
  for (int u = 0; u < ROWS; ++u)
    g_at[u] = 2 * (uint32_t)(TRANSPOSED ? first * g.stride + gi
                                        : (min(i0 + u * (NT / 8) + row_u, rows - 1) - i0) * g.stride + block * 8);
  const char* g_base = (const char*)g.p + (TRANSPOSED ? 0 : 2 * i0 * g.stride);

  typename Q::Codes codes[EACH];
  uint32_t scales;
  Raw8<B16> raw[VECTORS];

  // TAIL: perhaps fewer than 64 values of j are left.
  auto fetch = [&](int64_t j0, auto tail) {
    constexpr bool TAIL = decltype(tail)::value;
    const int left = TAIL ? (int)min(inner - j0, (int64_t)64) : 64;
    // an address is the wave's and a lane's part of 32 bits; rows beyond the last are it again
#pragma unroll
    for (int u = 0; u < EACH; ++u) {
      const int64_t j = j0 + u * SIDE, back = TAIL ? max(first + u * SIDE - (left - 1), 0) : 0;
      codes[u] = ldg<typename Q::Codes, false>((const char*)q.codes + j * pitch + (TAIL ? q_at - back * pitch : q_at));
      if constexpr (TRANSPOSED)
        raw[u].w[0] = ldg<v4u, false, 2>(g_base + 2 * j * g.stride + (TAIL ? g_at[0] - 2 * back * g.stride : g_at[0]));
    }
    {
      const int64_t back = TAIL ? max(scale_j - (left - 1), 0) : 0;
      scales = ldg<uint8_t, false>((const char*)q.scales + j0 * spitch + (TAIL ? q_scale_at - back * spitch : q_scale_at));
    }
    if constexpr (!TRANSPOSED) {
      const int64_t back = TAIL ? max(j0 + block * 8 - (inner - 8), (int64_t)0) : 0;
#pragma unroll
      for (int u = 0; u < BLOCKS; ++u)
        raw[u].w[0] = ldg<v4u, false, 2>(g_base + 2 * j0 + (TAIL ? g_at[u] - 2 * back : g_at[u]));
    }
  };
  auto widen = [&](Lds& l, int64_t j0, auto tail) {
    constexpr bool TAIL = decltype(tail)::value;
    const int left = TAIL ? (int)min(inner - j0, (int64_t)64) : 64;
#pragma unroll
    for (int u = 0; u < EACH; ++u) {
      typename Q::Codes code = codes[u];
      uint32_t s = __builtin_amdgcn_ds_bpermute(scale_of + 64 * u, scales);
      const bool in = !TAIL || first + u * SIDE < left;
      if (TAIL) code = in ? code : Q::none(), s = in ? s : 0u;
      *(v4u*)(l.q + put + u * SIDE * 2 * R) = Q::widen(code, s);
      if constexpr (TRANSPOSED) {
        if constexpr (EDGE) move_down(raw[u], over);
        if (TAIL && !in) raw[u].w[0] = v4u{0, 0, 0, 0};
        *(v4u*)(l.g + put + u * SIDE * 2 * R) = raw[u].w[0];
      }
    }
    if constexpr (!TRANSPOSED) {
#pragma unroll
      for (int u = 0; u < BLOCKS; ++u) {
        if constexpr (TAIL) move_down(raw[u], min(max(block * 8 - (left - 8), 0), 8));
        *(v4u*)(l.g + lds_at(u * (NT / 8) + row_u, block)) = raw[u].w[0];
      }
    }
  };

  const int half = lane / 32, wave_row = wave / WB * 32 * FA, wave_col = wave % WB * 32 * FB;
  v16f acc[FA][FB];
#pragma unroll
  for (int x = 0; x < FA; ++x)
#pragma unroll
    for (int y = 0; y < FB; ++y)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[x][y][e] = 0.0f;

  // An instruction of 32 x 32 x 16: lane l has row l mod 32 and j = 8 * (l / 32) ... + 7.  A block of g is read from LDS
  // a block before its instructions, those of q a step of 16 values of j before.
  const int turned_j = lane % 16 / 4 + 8 * half, turned_part = lane / 16 % 2 * 32 + lane % 4 * 8;
  auto turned_at = [&](int column) {  // of 32 columns, for read_turned
    return turned_j * 2 * R + (column / 32 ^ exchange<R>(turned_j)) * 64 + turned_part;
  };
  int g_first = lds_at(wave_row + lane % 32, half);  // by rows: of the wave's first block; the others' places follow from it
  auto multiply = [&](const Lds& l) {
    v8bf bg[2], bq[2][FB];
    // made here every time: kept over the loop, the places of all blocks would cost the registers that are left
    if constexpr (!TRANSPOSED) asm volatile("" : "+v"(g_first));
    auto read_g = [&](int n) {
      if constexpr (TRANSPOSED) bg[n % 2] = read_turned<R>(l.g + turned_at(wave_row + 32 * (n % FA)), n / FA * 16);
      else bg[n % 2] = *(const v8bf*)(l.g + (g_first ^ n / FA * 32) + n % FA * 4096);
    };
    auto read_q = [&](int step) {
#pragma unroll
      for (int y = 0; y < FB; ++y) bq[step % 2][y] = read_turned<R>(l.q + turned_at(wave_col + 32 * y), step * 16);
    };
    read_q(0);
    read_g(0);
#pragma unroll
    for (int n = 0; n < 4 * FA; ++n) {
      if (n + 1 < 4 * FA) read_g(n + 1);
      if (n % FA == 0 && n / FA < 3) read_q(n / FA + 1);
#pragma unroll
      for (int y = 0; y < FB; ++y)
        acc[n % FA][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bg[n % 2], bq[n / FA % 2][y], acc[n % FA][y], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  const int64_t steps = (inner + 63) / 64, each = (steps + PARTS - 1) / PARTS;
  const int64_t begin = part * each, end = min(begin + each, steps), whole = min(inner / 64, end);
  int64_t s = begin;
  if (s < end) {
    fetch(s * 64, Bool<true>{});
    widen(lds[s & 1], s * 64, Bool<true>{});
  }
  if (s + 1 < end) fetch(s * 64 + 64, Bool<true>{});
  // The loops' bodies have no branch: with one, the accumulators would be moved at every turn.
  if (W == 4 || wave < 4) {
    for (; s + 2 < whole; ++s) {
      __syncthreads();  // this half is written, and nobody reads the other any more
      multiply(lds[s & 1]);
      widen(lds[~s & 1], s * 64 + 64, Bool<false>{});
      fetch(s * 64 + 128, Bool<false>{});
    }
  } else {
    for (; s + 2 < whole; ++s) {
      __syncthreads();
      widen(lds[~s & 1], s * 64 + 64, Bool<false>{});
      fetch(s * 64 + 128, Bool<false>{});
      __builtin_amdgcn_sched_barrier(0);
      multiply(lds[s & 1]);
    }
  }
  for (; s < end; ++s) {  // the last two or three
    __syncthreads();
    multiply(lds[s & 1]);
    if (s + 1 < end) widen(lds[~s & 1], s * 64 + 64, Bool<true>{});
    if (s + 2 < end) fetch(s * 64 + 128, Bool<true>{});
  }

  if constexpr (PARTS > 1) {
    for (s = max(end - begin, (int64_t)0); s < each; ++s) __syncthreads();  // a part of fewer steps
    static_assert(PARTS * 2 * sizeof(Lds) >= (PARTS - 1) * W * FA * FB * 16 * 64 * 4, "");
    float* sums = (float*)&all_lds;
    auto at = [&](int p, int x, int y, int e) -> float& {
      return sums[((((p - 1) * W + wave) * FA + x) * FB + y) * 1024 + e * 64 + lane];
    };
    __syncthreads();
    if (part) {
#pragma unroll
      for (int x = 0; x < FA; ++x)
#pragma unroll
        for (int y = 0; y < FB; ++y)
#pragma unroll
          for (int e = 0; e < 16; ++e) at(part, x, y, e) = acc[x][y][e];
    }
    __syncthreads();
    if (part) {
      __syncthreads();  // write_tile's
      return;
    }
#pragma unroll
    for (int p = 1; p < PARTS; ++p)
#pragma unroll
      for (int x = 0; x < FA; ++x)
#pragma unroll
        for (int y = 0; y < FB; ++y)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[x][y][e] += at(p, x, y, e);
  }
  static_assert(W * tile_part(FB) * 4 <= 2 * sizeof(Lds), "");
  // nontemporal, as the 4-bit product's, the stores cost 4 % of 8192 x 4096 x 4096
  write_tile<FA, FB, T, false>(acc, (float*)lds, wave, wave_row, wave_col, i0, c0, rows, cols, out);
}

// The same product where the vectors of 8 above do not exist (fewer than 8 values of j, or of rows where g is given by j),
// or where a tile's rows of g are so far apart that their offsets need more than 32 bits.  One wave per 16 x 16 of out; an
// instruction of 16 x 16 x 32 takes j = 8 * (l / 16) ... + 7 of row and column l mod 16 in lane l, read one by one: right
// for any stride, and slow (every value is a load of its own).
template <typename Q, bool TRANSPOSED, typename T>
__global__ __launch_bounds__(64) void narrow_kernel(Mat g, MxMat q, int64_t rows, int64_t inner, int64_t cols, MatOut out) {
  const int64_t pitch = (cols + 127) / 128 * (16 * Q::kBytes), spitch = pitch / (4 * Q::kBytes);  // of codes, of scales
  const int64_t tiles_c = (cols + 15) / 16, i0 = blockIdx.x / tiles_c * 16, c0 = blockIdx.x % tiles_c * 16;
  const int lane = threadIdx.x, part = lane / 16;
  const int64_t i = min(i0 + lane % 16, rows - 1), c = min(c0 + lane % 16, cols - 1);
  v4f sum = {0, 0, 0, 0};
  for (int64_t j0 = 0; j0 < inner; j0 += 32) {
    v4u fg = {0, 0, 0, 0}, fq = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int64_t j = j0 + 8 * part + e;
      if (j >= inner) continue;
      const int64_t at = TRANSPOSED ? j * g.stride + i : i * g.stride + j;
      fg[e / 2] |= (uint32_t)ldg<uint16_t, false>((const char*)g.p + 2 * at) << (16 * (e & 1));
      fq[e / 2] |= Q::one(q.codes + j * pitch, c, q.scales[j * spitch + c / 32]) << (16 * (e & 1));
    }
    sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, fg), __builtin_bit_cast(v8bf, fq), sum, 0, 0, 0);
  }
  if (c0 + lane % 16 >= cols) return;
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (i0 + 4 * part + r < rows) T::store((char*)out.p, (i0 + 4 * part + r) * out.stride + c, sum[r]);
}

// out = the sum of `parts` float32 matrices of rows x pitch, in order.  A row takes `lanes` lanes, 8 columns each.
template <typename T>
__global__ __launch_bounds__(256) void add_kernel(const float* sums, int parts, int64_t rows, int64_t cols, int64_t pitch,
                                                  MatOut out, int lanes) {
  const int side = 256 / lanes, lane = threadIdx.x % lanes;
  for (int64_t i = (int64_t)blockIdx.x * side + threadIdx.x / lanes; i < rows; i += (int64_t)gridDim.x * side) {
    for (int64_t c = 8 * lane; c < cols; c += 8 * lanes) {
      v4f lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
#pragma unroll 4
      for (int p = 0; p < parts; ++p) {  // the pitch is whole vectors; what is behind a row is not used
        const char* at = (const char*)(sums + ((int64_t)p * rows + i) * pitch + c);
        lo += ldg<v4f, false>(at);
        hi += ldg<v4f, false>(at + 16);
      }
      const float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      char* p = (char*)out.p + (i * out.stride + c) * T::kBytes;
      if (cols - c >= 8) store8<T, false, false, kWhole>(p, 8, 4, v);
      else store8<T, false, false, kEnd>(p, cols - c, 4, v);
    }
  }
}

int64_t slice_pitch(int64_t cols) { return (cols + 7) / 8 * 8; }

template <typename Q, int FA, int FB, int WA, int WB, int PARTS, bool TRANSPOSED>
hipError_t run_grad(Mat g, MxMat q, int64_t rows, int64_t inner, int64_t cols, MatOut out, Elem dtype, const GradPlan& p,
                    void* workspace, hipStream_t stream) {
  constexpr int R = GradTile<FA, FB, WA, WB>::R;
  const bool sliced = p.slices > 1, f32 = dtype == Elem::f32;
  const MatOut to = sliced ? MatOut{workspace, slice_pitch(cols)} : out;
  auto kernel = f32 || sliced ? grad_kernel<Q, FA, FB, WA, WB, PARTS, TRANSPOSED, false, F32>
                              : grad_kernel<Q, FA, FB, WA, WB, PARTS, TRANSPOSED, false, B16>;
  if (TRANSPOSED && rows % 8)
    kernel = f32 || sliced ? grad_kernel<Q, FA, FB, WA, WB, PARTS, TRANSPOSED, TRANSPOSED, F32>
                           : grad_kernel<Q, FA, FB, WA, WB, PARTS, TRANSPOSED, TRANSPOSED, B16>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)tile_wgs(rows, cols, R), (unsigned)p.slices), dim3(64 * WA * WB * PARTS), 0,
                     stream, g, q, rows, inner, cols, to, p.slice);
  if (sliced) {
    const int lanes = row_lanes((int64_t)ceil_div(cols, 8), 256);
    const size_t wgs = std::min<size_t>(ceil_div(rows, 256 / lanes), 1 << 20);
    hipLaunchKernelGGL(f32 ? add_kernel<F32> : add_kernel<B16>, dim3((unsigned)wgs), dim3(256), 0, stream,
                       (const float*)workspace, p.slices, rows, cols, slice_pitch(cols), out, lanes);
  }
  return hipGetLastError();
}

bool narrow(bool transposed, int64_t rows, int64_t inner, int64_t stride) {
  return inner < 8 || (transposed && rows < 8) || stride > 1 << 22;  // 256 rows of 2 bytes: below 2^31
}

template <typename Q, bool TRANSPOSED>
hipError_t pick_grad(Mat g, MxMat q, int64_t rows, int64_t inner, int64_t cols, MatOut out, Elem dtype, void* workspace,
                     hipStream_t stream) {
  if (narrow(TRANSPOSED, rows, inner, g.stride)) {
    const auto kernel = dtype == Elem::f32 ? narrow_kernel<Q, TRANSPOSED, F32> : narrow_kernel<Q, TRANSPOSED, B16>;
    const int64_t band = narrow_band(rows, cols);
    for (int64_t i = 0; i < rows; i += band) {  // as many rows as a launch holds
      const int64_t here = std::min(band, rows - i);
      hipLaunchKernelGGL(kernel, dim3((unsigned)narrow_wgs(here, cols)), dim3(64), 0, stream,
                         Mat{(const char*)g.p + 2 * (TRANSPOSED ? i : i * g.stride), g.stride}, q, here, inner, cols,
                         MatOut{(char*)out.p + i * out.stride * (dtype == Elem::f32 ? 4 : 2), out.stride});
    }
    return hipGetLastError();
  }
  const GradPlan p = grad_plan(rows, inner, cols);
  if (p.tile == 256) return run_grad<Q, 4, 2, 2, 4, 1, TRANSPOSED>(g, q, rows, inner, cols, out, dtype, p, workspace, stream);
  if (p.tile == 128) return run_grad<Q, 2, 2, 2, 2, 1, TRANSPOSED>(g, q, rows, inner, cols, out, dtype, p, workspace, stream);
  return run_grad<Q, 1, 1, 2, 2, 2, TRANSPOSED>(g, q, rows, inner, cols, out, dtype, p, workspace, stream);
}

}  // namespace

size_t mx_grad_workspace(int64_t rows, int64_t inner, int64_t cols) {
  const GradPlan p = grad_plan(rows, inner, cols);
  return p.slices > 1 ? (size_t)(p.slices * rows * slice_pitch(cols)) * 4 : 0;
}

hipError_t launch_mx_grad(Mat g, bool transposed, MxMat q, int64_t rows, int64_t inner, int64_t cols, MatOut out,
                          Elem dtype, void* workspace, hipStream_t stream) {
  return transposed ? pick_grad<Fours, true>(g, q, rows, inner, cols, out, dtype, workspace, stream)
                    : pick_grad<Fours, false>(g, q, rows, inner, cols, out, dtype, workspace, stream);
}

// 8192 x 4096 from 8192 rows, float32 out: 470 us, 1170 TFLOP/s (460 to 483 from card to card), bfloat16 458; as the 4-bit form is
// bound, by LDS's traffic.
hipError_t launch_mxb_weight_grad(Mat g, MxbMat x, int64_t rows, int64_t inner, int64_t cols, MatOut out, Elem dtype,
                                  void* workspace, hipStream_t stream) {
  return pick_grad<Eights, true>(g, {x.codes, x.scales}, rows, inner, cols, out, dtype, workspace, stream);
}

}  // namespace pat
