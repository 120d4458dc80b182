// Products of a bfloat16 gradient with a 4-bit matrix, out[i][c] = sum over j of g[i][j] q[j][c] (or g[j][i]): both
// gradients of the 4-bit product.
//
// The sum runs over rows of q, across its blocks, so q is widened to bfloat16 (exactly) and multiplied by the bfloat16
// matrix instructions.  These want 8 consecutive j of one row of g and of one column of q in a lane: a lane reads an
// 8 x 8 patch of q (a word of codes from each of 8 rows), widens it and writes it to LDS turned round, one column of
// 8 values at a time; likewise g where it is given by j.
#include "ops_device.hpp"

namespace pat {
namespace {

// A workgroup of 2 x 2 waves computes 64 * F rows by 64 * F columns, a wave F x F blocks of 32 x 32, going through j 64
// at a time.  What the next 64 need is read into registers before these are multiplied, and widened into the other
// half of LDS after.
constexpr int kGradThreads = 256;

template <int F>
struct GradLds {
  static constexpr int kRows = 64 * F;
  uint8_t g[kRows * 128];  // rows of out: 64 values of j
  uint8_t q[kRows * 128];  // columns of out: 64 values of j
};

// Where 16-byte block `block` (8 values of j) of a row stands: lanes that read one block of consecutive rows, and
// lanes that write one block of every 8th row, both hit different banks.
__device__ __forceinline__ int lds_at(int row, int block) { return row * 128 + ((block ^ row ^ row >> 3) & 7) * 16; }

// Turns 8 rows of 8 bfloat16 round: out[c] holds column c's 8 values.
__device__ __forceinline__ void turn(const v4u (&rows)[8], v4u (&cols)[8]) {
#pragma unroll
  for (int c = 0; c < 8; ++c)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      cols[c][r] = __builtin_amdgcn_perm(rows[2 * r + 1][c / 2], rows[2 * r][c / 2], c & 1 ? 0x07060302u : 0x05040100u);
}

// Eight bfloat16 moved down by d places (0 to 8), zeros behind them.
__device__ __forceinline__ v4u move_down(v4u v, int d) {
  uint64_t lo = v[0] | (uint64_t)v[1] << 32, hi = v[2] | (uint64_t)v[3] << 32;
  if (d >= 4) lo = hi, hi = 0, d -= 4;
  if (d >= 4) lo = 0, d = 0;
  if (d > 0) lo = lo >> 16 * d | hi << (64 - 16 * d), hi >>= 16 * d;
  return v4u{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}

// The 8 codes of a word as 8 bfloat16.
__device__ __forceinline__ v4u widen8(uint32_t code, uint32_t s) {
  const float scale = mx_scale_value(s);
  auto pair = [&](v2bf v) { return __builtin_bit_cast(uint32_t, v); };
  const v4u v = {pair(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 0)),
                 pair(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 1)),
                 pair(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 2)),
                 pair(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 3))};
  return s == 255u ? v4u{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u} : v;
}

template <int F, bool TRANSPOSED, typename T>
__global__ __launch_bounds__(kGradThreads, F == 4 ? 1 : 2) void grad_kernel(Mat g, MxMat q, int64_t rows, int64_t inner,
                                                                             int64_t cols, MatOut out) {
  constexpr int R = 64 * F;
  __shared__ __attribute__((aligned(16))) GradLds<F> lds[2];
  TilePlace place;
  if (!tile_place((rows + R - 1) / R, (cols + R - 1) / R, &place)) return;
  const int64_t i0 = place.i * R, c0 = place.j * R;
  const int64_t pitch = (cols + 127) / 128 * 64;
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;

  // What a lane reads of 64 values of j.  q: a patch of 8 x 8, the columns' patches side by side over the lanes.
  // g by rows: blocks of 8 values, 8 of them a row.  g by j: a patch like q's.
  // Nothing is read beyond a matrix: rows of out beyond the last are the last again, j beyond the last likewise and
  // zeroed before they reach LDS, and a block or patch that would go over a row's end ends there instead.
  const int patch_c = tid % (R / 8), patch_j = tid / (R / 8);
  const bool has_patch = F == 4 || patch_j < 8;               // R patches in all: fewer than lanes below F = 4
  const int64_t qc = min(c0 + patch_c * 8, pitch * 2 - 8);    // in the stored form, which is whole groups wide
  const char* q_codes = (const char*)q.codes + qc / 2;
  const char* q_scales = (const char*)q.scales + qc / 32;
  const int64_t gi = min(i0 + patch_c * 8, rows - 8);         // TRANSPOSED: the patch's first row of out
  const int to_row = (int)(gi - i0);                          // its place in the tile, negative for a short last tile
  constexpr int ROWS = TRANSPOSED ? 1 : 2 * F;
  const char* g_row[ROWS];
#pragma unroll
  for (int u = 0; u < ROWS; ++u)
    g_row[u] = (const char*)g.p + 2 * (TRANSPOSED ? gi : min(i0 + u * 32 + tid / 8, rows - 1) * g.stride);

  uint32_t code[8], scale[8];
  v4u raw[TRANSPOSED ? 8 : 2 * F];

  // TAIL: fewer than 64 values of j are left.
  auto fetch = [&](int64_t j0, auto tail) {
    constexpr bool TAIL = decltype(tail)::value;
    const int left = TAIL ? (int)(inner - j0) : 64;
    if (has_patch) {
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const uint32_t j = TAIL ? min(patch_j * 8 + r, left - 1) : patch_j * 8 + r;
        code[r] = ldg<uint32_t, false>(q_codes + j0 * pitch + j * (uint32_t)pitch);
        scale[r] = ldg<uint8_t, false>(q_scales + j0 * (pitch / 16) + j * (uint32_t)(pitch / 16));
        if constexpr (TRANSPOSED) raw[r] = ldg<v4u, false, 2>(g_row[0] + 2 * j0 * g.stride + 2 * (uint64_t)j * g.stride);
      }
    }
    if constexpr (!TRANSPOSED) {
      const int64_t at = TAIL ? min(j0 + tid % 8 * 8, inner - 8) : j0 + tid % 8 * 8;
#pragma unroll
      for (int u = 0; u < 2 * F; ++u) raw[u] = ldg<v4u, false, 2>(g_row[u] + 2 * at);
    }
  };
  auto place_lds = [&](GradLds<F>& l, int64_t j0, auto tail) {
    if constexpr (decltype(tail)::value) {
      const int left = (int)(inner - j0);
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const bool in = patch_j * 8 + r < left;
        code[r] = in ? code[r] : 0u;
        scale[r] = in ? scale[r] : 0u;
        if constexpr (TRANSPOSED) raw[r] = in ? raw[r] : v4u{0, 0, 0, 0};
      }
      if constexpr (!TRANSPOSED) {
        const int d = min(max(tid % 8 * 8 - (left - 8), 0), 8);
#pragma unroll
        for (int u = 0; u < 2 * F; ++u) raw[u] = move_down(raw[u], d);
      }
    }
    if (has_patch) {
      v4u wide[8], turned[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) wide[r] = widen8(code[r], scale[r]);
      turn(wide, turned);
#pragma unroll
      for (int c = 0; c < 8; ++c) *(v4u*)(l.q + lds_at(patch_c * 8 + c, patch_j)) = turned[c];
      if constexpr (TRANSPOSED) {
        turn(raw, turned);
#pragma unroll
        for (int c = 0; c < 8; ++c)
          if (to_row + c >= 0) *(v4u*)(l.g + lds_at(to_row + c, patch_j)) = turned[c];
      }
    }
    if constexpr (!TRANSPOSED) {
#pragma unroll
      for (int u = 0; u < 2 * F; ++u) *(v4u*)(l.g + lds_at(u * 32 + tid / 8, tid % 8)) = raw[u];
    }
  };

  const int row_g = wave / 2 * 32 * F + lane % 32, row_q = wave % 2 * 32 * F + lane % 32, half = lane / 32;
  v16f acc[F][F];
#pragma unroll
  for (int x = 0; x < F; ++x)
#pragma unroll
    for (int y = 0; y < F; ++y)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[x][y][e] = 0.0f;

  // An instruction of 32 x 32 x 16: lane l has row l mod 32 and j = 8 * (l / 32) ... + 7.
  auto multiply = [&](const GradLds<F>& l) {
#pragma unroll
    for (int step = 0; step < 4; ++step) {
      v8bf fg[F], fq[F];
#pragma unroll
      for (int x = 0; x < F; ++x) {
        fg[x] = *(const v8bf*)(l.g + lds_at(row_g + 32 * x, step * 2 + half));
        fq[x] = *(const v8bf*)(l.q + lds_at(row_q + 32 * x, step * 2 + half));
      }
#pragma unroll
      for (int x = 0; x < F; ++x)
#pragma unroll
        for (int y = 0; y < F; ++y) acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fg[x], fq[y], acc[x][y], 0, 0, 0);
    }
  };

  // The loop's body has no branch: with one, the accumulators would be moved at every turn.
  const int64_t full = inner / 64;
  int at = 0;
  if (full) {
    fetch(0, Bool<false>{});
    place_lds(lds[0], 0, Bool<false>{});
  }
  for (int64_t step = 1; step < full; ++step, at ^= 1) {
    fetch(step * 64, Bool<false>{});
    __syncthreads();  // this half is written, and nobody reads the other any more
    multiply(lds[at]);
    place_lds(lds[at ^ 1], step * 64, Bool<false>{});
  }
  if (inner % 64) {
    fetch(full * 64, Bool<true>{});
    if (full) {
      __syncthreads();
      multiply(lds[at]);
      at ^= 1;
    }
    place_lds(lds[at], full * 64, Bool<true>{});
  }
  __syncthreads();
  multiply(lds[at]);

  // Lane l has column l mod 32 of a block and rows 8 * (e / 4) + 4 * (l / 32) + e mod 4.
#pragma unroll
  for (int x = 0; x < F; ++x) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int64_t i = i0 + wave / 2 * 32 * F + 32 * x + 8 * (e / 4) + 4 * half + e % 4;
      if (i >= rows) continue;
      char* p = (char*)out.p + (i * out.stride + c0) * T::kBytes;
#pragma unroll
      for (int y = 0; y < F; ++y)
        if (c0 + row_q + 32 * y < cols) T::store(p, row_q + 32 * y, acc[x][y][e]);
    }
  }
}

// The same product where the vectors of 8 above do not exist: fewer than 8 values of j, or of rows where g is given by
// j.  One wave per 16 x 16 of out; an instruction of 16 x 16 x 32 takes j = 8 * (l / 16) ... + 7 of row and column
// l mod 16 in lane l, read one by one.
template <bool TRANSPOSED, typename T>
__global__ __launch_bounds__(64) void narrow_kernel(Mat g, MxMat q, int64_t rows, int64_t inner, int64_t cols, MatOut out) {
  const int64_t pitch = (cols + 127) / 128 * 64;
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
      const uint32_t code = q.codes[j * pitch + c / 2] >> (4 * (c & 1)), s = q.scales[j * (pitch / 16) + c / 32];
      fq[e / 2] |= (widen8(code & 15u, s)[0] & 0xFFFFu) << (16 * (e & 1));
    }
    sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, fg), __builtin_bit_cast(v8bf, fq), sum, 0, 0, 0);
  }
  if (c0 + lane % 16 >= cols) return;
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (i0 + 4 * part + r < rows) T::store((char*)out.p, (i0 + 4 * part + r) * out.stride + c, sum[r]);
}

template <int F, bool TRANSPOSED>
hipError_t run_grad(Mat g, MxMat q, int64_t rows, int64_t inner, int64_t cols, MatOut out, Elem dtype, hipStream_t stream) {
  const size_t tiles = ceil_div(rows, 64 * F) * ceil_div(cols, 64 * F);
  const auto kernel = dtype == Elem::f32 ? grad_kernel<F, TRANSPOSED, F32> : grad_kernel<F, TRANSPOSED, B16>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(ceil_div(tiles, 8) * 8)), dim3(kGradThreads), 0, stream, g, q, rows, inner,
                     cols, out);
  return hipGetLastError();
}

template <bool TRANSPOSED>
hipError_t pick_grad(Mat g, MxMat q, int64_t rows, int64_t inner, int64_t cols, MatOut out, Elem dtype, hipStream_t stream) {
  if (inner < 8 || (TRANSPOSED && rows < 8)) {
    const auto kernel = dtype == Elem::f32 ? narrow_kernel<TRANSPOSED, F32> : narrow_kernel<TRANSPOSED, B16>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(ceil_div(rows, 16) * ceil_div(cols, 16))), dim3(64), 0, stream, g, q, rows,
                       inner, cols, out);
    return hipGetLastError();
  }
  auto wgs = [&](int f) { return ceil_div(rows, 64 * f) * ceil_div(cols, 64 * f); };
  if (wgs(4) >= 192) return run_grad<4, TRANSPOSED>(g, q, rows, inner, cols, out, dtype, stream);
  if (wgs(2) >= 192) return run_grad<2, TRANSPOSED>(g, q, rows, inner, cols, out, dtype, stream);
  return run_grad<1, TRANSPOSED>(g, q, rows, inner, cols, out, dtype, stream);
}

}  // namespace

size_t mx_grad_workspace(int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_mx_grad(Mat g, bool transposed, MxMat q, int64_t rows, int64_t inner, int64_t cols, MatOut out,
                          Elem dtype, void*, hipStream_t stream) {
  return transposed ? pick_grad<true>(g, q, rows, inner, cols, out, dtype, stream)
                    : pick_grad<false>(g, q, rows, inner, cols, out, dtype, stream);
}

}  // namespace pat
