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

// Waits until at most LATER of this wave's loads are on their way and all its reads of LDS are done, then for the other waves.
template <int LATER>
__device__ __forceinline__ void meet() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LATER) : "memory");
}

// Loads of 16 bytes a lane from base + at, and of 4 bytes from p, into LDS, lane after lane from `to` on.  Written out: the
// compiler's own ones make it wait for all of them before LDS is read, in every turn of the loop.  m0, which says where in LDS,
// is an operand: the compiler writes it and knows that it did.
__device__ __forceinline__ uint32_t lds_place(const uint8_t* to) {
  return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t*)to);
}
__device__ __forceinline__ void load_to_lds16(const uint8_t* base, uint32_t at, const uint8_t* to) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(lds_place(to)), "v"(at), "s"(base) : "memory");
}
__device__ __forceinline__ void load_to_lds4(const uint8_t* base, uint32_t at, const uint8_t* to) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %1, %2" ::"{m0}"(lds_place(to)), "v"(at), "s"(base) : "memory");
}
__device__ __forceinline__ void load_to_lds4(const uint8_t* p, const uint8_t* to) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %1, off" ::"{m0}"(lds_place(to)), "v"(p) : "memory");
}

// ---- tiles through LDS ---------------------------------------------------------------------------------------
//
// A workgroup of WN x WM waves computes a tile of N rows of the weight by M tokens, a wave FN x FM blocks of 32 x 32; of a
// gated tile's rows every wave has as many of either half, so that a and b of a value are the same lane's.  It goes through
// the terms 128 at a time.  What the step after the next multiplies is on its way into LDS, written there by the loads
// themselves: the tokens' 128 bytes a row, and with every other step the 128 bytes that hold 256 terms of the weight's rows
// (half lines would take twice the requests), and both sides' scales of 256 terms.
//
// LDS holds a row's eight 16-byte pieces at place piece ^ (row / 2 mod 8): a row is half of the 64 banks, so 16 lanes that
// read one piece of consecutive rows hit all banks once.  The loads write lane after lane, so each lane fetches the piece
// that belongs at its place.  An instruction of 32 x 32 x 64 takes two blocks of 32 terms: of the weight lane l has row
// l mod 32 and all of block l / 32, of the activations 16 terms of each.  Any two blocks will do as long as both sides
// take the same; the J-th instruction of a step takes the J-th and the J + 2-nd of its four, so that a lane's scales
// are two neighbouring bytes, of which the instruction picks the J-th.
//
// Bound by the matrix instructions' rate, of which the loads into LDS take a part.  8192 tokens, 2 x 8192 rows, 4096 terms in
// 404 us, 2.7 PFLOP/s, 8192^3 with a residual in 419, 2.6 (medians of one card; 381 to 406 and 406 to 420 from card to card): the
// instructions out of registers alone give 4.5 at the clock of short runs.  In 8 bits the former takes 418, with a
// checkpoint 474, in float32 462.  Measured for the former (418 us then): a wave of higher priority 540, scales packed 458,
// three steps on their way, the weight by half lines, 455, bands of 3, 4 or 8 tiles of tokens no faster, no loads at all 340.
// Each instruction followed by its share of the reads and loads, and the loads' waits counted, gave the last 8 %: issued together
// after the barrier they kept the instructions behind them waiting.  Two workgroups of 128 tokens a CU, the weight by half lines: 532.
template <int FN, int FM, int WN, int WM>
struct Tile {
  static constexpr int kWaves = WN * WM, N = 32 * FN * WN, M = 32 * FM * WM;
  struct Pair {  // 256 terms
    uint8_t codes[N * 128];
    uint8_t w_scales[N * 8], x_scales[M * 8];
  };
  struct Step {  // 128 terms
    uint8_t codes[M * 128];
  };
};

// Writes NB blocks of 32 columns, of one token a lane as the instructions leave them (lane l: token l mod 32, columns
// 8 * (c / 4) + 4 * (l / 32) + c mod 4), to columns j ... of tokens i ...: the wave turns them round in `part`, LDS of its own.
constexpr int turn_floats(int nb) { return 32 * (32 * nb + 4); }

template <int NB>
struct Turn {
  static constexpr int LANES = 4 * NB, ROWS = 64 / LANES, N = 32 / ROWS;  // lanes and tokens of an access, accesses
};
template <typename T>
__device__ __forceinline__ void add8(const Raw8<T>& r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t w = r.w[i * T::kBytes / 16][i * T::kBytes / 4 % 4];
    v[i] += T::kBytes == 4 ? __uint_as_float(w) : i & 1 ? bf16_hi(w) : bf16_lo(w);
  }
}

// INSIDE: all tokens and columns are there, and `added`, where it is not null, is what the residual has for them.
template <int NB, bool INSIDE, typename T, bool NT>
__device__ __forceinline__ void store_turned(const float (&v)[NB][16], const Raw8<T>* added, float* part, int64_t i, int64_t j, int64_t m,
                                             int64_t n, Mat residual, MatOut out) {
  constexpr int P = 32 * NB + 4, LANES = Turn<NB>::LANES, ROWS = Turn<NB>::ROWS;  // P: floats a token
  const int lane = threadIdx.x % 64, half = lane / 32, c = lane % LANES * 8;
  const int64_t left = n - j - c;
#pragma unroll
  for (int x = 0; x < NB; ++x)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      *(v4f*)(part + lane % 32 * P + 32 * x + 8 * e + 4 * half) = v4f{v[x][4 * e], v[x][4 * e + 1], v[x][4 * e + 2], v[x][4 * e + 3]};
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
  for (int u = 0; u < Turn<NB>::N; ++u) {
    const int token = u * ROWS + lane / LANES;
    const v4f lo = *(const v4f*)(part + token * P + c), hi = *(const v4f*)(part + token * P + c + 4);
    float r[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    char* p = (char*)out.p + ((i + token) * out.stride + j + c) * T::kBytes;
    if constexpr (INSIDE) {
      if (added) add8<T>(added[u], r);
      store8<T, false, NT, kWhole>(p, 8, 4, r);
    } else if (i + token < m && left > 0) {
      if (residual.p) {
        const char* q = (const char*)residual.p + ((i + token) * residual.stride + j + c) * T::kBytes;
        add8<T>(left >= 8 ? load_raw8<T, kWhole>(q, 0, 8) : load_raw8<T, kFew>(q, 0, left), r);
      }
      if (left >= 8) store8<T, false, NT, kWhole>(p, 8, 4, r);
      else store8<T, false, NT, kEnd>(p, left, 4, r);
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// One block of 32 columns from column j, of one token a lane, as above, in 8 bits: 16 bytes of codes a lane.
__device__ __forceinline__ void store_block(const float (&f)[16], int64_t i, int64_t j, int64_t m, int64_t n, MxbOut to) {
  const int half = threadIdx.x % 64 / 32;
  float v[16];
  uint32_t high = 0;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    v[e] = j + 8 * (e / 4) + 4 * half + e % 4 < n ? f[e] : 0.0f;
    high = max(high, __float_as_uint(v[e]) & 0x7FFFFFFFu);
  }
  const auto other = __builtin_amdgcn_permlane32_swap(high, high, false, false);
  const uint32_t s = mxb_scale_byte(max(other[0], other[1]));
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = mxb_codes(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3], s);
  // the halves have every other word of the block: the first two and the last two change hands
  const auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false), b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
  const int64_t groups = (n + 127) / 128;
  if (i >= m || j >= groups * 128) return;
  stg<false>((char*)to.codes + i * groups * 128 + j + 16 * half, v4u{a[0], a[1], b[0], b[1]});
  if (half == 0) stg<false>((char*)to.scales + i * groups * 4 + j / 32, (uint8_t)s);
}

// What a wave leaves of its FN x FM blocks: tokens i ... and columns j ... of the output.
template <int FN, int FM, bool GATED, typename O, bool NT>
__device__ __forceinline__ void leave(const v16f (&acc)[FN][FM], float* part, int64_t i, int64_t j, int64_t m, int64_t n, const Epilogue& ep) {
  static_assert(FN % 2 == 0, "");
  const int lane = threadIdx.x % 64;
  if constexpr (!GATED) {
    // Two blocks at a time, and the residual of as many twos at once as there are registers for.
    constexpr int TWOS = FN / 2 * FM, MOST = O::kBytes == 4 ? 2 : 4, ONCE = TWOS < MOST ? TWOS : MOST;
    static_assert(TWOS % ONCE == 0, "");
    auto put = [&](auto inside, const Raw8<O>* added, int two) {
      const int b = two / (FN / 2), a = two % (FN / 2) * 2;
      float v[2][16];
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int e = 0; e < 16; ++e) v[y][e] = acc[a + y][b][e];
      store_turned<2, decltype(inside)::value == 1, O, NT>(v, added, part, i + 32 * b, j + 32 * a, m, n, ep.residual, ep.out);
    };
    if (i + 32 * FM <= m && j + 32 * FN <= n) {
#pragma unroll
      for (int first = 0; first < TWOS; first += ONCE) {
        Raw8<O> added[ONCE][Turn<2>::N];
        if (ep.residual.p) {
#pragma unroll
          for (int u = 0; u < ONCE * Turn<2>::N; ++u) {
            const int two = first + u / Turn<2>::N;
            const int64_t row = i + two / (FN / 2) * 32 + u % Turn<2>::N * Turn<2>::ROWS + lane / Turn<2>::LANES;
            const int64_t col = j + two % (FN / 2) * 64 + lane % Turn<2>::LANES * 8;
            added[u / Turn<2>::N][u % Turn<2>::N] =
                load_raw8<O, kWhole>((const char*)ep.residual.p + (row * ep.residual.stride + col) * O::kBytes, 0, 8);
          }
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int u = 0; u < ONCE; ++u) put(Int<1>{}, added[u], first + u);
        } else {
#pragma unroll
          for (int u = 0; u < ONCE; ++u) put(Int<1>{}, nullptr, first + u);
        }
      }
    } else {
#pragma unroll
      for (int two = 0; two < TWOS; ++two) put(Int<0>{}, nullptr, two);
    }
  } else {
#pragma unroll
    for (int b = 0; b < FM; ++b, i += 32) {
      constexpr int H = FN / 2;
      float v[H][16];
#pragma unroll
      for (int a = 0; a < H; ++a) {
        float va[16], vb[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          va[e] = acc[a][b][e], vb[e] = acc[H + a][b][e];
          v[a][e] = activate(ep.act, va[e]) * vb[e];
        }
        if (ep.saved_a.codes) {
          store_block(va, i + lane % 32, j + 32 * a, m, n, ep.saved_a);
          store_block(vb, i + lane % 32, j + 32 * a, m, n, ep.saved_b);
        }
        if constexpr (O::kBytes == 1) store_block(v[a], i + lane % 32, j + 32 * a, m, n, ep.blocks);
      }
      if constexpr (O::kBytes > 1) store_turned<H, false, O, NT>(v, nullptr, part, i, j, m, n, {nullptr, 0}, ep.out);
    }
  }
}

template <int FN, int FM, int WN, int WM, bool GATED, typename O>
__global__ __launch_bounds__(64 * WN * WM, 2) void tile_kernel(MxbMat x, MxMat w, int64_t m, int64_t n, int groups, int64_t tiles_n,
                                                               Epilogue ep) {
  typedef Tile<FN, FM, WN, WM> S;
  typedef typename S::Pair Pair;
  typedef typename S::Step Step;
  constexpr int N = S::N, M = S::M, W = S::kWaves, COLS = GATED ? N / 2 : N;
  __shared__ __attribute__((aligned(16))) Pair pair0;
  __shared__ __attribute__((aligned(16))) Pair pair1;
  __shared__ __attribute__((aligned(16))) Step step0;
  __shared__ __attribute__((aligned(16))) Step step1;
  TilePlace place;
  if (!tile_place((m + M - 1) / M, tiles_n, &place)) return;
  const int64_t i0 = place.i * M, j0 = place.j * COLS;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint32_t w_pitch = groups * 64, x_pitch = groups * 128, s_pitch = groups * 4;

  // Rows beyond a matrix are its last row again; what they give is not stored.
  const int64_t jb = min(j0, n - 1);
  const int rows_w = (int)min((int64_t)COLS, n - jb), rows_x = (int)min((int64_t)M, m - i0);
  // Of a gated tile's row: its column, and (the same for 32 rows) whether it is of the second half.
  auto column = [&](int row) { return GATED ? row / (32 * FN) * (16 * FN) + row / 32 % (FN / 2) * 32 + row % 32 : row; };
  auto second = [&](int row) { return GATED && row / 32 % FN >= FN / 2; };
  constexpr int LOADS_W = N / 8 / W, LOADS_X = M / 8 / W;  // of codes, 8 rows each, a wave
  static_assert(LOADS_W * 8 * W == N && LOADS_X * 8 * W == M && W % 2 == 0, "");
  uint32_t at_w[LOADS_W], at_x[LOADS_X];  // of this lane's piece, in the rows' codes
  const int piece = (lane ^ (wave * 8 + lane / 8) / 2) % 8;
#pragma unroll
  for (int u = 0; u < LOADS_W; ++u) at_w[u] = (uint32_t)min(column((u * W + wave) * 8 + lane / 8), rows_w - 1) * w_pitch + piece * 16;
#pragma unroll
  for (int u = 0; u < LOADS_X; ++u) at_x[u] = (uint32_t)min((u * W + wave) * 8 + lane / 8, rows_x - 1) * x_pitch + piece * 16;
  // a wave loads the scales of 32 rows, two words each
  const int s_row = wave * 32 + lane / 2;
  static_assert(N / 32 == W && M / 32 == W, "");
  const uint32_t sat_w = (uint32_t)min(column(s_row), rows_w - 1) * s_pitch + lane % 2 * 4;
  const uint32_t sat_x = (uint32_t)min(s_row, rows_x - 1) * s_pitch + lane % 2 * 4;
  const uint8_t *codes_w = w.codes + jb * w_pitch, *scales_w = w.scales + jb * s_pitch;
  const uint8_t *codes_x = x.codes + i0 * x_pitch, *scales_x = x.scales + i0 * s_pitch;

  // A pair's loads: the weight's codes, both sides' scales.
  constexpr int LOADS_P = LOADS_W + 2, THIRD = LOADS_P / 3;
  static_assert(THIRD * 3 == LOADS_P, "");
  auto fetch_x = [&](Step& l, int g, int u) { load_to_lds16(codes_x + (int64_t)g * 128, at_x[u], l.codes + (u * W + wave) * 1024); };
  auto fetch_w = [&](Pair& l, int g, int u, uint32_t back, uint32_t sback) {
    if (u < LOADS_W) {
      const uint8_t* p = codes_w + (int64_t)g * 64 + (second((u * W + wave) * 8) ? n * w_pitch : 0);
      load_to_lds16(p, at_w[u] - back, l.codes + (u * W + wave) * 1024);
    } else if (u == LOADS_W) {
      load_to_lds4(scales_w + (int64_t)g * 4 + (second(wave * 32) ? n * s_pitch : 0), sat_w - sback, l.w_scales + wave * 256);
    } else {
      load_to_lds4(scales_x + (int64_t)g * 4, sat_x - sback, l.x_scales + wave * 256);
    }
  };

  const int half = lane / 32, wave_n = wave / WM * 32 * FN, wave_m = wave % WM * 32 * FM;
  const int row_w = wave_n + lane % 32, row_x = wave_m + lane % 32;
  v16f acc[FN][FM];
#pragma unroll
  for (int a = 0; a < FN; ++a)
#pragma unroll
    for (int b = 0; b < FM; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[a][b][e] = 0.0f;

  // What the next instructions multiply is read from LDS while these run, from one register set into the other.
  struct Blocks {
    v4i w[FN], x[FM][2];
  };
  struct Scales {
    int w[FN], x[FM];
  };
  auto read_scales = [&](const Pair& l, int h, Scales& s) {  // of the h-th group of the pair
#pragma unroll
    for (int a = 0; a < FN; ++a) s.w[a] = *(const uint16_t*)(l.w_scales + (row_w + 32 * a) * 8 + 4 * h + 2 * half);
#pragma unroll
    for (int b = 0; b < FM; ++b) s.x[b] = *(const uint16_t*)(l.x_scales + (row_x + 32 * b) * 8 + 4 * h + 2 * half);
  };
  // The i-th of the reads of what the j-th instructions multiply.  Places are formed anew in every step: kept for all pieces
  // they would take more registers than there are.
  constexpr int READS = FN + 2 * FM;
  const int swap = lane >> 1 & 7;
  int from_w = row_w * 128 + (2 * half ^ swap) * 16, from_x = row_x * 128 + (half ^ swap) * 16;
  auto read = [&](const Pair& p, const Step& l, int h, int j, int i, Blocks& c) {
    if (i < FN) c.w[i] = *(const v4i*)(p.codes + (from_w ^ (4 * h + j) * 16) + 32 * i * 128);
    else {
      const int b = (i - FN) / 2, k = (i - FN) % 2;
      c.x[b][k] = *(const v4i*)(l.codes + (from_x ^ (4 * k + 2 * j) * 16) + 32 * b * 128);
    }
  };
  // After each instruction comes its share of the loads.
  auto multiply = [&](const Blocks& c, const Scales& s, auto which, auto between) {
    constexpr int J = decltype(which)::value;
#pragma unroll
    for (int a = 0; a < FN; ++a)
#pragma unroll
      for (int b = 0; b < FM; ++b) {
        acc[a][b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(frag(c.w[a]), frag(c.x[b][0], c.x[b][1]), acc[a][b], 4, 0, J, s.w[a],
                                                                   J, s.x[b]);
        between(a * FM + b);
        __builtin_amdgcn_sched_barrier(0);
      }
  };
  constexpr int SLOTS = FN * FM;
  auto share = [&](int slot, int items, auto f) {
#pragma unroll
    for (int i = 0; i < items; ++i)
      if (i * SLOTS / items == slot) f(i);
  };
  // A row of the weight's blocks is read once the same of the blocks before is used up.
  auto read_share = [&](int slot, auto f) {
#pragma unroll
    for (int i = 0; i < READS; ++i)
      if ((i < FN ? min(i * FM + FM - 1, SLOTS - 2) : (i - FN) * SLOTS / (4 * FM)) == slot) f(i);
  };

  Blocks c0, c1;
  Scales s0, s1;
  // Step g, the H-th of pair `p`, out of `l`; the first instructions' blocks are in c0 and the scales in `s`.  Before the second
  // ones the next step has arrived and this step's LDS has been read by all, so both the next first blocks and what
  // comes two steps later come in under them, with a third of a pair.  A pair's thirds follow each other, the first in the place of
  // `p` once that is read, two in that of `other` under the next step's first and second instructions: for 1500 tokens by 4096 rows of
  // 4096 terms 30 us, 33 with halves under the second ones alone.  What came of the pair by the barrier after that is not
  // waited for there.  No branch: beyond the last it is fetched again.
  auto step = [&](Pair& p, Step& l, Pair& other, const Step& next_l, auto which, const Scales& s, Scales& next_s, int g) {
    constexpr int H = decltype(which)::value;
    asm volatile("" : "+v"(from_w), "+v"(from_x));
    const int gx = min(g + 2, groups - 1), gw = min(g + 2 + H, (groups - 1) / 2 * 2);
    const uint32_t back = gw + 1 < groups ? 0 : (piece >= 4 ? 64 : 0), sback = gw + 1 < groups ? 0 : lane % 2 * 4;
    multiply(c0, s, Int<0>{}, [&](int slot) {
      read_share(slot, [&](int i) { read(p, l, H, 1, i, c1); });
      if constexpr (H == 0) share(slot, THIRD, [&](int i) { fetch_w(other, gw, THIRD + i, back, sback); });
    });
    meet<H == 0 ? 2 * THIRD : 0>();
    const Pair& next_p = H ? other : p;
    multiply(c1, s, Int<1>{}, [&](int slot) {
      if (slot == 0) read_scales(next_p, 1 - H, next_s);
      read_share(slot, [&](int i) { read(next_p, next_l, 1 - H, 0, i, c0); });
      share(slot, LOADS_X + THIRD, [&](int i) {
        if (i < LOADS_X) fetch_x(l, gx, i);
        else fetch_w(H ? p : other, gw, (H ? 0 : 2 * THIRD) + i - LOADS_X, back, sback);
      });
    });
  };
  auto first = [&](Pair& l, int g, int begin, int end) {
    const uint32_t back = g + 1 < groups ? 0 : (piece >= 4 ? 64 : 0), sback = g + 1 < groups ? 0 : lane % 2 * 4;
#pragma unroll
    for (int u = begin; u < end; ++u) fetch_w(l, g, u, back, sback);
  };
  first(pair0, 0, 0, LOADS_P);
#pragma unroll
  for (int u = 0; u < LOADS_X; ++u) fetch_x(step0, 0, u);
  meet<0>();
#pragma unroll
  for (int u = 0; u < LOADS_X; ++u) fetch_x(step1, min(1, groups - 1), u);
  first(pair1, min(2, (groups - 1) / 2 * 2), 0, THIRD);
  read_scales(pair0, 0, s0);
#pragma unroll
  for (int i = 0; i < READS; ++i) read(pair0, step0, 0, 0, i, c0);
  int g = 0;
  for (; g + 4 <= groups; g += 4) {
    step(pair0, step0, pair1, step1, Int<0>{}, s0, s1, g);
    step(pair0, step1, pair1, step0, Int<1>{}, s1, s0, g + 1);
    step(pair1, step0, pair0, step1, Int<0>{}, s0, s1, g + 2);
    step(pair1, step1, pair0, step0, Int<1>{}, s1, s0, g + 3);
  }
  if (g < groups) step(pair0, step0, pair1, step1, Int<0>{}, s0, s1, g);
  if (g + 1 < groups) step(pair0, step1, pair1, step0, Int<1>{}, s1, s0, g + 1);
  if (g + 2 < groups) step(pair1, step0, pair0, step1, Int<0>{}, s0, s1, g + 2);

  // Results leave through LDS, whose last loads have to have come first.
  meet<0>();
  static_assert(sizeof(Pair) >= W / 2 * turn_floats(2) * 4, "");
  float* part = (wave < W / 2 ? (float*)&pair0 : (float*)&pair1) + wave % (W / 2) * turn_floats(2);
  leave<FN, FM, GATED, O, (N * M >= 256 * 256)>(acc, part, i0 + wave_m, j0 + (GATED ? wave_n / 2 : wave_n), m, n, ep);
}

// ---- small tiles -------------------------------------------------------------------------------------------------
//
// Where a tile is small its steps are latencies one after the other.  PARTS groups of WN x WM waves in a workgroup take a part of
// the terms each, in LDS of their own, and their sums are added in order at the end; D steps are in LDS or on their way
// at once.  The weight's rows come as half lines then, 64 bytes a step, at place piece ^ (row / 4 mod 4) of a row's four (a
// row is a quarter of the banks).  Every wave has the same number of loads a step, and waits for those of the next step alone.
// Bound by the loads' latency: 64 tokens by 4096 rows of 4096 terms in 8.9 us, 1001 by 2000 of 1333 in 6.6, of which starting,
// filling LDS and leaving take five.
template <int FN, int FM, int WN, int WM>
struct Stage {
  static constexpr int kWaves = WN * WM, N = 32 * FN * WN, M = 32 * FM * WM;
  uint8_t w[N * 64], x[M * 128];
  uint8_t scales[N * 4 + M * 4];  // the weight's, the tokens'
};

template <int FN, int FM, int WN, int WM, int PARTS, int D, bool GATED, typename O>
__global__ __launch_bounds__(64 * WN * WM * PARTS, WN * WM * PARTS == 8 ? 2 : 1) void deep_kernel(MxbMat x, MxMat w, int64_t m, int64_t n,
                                                                                                 int groups, int64_t tiles_n, Epilogue ep) {
  typedef Stage<FN, FM, WN, WM> S;
  constexpr int N = S::N, M = S::M, W = S::kWaves, COLS = GATED ? N / 2 : N;
  __shared__ __attribute__((aligned(16))) S all_lds[PARTS][D];
  TilePlace place;
  if (!tile_place((m + M - 1) / M, tiles_n, &place)) return;
  const int64_t i0 = place.i * M, j0 = place.j * COLS;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64 % W);
  const int part = __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * W));
  S* lds = all_lds[part];
  const uint32_t w_pitch = groups * 64, x_pitch = groups * 128, s_pitch = groups * 4;

  // Rows as tile_kernel has them.
  const int64_t jb = min(j0, n - 1);
  const int rows_w = (int)min((int64_t)COLS, n - jb), rows_x = (int)min((int64_t)M, m - i0);
  auto column = [&](int row) { return GATED ? row / (32 * FN) * (16 * FN) + row / 32 % (FN / 2) * 32 + row % 32 : row; };
  auto second = [&](int row) { return GATED && row / 32 % FN >= FN / 2; };
  constexpr int LOADS_W = N / 16 / W, LOADS_X = M / 8 / W;  // of codes, 16 and 8 rows each, a wave
  static_assert(LOADS_W * 16 * W == N && LOADS_X * 8 * W == M && W % 2 == 0, "");
  uint32_t at_w[LOADS_W], at_x[LOADS_X];  // of this lane's piece, in the rows' codes
  const int piece = (lane ^ (wave * 8 + lane / 8) / 2) % 8, piece_w = (lane ^ lane / 16) % 4;
#pragma unroll
  for (int u = 0; u < LOADS_W; ++u) at_w[u] = (uint32_t)min(column((u * W + wave) * 16 + lane / 4), rows_w - 1) * w_pitch + piece_w * 16;
#pragma unroll
  for (int u = 0; u < LOADS_X; ++u) at_x[u] = (uint32_t)min((u * W + wave) * 8 + lane / 8, rows_x - 1) * x_pitch + piece * 16;
  // a wave loads the scales of 64 rows of either side, or those of others again
  const int s_wave = wave % (N / 64 + M / 64);
  const bool s_of_w = s_wave < N / 64;
  const int s_row = (s_of_w ? s_wave : s_wave - N / 64) * 64 + lane;
  static_assert(N / 64 + M / 64 <= W, "");
  const uint8_t *codes_w = w.codes + jb * w_pitch, *codes_x = x.codes + i0 * x_pitch;
  const uint8_t* scales = s_of_w ? w.scales + (jb + (second(s_row) ? n : 0) + min(column(s_row), rows_w - 1)) * s_pitch
                                 : x.scales + (i0 + min(s_row, rows_x - 1)) * s_pitch;

  auto fetch = [&](S& l, int g) {
    load_to_lds4(scales + (int64_t)g * 4, l.scales + s_wave * 256);
#pragma unroll
    for (int u = 0; u < LOADS_W; ++u)
      load_to_lds16(codes_w + (int64_t)g * 64 + (second((u * W + wave) * 16) ? n * w_pitch : 0), at_w[u], l.w + (u * W + wave) * 1024);
#pragma unroll
    for (int u = 0; u < LOADS_X; ++u) load_to_lds16(codes_x + (int64_t)g * 128, at_x[u], l.x + (u * W + wave) * 1024);
  };
  constexpr int LOADS = 1 + LOADS_W + LOADS_X;

  const int half = lane / 32, wave_n = wave / WM * 32 * FN, wave_m = wave % WM * 32 * FM;
  const int row_w = wave_n + lane % 32, row_x = wave_m + lane % 32;
  v16f acc[FN][FM];
#pragma unroll
  for (int a = 0; a < FN; ++a)
#pragma unroll
    for (int b = 0; b < FM; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[a][b][e] = 0.0f;

  struct Blocks {
    v4i w[FN], x[FM][2];
  };
  struct Scales {
    int w[FN], x[FM];
  };
  auto read_scales = [&](const S& l, Scales& s) {
#pragma unroll
    for (int a = 0; a < FN; ++a) s.w[a] = *(const uint16_t*)(l.scales + (row_w + 32 * a) * 4 + 2 * half);
#pragma unroll
    for (int b = 0; b < FM; ++b) s.x[b] = *(const uint16_t*)(l.scales + (N + row_x + 32 * b) * 4 + 2 * half);
  };
  auto read = [&](const S& l, int j, Blocks& c) {
    auto at = [&](int piece) { return (piece ^ (lane >> 1 & 7)) * 16; };
#pragma unroll
    for (int a = 0; a < FN; ++a) c.w[a] = *(const v4i*)(l.w + (row_w + 32 * a) * 64 + ((2 * half + j) ^ (lane >> 2 & 3)) * 16);
#pragma unroll
    for (int b = 0; b < FM; ++b) {
      c.x[b][0] = *(const v4i*)(l.x + (row_x + 32 * b) * 128 + at(2 * j + half));
      c.x[b][1] = *(const v4i*)(l.x + (row_x + 32 * b) * 128 + at(4 + 2 * j + half));
    }
  };
  auto multiply = [&](const Blocks& c, const Scales& s, auto which) {
    constexpr int J = decltype(which)::value;
#pragma unroll
    for (int a = 0; a < FN; ++a)
#pragma unroll
      for (int b = 0; b < FM; ++b)
        acc[a][b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(frag(c.w[a]), frag(c.x[b][0], c.x[b][1]), acc[a][b], 4, 0, J, s.w[a],
                                                                   J, s.x[b]);
    __builtin_amdgcn_sched_barrier(0);
  };

  // This part's steps; all parts go through as many turns as the longest has.
  const int begin = (int)((int64_t)groups * part / PARTS), count = (int)((int64_t)groups * (part + 1) / PARTS) - begin;
  const int most = (groups + PARTS - 1) / PARTS, last = groups - 1;
  Blocks c0, c1;
  Scales s, next_s;
  // Step g out of `l`, its first instructions' blocks in c0 and its scales in s; beyond the last step it is fetched again.
  auto step = [&](S& l, const S& next, int g, bool mine) {
    read(l, 1, c1);
    if (mine) multiply(c0, s, Int<0>{});
    meet<(D - 2) * LOADS>();
    read_scales(next, next_s);
    read(next, 0, c0);
    fetch(l, min(begin + g + D, last));
    if (mine) multiply(c1, s, Int<1>{});
    s = next_s;
  };
#pragma unroll
  for (int d = 0; d < D; ++d) fetch(lds[d], min(begin + d, last));
  meet<(D - 1) * LOADS>();
  read_scales(lds[0], s);
  read(lds[0], 0, c0);
  int g = 0;
  for (; g + D <= groups / PARTS; g += D) {
#pragma unroll
    for (int d = 0; d < D; ++d) step(lds[d], lds[(d + 1) % D], g + d, true);
  }
#pragma unroll
  for (int d = 0; d < D; ++d)
    if (g + d < most) step(lds[d], lds[(d + 1) % D], g + d, g + d < count);

  // Results leave through LDS, whose last loads have to have come first.
  meet<0>();
  float* room = (float*)all_lds;
  if constexpr (PARTS > 1) {
    constexpr int SIZE = FN * FM * 16 * 64;  // floats of a wave's sums
    static_assert(sizeof(all_lds) >= (PARTS - 1) * W * SIZE * 4, "");
    auto sums = [&](int p, int a, int b, int e) -> v4f& {
      return *(v4f*)(room + ((p - 1) * W + wave) * SIZE + (((a * FM + b) * 4 + e) * 64 + lane) * 4);
    };
    if (part) {
#pragma unroll
      for (int a = 0; a < FN; ++a)
#pragma unroll
        for (int b = 0; b < FM; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            sums(part, a, b, e) = v4f{acc[a][b][4 * e], acc[a][b][4 * e + 1], acc[a][b][4 * e + 2], acc[a][b][4 * e + 3]};
    }
    __syncthreads();
    if (part) {
      __syncthreads();
      return;
    }
#pragma unroll
    for (int p = 1; p < PARTS; ++p)
#pragma unroll
      for (int a = 0; a < FN; ++a)
#pragma unroll
        for (int b = 0; b < FM; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const v4f v = sums(p, a, b, e);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[a][b][4 * e + i] += v[i];
          }
    __syncthreads();  // nobody reads the sums any more
  }
  static_assert(sizeof(all_lds) >= W * turn_floats(2) * 4, "");
  leave<FN, FM, GATED, O, false>(acc, room + wave * turn_floats(2), i0 + wave_m, j0 + (GATED ? wave_n / 2 : wave_n), m, n, ep);
}

typedef void (*Product)(MxbMat, MxMat, int64_t, int64_t, int, int64_t, Epilogue);

// `kernel` with the tiles of a plan, its shape S, in PARTS groups of waves.
template <int TILE, typename S, int PARTS>
hipError_t run_tiles(Product kernel, const ProductPlan& p, MxbMat x, MxMat w, int64_t m, int64_t n, int64_t k, const Epilogue& e,
                     hipStream_t stream) {
  static_assert(S::M == tile_tokens(TILE) && S::N == tile_rows(TILE) && 64 * S::kWaves * PARTS == tile_threads(TILE), "");
  hipLaunchKernelGGL(kernel, dim3((unsigned)p.wgs), dim3(p.threads), 0, stream, x, w, m, n, (int)groups_of(k), p.tiles_n, e);
  return hipGetLastError();
}

template <bool GATED, typename O>
hipError_t pick_tile(const ProductPlan& p, MxbMat x, MxMat w, int64_t m, int64_t n, int64_t k, const Epilogue& e, hipStream_t stream) {
  switch (p.tile) {
    case 256: return run_tiles<256, Tile<4, 2, 2, 4>, 1>(tile_kernel<4, 2, 2, 4, GATED, O>, p, x, w, m, n, k, e, stream);
    case 128: return run_tiles<128, Tile<2, 2, 2, 2>, 1>(tile_kernel<2, 2, 2, 2, GATED, O>, p, x, w, m, n, k, e, stream);
    case 64: return run_tiles<64, Stage<2, 1, 2, 2>, 1>(deep_kernel<2, 1, 2, 2, 1, 3, GATED, O>, p, x, w, m, n, k, e, stream);
    default: return run_tiles<32, Stage<2, 1, 1, 2>, 2>(deep_kernel<2, 1, 1, 2, 2, 3, GATED, O>, p, x, w, m, n, k, e, stream);
  }
}

// ---- few tokens ----------------------------------------------------------------------------------------------
//
// A workgroup computes 16 * MT tokens by 16 * H columns (gated: 16 * 2 H rows of the weight); its waves take 512 terms (four
// groups) in turn, a group an instruction of 16 x 16 x 128: lane l has row l mod 16 of either side, of the weight all of
// block l / 16, of the activations 16 values of block l / 32 and 16 of block 2 + l / 32, so that a load takes 64 bytes in a row of
// each of 16 rows.  Scales come a group's word a lane, in one load for the four groups, and are turned round between the lanes.
//
// Bound by the weight's bytes and one latency each of loading, joining and storing: one token by 2 x 8192 gated rows of 4096 terms
// (35.7 MB) in 8.8 us, by 8192 rows (17.8 MB) in 5.6; by 2 x 28672 of 8192 (250 MB) in 55, 4.6 TB/s.  A lane with 64 bytes in a row of
// the weight instead: 8.9, 5.7 and 56.

// Of four words of lanes l, l + 16, l + 32 and l + 48 the byte l / 16 of each, in order.
__device__ __forceinline__ int turn_bytes(int w) {
  const int quarter = threadIdx.x % 64 / 16;
  const auto a = __builtin_amdgcn_permlane16_swap(w, w, false, false);  // of quarters 0 and 2; of 1 and 3
  const int v = __builtin_amdgcn_perm(a[1], a[0], quarter & 1 ? 0x07030501 : 0x06020400);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);  // of quarters 0 and 1; of 2 and 3
  return __builtin_amdgcn_perm(b[1], b[0], quarter & 2 ? 0x07060302 : 0x05040100);
}

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
    px[y] = x.codes + i * 2 * pitch + quarter * 16;
    qx[y] = x.scales + i * (pitch / 16);
  }
#pragma unroll
  for (int z = 0; z < NT; ++z) {
    const int64_t j = min(j0 + 16 * (z % H) + lane % 16, n - 1) + (z < H ? 0 : n);
    pw[z] = w.codes + j * pitch + quarter * 16;
    qw[z] = w.scales + j * (pitch / 16);
  }

  v4f acc[MT][NT];
#pragma unroll
  for (int y = 0; y < MT; ++y)
#pragma unroll
    for (int z = 0; z < NT; ++z) acc[y][z] = v4f{0, 0, 0, 0};

  // A turn's loads, all before its first instruction: loads come back in their order, and what came after the weight's would
  // cost a latency of its own.  From 33 tokens on the registers do not suffice, and the second half of the tokens' comes later.
  // (The next turn's loads before this turn's instructions: no faster where the registers hold both.)
  constexpr int HALVES = MT * NT > 8 ? 2 : 1, J = 4 / HALVES;
  struct Turn {
    v4i x[MT][J][2], w[NT][4];
    int sw[NT], sx[MT];
  };
  auto load_x = [&](Turn& c, int g0, int j0) {  // beyond the last group that one again, not multiplied
#pragma unroll
    for (int y = 0; y < MT; ++y)
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const char* p = (const char*)px[y] + (int64_t)min(g0 + j0 + j, groups - 1) * 128;
        c.x[y][j][0] = ldg<v4i, false>(p);
        c.x[y][j][1] = ldg<v4i, false>(p + 64);
      }
  };
  auto load = [&](Turn& c, int g0) {
    const int g = min(g0 + quarter, groups - 1);
    load_x(c, g0, 0);
#pragma unroll
    for (int y = 0; y < MT; ++y) c.sx[y] = ldg<int, false>((const char*)qx[y] + (int64_t)g * 4);
#pragma unroll
    for (int z = 0; z < NT; ++z) c.sw[z] = ldg<int, false>((const char*)qw[z] + (int64_t)g * 4);
#pragma unroll
    for (int z = 0; z < NT; ++z)
#pragma unroll
      for (int j = 0; j < 4; ++j) c.w[z][j] = ldg<v4i, false>((const char*)pw[z] + (int64_t)min(g0 + j, groups - 1) * 64);
    __builtin_amdgcn_sched_barrier(0);
  };
  auto multiply = [&](Turn& c, int g0) {
#pragma unroll
    for (int z = 0; z < NT; ++z) c.sw[z] = turn_bytes(c.sw[z]);
#pragma unroll
    for (int y = 0; y < MT; ++y) c.sx[y] = turn_bytes(c.sx[y]);
    auto step = [&](auto which) {
      constexpr int I = decltype(which)::value;
      if constexpr (I == J) load_x(c, g0, J);
      if (g0 + I >= groups) return;
#pragma unroll
      for (int y = 0; y < MT; ++y)
#pragma unroll
        for (int z = 0; z < NT; ++z)
          acc[y][z] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(frag(c.w[z][I]), frag(c.x[y][I % J][0], c.x[y][I % J][1]), acc[y][z],
                                                                      4, 0, I, c.sw[z], I, c.sx[y]);
    };
    step(Int<0>{});
    step(Int<1>{});
    step(Int<2>{});
    step(Int<3>{});
  };
  for (int g0 = 4 * wave; g0 < groups; g0 += 4 * kFewWaves) {
    Turn c;
    load(c, g0);
    multiply(c, g0);
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
hipError_t run_few(const ProductPlan& p, MxbMat x, MxMat w, int64_t m, int64_t n, int64_t k, Epilogue e, hipStream_t stream) {
  const int64_t groups = groups_of(k), out_groups = groups_of(n), band = p.band;
  for (int64_t i = 0; i < m; i += band) {  // as many rows as a launch holds
    const int64_t here = std::min(band, m - i);
    hipLaunchKernelGGL((few_kernel<MT, H, GATED, O>), dim3((unsigned)(ceil_div(here, 16 * MT) * p.tiles_n)), dim3(p.threads),
                       (size_t)kFewWaves * MT * H * (GATED ? 2 : 1) * 1024, stream, x, w, here, n, (int)groups, p.tiles_n, e);
    x.codes += band * groups * 128, x.scales += band * groups * 4;
    for (MxbOut* q : {&e.blocks, &e.saved_a, &e.saved_b})
      if (q->codes) q->codes += band * out_groups * 128, q->scales += band * out_groups * 4;
    if (e.out.p) e.out.p = (char*)e.out.p + band * e.out.stride * O::kBytes;
    if (e.residual.p) e.residual.p = (const char*)e.residual.p + band * e.residual.stride * O::kBytes;
  }
  return hipGetLastError();
}

template <int MT, typename O>
hipError_t pick_few(const ProductPlan& p, MxbMat x, MxMat w, int64_t m, int64_t n, int64_t k, const Epilogue& e, hipStream_t stream) {
  switch (p.columns) {
    case 1: return run_few<MT, 1, false, O>(p, x, w, m, n, k, e, stream);
    case 2: return run_few<MT, 2, false, O>(p, x, w, m, n, k, e, stream);
    default: return run_few<MT, 4, false, O>(p, x, w, m, n, k, e, stream);
  }
}

template <typename O>
hipError_t linear(MxbMat x, MxMat w, int64_t m, int64_t n, int64_t k, const Epilogue& e, hipStream_t stream) {
  const ProductPlan p = product_plan(m, n, k, false, false);
  if (p.tile) return pick_tile<false, O>(p, x, w, m, n, k, e, stream);
  if (p.tokens == 1) return pick_few<1, O>(p, x, w, m, n, k, e, stream);
  if (p.tokens == 2) return pick_few<2, O>(p, x, w, m, n, k, e, stream);
  return pick_few<3, O>(p, x, w, m, n, k, e, stream);
}

template <typename O>
hipError_t gated(MxbMat x, MxMat w, int64_t m, int64_t n, int64_t k, const Epilogue& e, hipStream_t stream) {
  const ProductPlan p = product_plan(m, n, k, true, O::kBytes == 1 || e.saved_a.codes);
  if (p.tile) return pick_tile<true, O>(p, x, w, m, n, k, e, stream);
  if (p.tokens == 1) return run_few<1, 2, true, O>(p, x, w, m, n, k, e, stream);
  return run_few<2, 2, true, O>(p, x, w, m, n, k, e, stream);
}

}  // namespace

hipError_t launch_mxb_product(MxbMat x, MxMat w, int64_t m, int64_t n, int64_t k, const Epilogue& e, hipStream_t stream) {
  const bool f32 = e.dtype == Elem::f32;
  if (!e.gated) return f32 ? linear<F32>(x, w, m, n, k, e, stream) : linear<B16>(x, w, m, n, k, e, stream);
  if (!e.out.p) return gated<Q8>(x, w, m, n, k, e, stream);
  return f32 ? gated<F32>(x, w, m, n, k, e, stream) : gated<B16>(x, w, m, n, k, e, stream);
}

}  // namespace pat
