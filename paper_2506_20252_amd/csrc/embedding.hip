// Embedding lookup with scaling, and its dense gradient by sorted tokens.
#include <algorithm>

#include "ops_device.hpp"

namespace pat {
namespace {

__device__ __forceinline__ int64_t load_token(const char* tokens, int token_bytes, int64_t t) {
  return token_bytes == 4 ? (int64_t)ldg<int32_t, false>(tokens + 4 * t) : ldg<int64_t, false>(tokens + 8 * t);
}

// A token's table row, or -1 where the table does not hold it.  The subtraction is modulo 2^64: a token
// below `first` becomes a number above every row count.
__device__ __forceinline__ int64_t token_row(const char* tokens, int token_bytes, int64_t t, int64_t first, int64_t rows) {
  const uint64_t row = (uint64_t)load_token(tokens, token_bytes, t) - (uint64_t)first;
  return row < (uint64_t)rows ? (int64_t)row : -1;
}

// A row is taken by `lanes` lanes, 8 columns each at a time; a workgroup holds 256 / lanes tokens side by side and
// TOKENS of them in turn, whose table rows a lane reads before it writes any.
//
// Bound by memory: 65536 random tokens of 4096 bfloat16 columns, a table of 32768 rows, in 156 us: 649 MB if each row were
// read once, 837 MB counted (a row that comes again is mostly gone from the caches), 5.4 TB/s.
template <int TOKENS, typename TI, typename TO>
__global__ __launch_bounds__(256) void lookup_kernel(const char* tokens, int token_bytes, int64_t ntokens, Mat table,
                                                     int64_t first, int64_t rows, int64_t cols, float scale, MatOut out,
                                                     int lanes) {
  constexpr bool SPLIT = Split<TI, TO>::value;
  const int side = 256 / lanes, lane = threadIdx.x % lanes;
  const int64_t step = (int64_t)side * TOKENS, gap = lane_gap<SPLIT>(lanes);
  for (int64_t t0 = blockIdx.x * step + threadIdx.x / lanes; t0 < ntokens; t0 += gridDim.x * step) {
    int64_t row[TOKENS];
#pragma unroll
    for (int u = 0; u < TOKENS; ++u) {
      const int64_t t = t0 + u * side;
      row[u] = t < ntokens ? token_row(tokens, token_bytes, t, first, rows) : -1;
    }
    auto columns = [&](int64_t c, auto cover) {
      constexpr Cover C = decltype(cover)::value;
      float v[TOKENS][8];
#pragma unroll
      for (int u = 0; u < TOKENS; ++u)  // a token that the table does not hold reads row 0 and is zeroed below
        load8<TI, SPLIT, false, C>((const char*)table.p + (max(row[u], (int64_t)0) * table.stride + c) * TI::kBytes,
                                   rows ? cols - c : 0, gap, v[u]);
#pragma unroll
      for (int u = 0; u < TOKENS; ++u) {
        const int64_t t = t0 + u * side;
        if (t >= ntokens) break;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[u][i] = row[u] < 0 ? 0.0f : v[u][i] * scale;
        store8<TO, SPLIT, true, C>((char*)out.p + (t * out.stride + c) * TO::kBytes, cols - c, gap, v[u]);
      }
    };
    for (int64_t c = lane_column<SPLIT>(lane); c < cols; c += 8 * lanes) {
      const Cover cover = rows ? cover_of(cols - c, gap, cols) : kFew;  // a table without rows is not read
      if (cover == kWhole) columns(c, CoverOf<kWhole>{});
      else if (cover == kEnd) columns(c, CoverOf<kEnd>{});
      else columns(c, CoverOf<kFew>{});
    }
  }
}

// ---- gradient of few tokens, in one launch ----------------------------------------------------------------
//
// A workgroup of 16 waves takes `each` rows a wave in turn and reads all tokens itself, one a lane.  Those of its rows
// are listed in order; then a wave adds up its rows one by one, or writes zeros.  A row with far more than its share of
// the list is added up by all waves, a section of the list each, and the waves' sums in order.
//
// Bound by latency: a load of tokens, a load of rows of g after it, and a launch: 5.4 us for 1001 tokens of 333 columns all
// over 1251 rows, of which 3 are a launch of anything (sorted first, in three launches: 19).  7.4 to 7.7 where a token comes
// more often, 64 times.

constexpr int kFewWaves = 16, kFewMostEach = 8;
static_assert(kFewTokens == 64 * kFewWaves, "a token a lane");

struct FewArgs {
  const char* tokens;
  int token_bytes, ntokens, each;
  int64_t first, rows, cols;
  Mat g;
  MatOut out;
  float scale;
};

template <typename TI, typename TO>
__global__ __launch_bounds__(kFewTokens) void few_kernel(FewArgs a) {
  constexpr bool SPLIT = Split<TI, TO>::value;
  __shared__ uint32_t list[kFewTokens];  // the token's number, and its row in the bits above
  __shared__ int32_t totals[kFewWaves], counts[kFewWaves * kFewMostEach], crowd[8], crowds;
  __shared__ float part[kFewWaves][8 * 64];
  const int t = threadIdx.x, lane = t % 64, wave = __builtin_amdgcn_readfirstlane(t / 64), here = kFewWaves * a.each;
  const int64_t gap = lane_gap<SPLIT>(64);
  for (int64_t r0 = (int64_t)blockIdx.x * here; r0 < a.rows; r0 += (int64_t)gridDim.x * here) {
    if (t < here) counts[t] = 0;
    if (t == 0) crowds = 0;
    __syncthreads();
    const int64_t r = t < a.ntokens ? token_row(a.tokens, a.token_bytes, t, a.first, a.rows) - r0 : -1;
    const bool listed = r >= 0 && r < here;
    const uint64_t ours = __ballot(listed);
    if (listed) atomicAdd(&counts[r], 1);
    if (lane == 0) totals[wave] = __popcll(ours);
    __syncthreads();
    int at = 0, n = 0;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
      if (w == wave) at = n;
      n += totals[w];
    }
    n = __builtin_amdgcn_readfirstlane(n);
    if (listed) list[at + __popcll(ours & (((uint64_t)1 << lane) - 1))] = (uint32_t)(t | (int)r << 10);
    // more than an eighth of the list (seven rows at most), and more than a wave adds up before all have met: a row of 32
    // tokens 7.0 us so and 10.2 by one wave, one of 16 tokens 7.3 and 7.1
    const int many = 16 + n / 8;
    if (t < here && counts[t] > many) crowd[atomicAdd(&crowds, 1)] = t;
    __syncthreads();

    auto columns = [&](int64_t c, auto cover) {
      constexpr Cover C = decltype(cover)::value;
      const int64_t left = a.cols - c;
      // adds a row's entries of list[from, to) to `sum`, in order, U loads at a time
      auto add = [&](int row, int from, int to, float (&sum)[8]) {
        constexpr int U = C == kFew ? 4 : 8;
        for (int i = from; i < to; i += 64) {
          const uint32_t entry = i + lane < to ? list[i + lane] : 0xFFFFFFFFu;
          uint64_t mine = __ballot((int)(entry >> 10) == row);
          while (mine) {
            const int have = min(__popcll(mine), U);
            float v[U][8];
            int src = 0;
#pragma unroll
            for (int u = 0; u < U; ++u) {
              src = mine ? __builtin_ctzll(mine) : src;  // beyond the last the last again, not added
              mine &= mine - 1;
              const int64_t token = __builtin_amdgcn_readlane(entry, src) & (kFewTokens - 1);
              load8<TI, SPLIT, false, C>((const char*)a.g.p + (token * a.g.stride + c) * TI::kBytes, left, gap, v[u]);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
              if (u >= have) break;
#pragma unroll
              for (int j = 0; j < 8; ++j) sum[j] += v[u][j];
            }
          }
        }
      };
      auto write = [&](int row, float (&sum)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] *= a.scale;
        store8<TO, SPLIT, true, C>((char*)a.out.p + ((r0 + row) * a.out.stride + c) * TO::kBytes, left, gap, sum);
      };
      for (int row = wave; row < here && r0 + row < a.rows; row += kFewWaves) {
        const int count = __builtin_amdgcn_readfirstlane(counts[row]);
        if (count > many) continue;
        float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (count) add(row, 0, n, sum);
        write(row, sum);
      }
      const int rest = __builtin_amdgcn_readfirstlane(crowds), section = (n + kFewWaves - 1) / kFewWaves;
      for (int x = 0; x < rest; ++x) {
        const int row = __builtin_amdgcn_readfirstlane(crowd[x]);
        float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        add(row, wave * section, min(n, (wave + 1) * section), sum);
#pragma unroll
        for (int j = 0; j < 8; ++j) part[wave][64 * j + lane] = sum[j];
        __syncthreads();
        if (wave == 0) {
#pragma unroll 1
          for (int w = 1; w < kFewWaves; ++w)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += part[w][64 * j + lane];
          write(row, sum);
        }
        __syncthreads();
      }
    };
    for (int64_t c0 = (int64_t)blockIdx.y * 512; c0 < a.cols; c0 += (int64_t)gridDim.y * 512) {
      const int64_t c = c0 + lane_column<SPLIT>(lane);
      const Cover cover = cover_of(a.cols - c, gap, a.cols);  // the same for every wave
      if (cover == kWhole) columns(c, CoverOf<kWhole>{});
      else if (cover == kEnd) columns(c, CoverOf<kEnd>{});
      else columns(c, CoverOf<kFew>{});
    }
    __syncthreads();  // all have read the list
  }
}

// ---- stable radix sort of (row, token index) by row -------------------------------------------------------
//
// A pass takes `bits` bits of the row, the low ones first.  Its input is cut into tiles of consecutive entries,
// one per workgroup: count_kernel writes each tile's histogram, scatter_kernel adds up what stands before
// its tile (smaller digits anywhere, equal digits in earlier tiles), then places its entries in order: its waves
// take consecutive sections, a wave 64 entries at a time, entries of one digit by their lane.  The first pass
// reads the tokens themselves and leaves out those the table does not hold.
//
// Bound by latency, not by bytes: 131072 tokens of 65536 rows, two passes, 27 us (5 + 9 and 5 + 8) for 3 MB.

constexpr int kSortWaves = kSortThreads / 64;
constexpr int kMaxBins = 1 << kMaxBits;

struct SortArgs {
  const char* tokens;  // first pass
  int token_bytes;
  int64_t ntokens, first, rows;
  const int32_t *keys_in, *pos_in;  // later passes
  int32_t *keys_out, *pos_out;
  int32_t* counts;  // [tiles][bins]
  int32_t* nvalid;  // entries that the first pass keeps
  int shift, bits;
  int64_t tile;
  int32_t tiles;
};

// Entries i, i + step ... of a pass, below `end`: their rows (-1: none) and token indices.  All loads are in flight together.
constexpr int kEntries = 4;
template <bool FIRST>
__device__ __forceinline__ void entries(const SortArgs& a, int64_t i, int64_t step, int64_t end, int32_t (&key)[kEntries],
                                        int32_t (&pos)[kEntries]) {
#pragma unroll
  for (int u = 0; u < kEntries; ++u) {
    const int64_t at = min(i + u * step, end - 1);
    if constexpr (FIRST) {
      pos[u] = (int32_t)at;
      key[u] = (int32_t)token_row(a.tokens, a.token_bytes, at, a.first, a.rows);
    } else {
      pos[u] = ldg<int32_t, false>((const char*)(a.pos_in + at));
      key[u] = ldg<int32_t, false>((const char*)(a.keys_in + at));
    }
  }
#pragma unroll
  for (int u = 0; u < kEntries; ++u)
    if (i + u * step >= end) key[u] = -1;
}

template <bool FIRST>
__global__ __launch_bounds__(kSortThreads) void count_kernel(SortArgs a) {
  __shared__ int32_t hist[kMaxBins];
  const int bins = 1 << a.bits;
  for (int b = threadIdx.x; b < bins; b += kSortThreads) hist[b] = 0;
  __syncthreads();
  const int64_t n = FIRST ? a.ntokens : *a.nvalid, begin = blockIdx.x * a.tile;
  const int64_t end = min(begin + a.tile, n);
  for (int64_t i = begin + threadIdx.x; i < end; i += kEntries * kSortThreads) {
    int32_t key[kEntries], pos[kEntries];
    entries<FIRST>(a, i, kSortThreads, end, key, pos);
#pragma unroll
    for (int u = 0; u < kEntries; ++u)
      if (key[u] >= 0) atomicAdd(&hist[key[u] >> a.shift & (bins - 1)], 1);
  }
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += kSortThreads) a.counts[(int64_t)blockIdx.x * bins + b] = hist[b];
}

template <bool FIRST>
__global__ __launch_bounds__(kSortThreads) void scatter_kernel(SortArgs a) {
  __shared__ int32_t next[kSortWaves][kMaxBins];  // per wave and digit: where its next entry goes
  __shared__ __attribute__((aligned(16))) int32_t totals[kSortWaves][kMaxBins], befores[kSortWaves][kMaxBins];
  __shared__ int32_t sums[kSortThreads];
  const int bins = 1 << a.bits, t = threadIdx.x, wave = t / 64, lane = t % 64;
  const int64_t n = FIRST ? a.ntokens : *a.nvalid;
  const int64_t section = a.tile / kSortWaves, begin = blockIdx.x * a.tile + wave * section;

  for (int i = t; i < kSortWaves * bins; i += kSortThreads) next[i / bins][i % bins] = 0;
  __syncthreads();
  const int64_t end = min(begin + section, n);
  for (int64_t i = begin; i < end; i += kEntries * 64) {
    int32_t key[kEntries], pos[kEntries];
    entries<FIRST>(a, i + lane, 64, end, key, pos);
#pragma unroll
    for (int u = 0; u < kEntries; ++u)
      if (key[u] >= 0) atomicAdd(&next[wave][key[u] >> a.shift & (bins - 1)], 1);
  }

  // What the tiles' histograms hold, in all and before this tile: a wave adds up a quarter of them, four digits a lane.
  const int32_t quarter = (a.tiles + kSortWaves - 1) / kSortWaves;
  const int32_t w0 = wave * quarter, w1 = min(w0 + quarter, a.tiles);
  for (int b = 4 * lane; b < bins; b += 256) {
    v4i total = {0, 0, 0, 0}, before = {0, 0, 0, 0};
#pragma unroll 8
    for (int32_t w = w0; w < w1; ++w) {
      const v4i c = ldg<v4i, false>((const char*)(a.counts + (int64_t)w * bins + b));
      total += c;
      if (w < (int32_t)blockIdx.x) before += c;
    }
    *(v4i*)&totals[wave][b] = total;
    *(v4i*)&befores[wave][b] = before;
  }
  __syncthreads();

  // digits of lane t: consecutive ones, so that the scan over lanes is the scan over digits
  const int per = (bins + kSortThreads - 1) / kSortThreads;
  int32_t before[kMaxBins / kSortThreads], all = 0;
#pragma unroll
  for (int j = 0; j < kMaxBins / kSortThreads; ++j) {
    const int b = t * per + j;
    before[j] = all;
    if (j >= per || b >= bins) continue;
    for (int w = 0; w < kSortWaves; ++w) {
      before[j] += befores[w][b];
      all += totals[w][b];
    }
  }
  sums[t] = all;
  __syncthreads();
  for (int d = 1; d < kSortThreads; d <<= 1) {
    const int32_t left = t >= d ? sums[t - d] : 0;
    __syncthreads();
    sums[t] += left;
    __syncthreads();
  }
  if (FIRST && blockIdx.x == 0 && t == kSortThreads - 1) *a.nvalid = sums[t];
  const int32_t base = t ? sums[t - 1] : 0;
#pragma unroll
  for (int j = 0; j < kMaxBins / kSortThreads; ++j) {
    const int b = t * per + j;
    if (j >= per || b >= bins) continue;
    int32_t at = base + before[j];
    for (int w = 0; w < kSortWaves; ++w) {
      const int32_t c = next[w][b];
      next[w][b] = at;
      at += c;
    }
  }
  __syncthreads();

  for (int64_t i = begin; i < end; i += kEntries * 64) {
    int32_t keys[kEntries], pos[kEntries];
    entries<FIRST>(a, i + lane, 64, end, keys, pos);
#pragma unroll
    for (int u = 0; u < kEntries; ++u) {
      const int32_t key = keys[u];
      const int digit = key >> a.shift & (bins - 1);
      uint64_t same = __ballot(key >= 0);  // lanes of this lane's digit
      for (int b = 0; b < a.bits; ++b) {
        const bool one = digit >> b & 1;
        const uint64_t m = __ballot(one);
        same &= one ? m : ~m;
      }
      if (key >= 0) {
        const int leader = __builtin_ctzll(same);
        int32_t at = 0;
        if (lane == leader) at = atomicAdd(&next[wave][digit], __popcll(same));
        at = __shfl(at, leader) + __popcll(same & (((uint64_t)1 << lane) - 1));
        a.keys_out[at] = key;
        a.pos_out[at] = pos[u];
      }
    }
  }
}

// The whole sort in one workgroup, for so few tokens that launches are what it costs: 8 us for 2048 tokens of 1251 rows, 14
// for 4096 of 50000 (both ways' times stand at the rule, with kSmallTokens).  Entries stay in LDS from pass to pass; a wave takes a section of them, 64 at a time.
constexpr int kSmallThreads = 1024, kSmallWaves = kSmallThreads / 64;

__global__ __launch_bounds__(kSmallThreads) void small_sort_kernel(SortArgs a, int passes) {
  __shared__ int32_t next[kSmallWaves][1 << kSmallBits];
  __shared__ int32_t key[2][kSmallTokens];
  __shared__ int16_t pos[2][kSmallTokens];
  __shared__ int32_t sums[1 << kSmallBits];
  const int bins = 1 << a.bits, t = threadIdx.x, wave = t / 64, lane = t % 64;
  for (int i = t; i < a.ntokens; i += kSmallThreads) {
    key[0][i] = (int32_t)token_row(a.tokens, a.token_bytes, i, a.first, a.rows);
    pos[0][i] = (int16_t)i;
  }
  int n = (int)a.ntokens, at = 0;  // the first pass drops the entries of key -1
  for (int p = 0; p < passes; ++p, at ^= 1) {
    const int shift = p * a.bits, section = (n + kSmallThreads - 1) / kSmallThreads * 64, begin = wave * section;
    for (int i = t; i < kSmallWaves * bins; i += kSmallThreads) next[i / bins][i % bins] = 0;
    __syncthreads();
    for (int i = begin + lane; i < begin + section; i += 64) {
      const int32_t k = i < n ? key[at][i] : -1;
      if (k >= 0) atomicAdd(&next[wave][k >> shift & (bins - 1)], 1);
    }
    __syncthreads();
    int32_t total = 0;
    if (t < bins) {
      for (int w = 0; w < kSmallWaves; ++w) total += next[w][t];
      sums[t] = total;
    }
    __syncthreads();
    for (int d = 1; d < bins; d <<= 1) {
      const int32_t left = t < bins && t >= d ? sums[t - d] : 0;
      __syncthreads();
      if (t < bins) sums[t] += left;
      __syncthreads();
    }
    if (t < bins) {
      int32_t base = sums[t] - total;
      for (int w = 0; w < kSmallWaves; ++w) {
        const int32_t c = next[w][t];
        next[w][t] = base;
        base += c;
      }
    }
    __syncthreads();
    for (int i = begin + lane; i < begin + section; i += 64) {
      const int32_t k = i < n ? key[at][i] : -1;
      const int digit = k >> shift & (bins - 1);
      uint64_t same = __ballot(k >= 0);
      for (int b = 0; b < a.bits; ++b) {
        const bool one = digit >> b & 1;
        const uint64_t m = __ballot(one);
        same &= one ? m : ~m;
      }
      if (k >= 0) {
        const int leader = __builtin_ctzll(same);
        int32_t to = 0;
        if (lane == leader) to = atomicAdd(&next[wave][digit], __popcll(same));
        to = __shfl(to, leader) + __popcll(same & (((uint64_t)1 << lane) - 1));
        key[at ^ 1][to] = k;
        pos[at ^ 1][to] = pos[at][i];
      }
    }
    __syncthreads();
    n = sums[bins - 1];
    __syncthreads();
  }
  if (t == 0) *a.nvalid = n;
  for (int i = t; i < n; i += kSmallThreads) {
    a.keys_out[i] = key[at][i];
    a.pos_out[i] = pos[at][i];
  }
}

// First entry of keys[0, n) that is not below `key`, by a whole wave: 64 places are looked at together, so a search of
// 2^18 entries waits for three loads in turn and not for 18.
__device__ __forceinline__ int32_t wave_lower_bound(const int32_t* keys, int32_t n, int32_t key) {
  int32_t lo = 0, hi = n;
  while (lo < hi) {
    const int32_t step = (hi - lo + 63) / 64, at = lo + (threadIdx.x % 64 + 1) * step - 1;
    const int32_t below = __popcll(__ballot(at < hi && ldg<int32_t, false>((const char*)(keys + min(at, hi - 1))) < key));
    hi = min(hi, lo + (below + 1) * step - 1);
    lo += below * step;
  }
  return lo;
}

// ---- sums over the sorted entries -------------------------------------------------------------------------
//
// The sorted entries are cut into pieces of equal length, whatever rows they belong to, so that a frequent token is
// as much work as rare ones.  A row's entries inside one piece are summed in registers and written out at once;
// what a row has in several pieces goes to the workspace, a row of float32 per piece, and join_kernel adds these in
// order.  A piece has two such rows at most: slot 0 for the row of its first entry, slot 1 for that of its last.
// Rows without an entry are zeroed by workgroups of their own in the same launch.
//
// Bound by memory: 131072 tokens of 2048 bfloat16 columns into 65536 float32 rows (1.07 GB) in 210 to 222 us, 5.1 TB/s, and
// 17 us for the rows over pieces.  2048 float32 tokens of 333 columns, 1251 rows: 8 and 5 us, launches and one chain of loads.

struct SumArgs {
  const int32_t *keys, *pos, *nvalid;
  Mat g;
  MatOut out;
  float* partial;  // [pieces][2][pitch]
  int64_t rows, cols, pitch;
  float scale;
  int32_t piece;  // entries, a multiple of 8
  int lanes, sum_wgs, zero_wgs;
};

template <typename TO>
__device__ void zero_rows(const SumArgs& a, int wg, int32_t n) {
  __shared__ int32_t ends[2];
  __shared__ unsigned long long present;
  const int64_t r0 = (int64_t)wg * kZeroRows;
  if (threadIdx.x == 0) present = 0;
  if (threadIdx.x < 128) {
    const int32_t end = wave_lower_bound(a.keys, n, (int32_t)min(r0 + (threadIdx.x / 64 ? kZeroRows : 0), a.rows));
    if (threadIdx.x % 64 == 0) ends[threadIdx.x / 64] = end;
  }
  __syncthreads();
  const int32_t lo = ends[0], hi = ends[1];
  if (hi - lo <= 16 * 256) {  // the rows' entries, all looked at
    unsigned long long mine = 0;
    for (int32_t i = lo + (int)threadIdx.x; i < hi; i += 256) mine |= 1ull << (a.keys[i] - r0);
    if (mine) atomicOr(&present, mine);
  } else if (threadIdx.x < 64 && r0 + threadIdx.x < a.rows) {  // or each row searched for between them
    const int32_t row = (int32_t)(r0 + threadIdx.x);
    int32_t first = lo, end = hi;
    while (first < end) {
      const int32_t mid = first + (end - first) / 2;
      if (a.keys[mid] < row) first = mid + 1;
      else end = mid;
    }
    if (first < hi && a.keys[first] == row) atomicOr(&present, 1ull << threadIdx.x);
  }
  __syncthreads();
  constexpr bool SPLIT = Split<TO, TO>::value;
  const int side = 256 / a.lanes, lane = threadIdx.x % a.lanes;
  const int64_t gap = lane_gap<SPLIT>(a.lanes);
  const float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  const uint64_t m = present;
  const int here = (int)min((int64_t)kZeroRows, a.rows - r0);
  for (int i = threadIdx.x / a.lanes; i < here; i += side) {
    if (m >> i & 1) continue;
    for (int64_t c = lane_column<SPLIT>(lane); c < a.cols; c += 8 * a.lanes) {
      char* p = (char*)a.out.p + ((r0 + i) * a.out.stride + c) * TO::kBytes;
      if (a.cols - c >= gap + 4) store8<TO, SPLIT, true, kWhole>(p, a.cols - c, gap, zero);
      else store8<TO, SPLIT, true, kEnd>(p, a.cols - c, gap, zero);
    }
  }
}

// UNIFORM: a piece's lanes are whole waves (rows of 257 columns and more).  A wave then holds 64 entries at a time, one
// per lane, and takes each from its lane into scalar registers: no load of a row waits for a load of its entry.
template <bool UNIFORM, typename TI, typename TO>
__global__ __launch_bounds__(256) void sum_kernel(SumArgs a) {
  const int32_t n = *a.nvalid;
  // both kinds of workgroups in turn, as long as there are both
  const int both = 2 * min(a.sum_wgs, a.zero_wgs), rest = (int)blockIdx.x - both;
  const bool zeroes = rest < 0 ? blockIdx.x & 1 : a.zero_wgs > a.sum_wgs;
  const int wg = rest < 0 ? blockIdx.x / 2 : both / 2 + rest;
  if (zeroes) {
    if (blockIdx.y == 0) zero_rows<TO>(a, wg, n);
    return;
  }
  int side = threadIdx.x / a.lanes;
  if constexpr (UNIFORM) side = __builtin_amdgcn_readfirstlane(side);
  const int64_t piece = (int64_t)wg * (256 / a.lanes) + side;
  constexpr bool SPLIT = Split<TI, TO>::value;
  const int64_t i0 = piece * a.piece, gap = lane_gap<SPLIT>(a.lanes);
  const int64_t c = 8 * (int64_t)blockIdx.y * a.lanes + lane_column<SPLIT>(threadIdx.x % a.lanes);
  if (i0 >= n) return;
  const int64_t i1 = min(i0 + a.piece, (int64_t)n), left = a.cols - c;
  const bool open_left = i0 > 0 && a.keys[i0 - 1] == a.keys[i0];
  const bool open_right = i1 < n && a.keys[i1] == a.keys[i1 - 1];

  auto columns = [&](auto cover) {
    constexpr Cover C = decltype(cover)::value;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    int32_t row = a.keys[i0];
    bool head = true;  // still in the row of the piece's first entry
    auto flush = [&](bool last) {
      if ((head && open_left) || (last && open_right)) {
        float* p = a.partial + (2 * piece + (head ? 0 : 1)) * a.pitch + c;
        store8<F32, SPLIT, false, C>((char*)p, left, gap, sum);
      } else {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = sum[j] * a.scale;
        store8<TO, SPLIT, true, C>((char*)a.out.p + ((int64_t)row * a.out.stride + c) * TO::kBytes, left, gap, v);
      }
    };
    constexpr int U = 8;
    int32_t key64 = 0, pos64 = 0;
    for (int64_t i = i0; i < i1; i += U) {
      if (UNIFORM && (i - i0) % 64 == 0) {
        const int64_t at = min(i + threadIdx.x % 64, i1 - 1);
        key64 = a.keys[at];
        pos64 = a.pos[at];
      }
      int32_t key[U];
      float v[U][8];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        int64_t pos;
        if constexpr (UNIFORM) {
          const int src = (int)min(i + u, i1 - 1) - (int)(i - (i - i0) % 64);
          key[u] = __builtin_amdgcn_readlane(key64, src);
          pos = __builtin_amdgcn_readlane(pos64, src);
        } else {
          const int64_t at = min(i + u, i1 - 1);
          key[u] = a.keys[at];
          pos = a.pos[at];
        }
        load8<TI, SPLIT, true, C>((const char*)a.g.p + (pos * a.g.stride + c) * TI::kBytes, left, gap, v[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i + u >= i1) break;
        if (key[u] != row) {
          flush(false);
          row = key[u];
          head = false;
#pragma unroll
          for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += v[u][j];
      }
    }
    flush(true);
  };
  // one way for the whole wave: entries are taken from every lane, so every lane has to be there
  const Cover cover = cover_of(left, gap, a.cols);
  if (cover == kWhole) columns(CoverOf<kWhole>{});
  else if (cover == kEnd) columns(CoverOf<kEnd>{});
  else columns(CoverOf<kFew>{});
}

// A workgroup looks at kJoinPieces boundaries between pieces, for 256 columns.  Where a row goes over a boundary and
// over none before it, the workgroup adds up the row's partial sums: each wave takes a section of the pieces, then
// the waves' sums are added in order.
constexpr int kJoinWaves = 4, kJoinPieces = 4;

template <typename TO>
__global__ __launch_bounds__(64 * kJoinWaves) void join_kernel(SumArgs a) {
  __shared__ v4f part[kJoinWaves][64];
  const int32_t n = *a.nvalid;
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const int64_t b0 = (int64_t)blockIdx.x * kJoinPieces + 1, at = (b0 + lane) * a.piece;
  bool starts = false;
  if (lane < kJoinPieces && at < n) {
    const int32_t row = a.keys[at];
    starts = a.keys[at - 1] == row && !(b0 + lane > 1 && a.keys[at - a.piece - 1] == row);
  }
  const int64_t c = 256 * (int64_t)blockIdx.y + 4 * lane;
  for (uint64_t todo = __ballot(starts); todo; todo &= todo - 1) {  // the same in every wave
    const int64_t b = b0 + __builtin_ctzll(todo), p0 = b - 1;
    const int32_t row = a.keys[b * a.piece];
    // pieces after p0 that begin with the row, 64 looked at together
    int64_t p1 = b + 1;
    for (;;) {
      const int64_t p = p1 + lane;
      const uint64_t other = __ballot(p * a.piece >= n || a.keys[p * a.piece] != row);
      p1 += other ? __builtin_ctzll(other) : 64;
      if (other) break;
    }
    const int64_t per = (p1 - p0 + kJoinWaves - 1) / kJoinWaves, lo = p0 + wave * per, hi = min(lo + per, p1);
    const bool first_slot = a.keys[p0 * a.piece] == row;  // only the first piece may begin with another row
    v4f sum = {0, 0, 0, 0};
    if (c < a.cols) {
#pragma unroll 4
      for (int64_t p = lo; p < hi; ++p) {
        const int64_t slot = 2 * p + (p == p0 && !first_slot ? 1 : 0);
        sum += ldg<v4f, false>((const char*)(a.partial + slot * a.pitch + c));
      }
    }
    part[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && c < a.cols) {
#pragma unroll
      for (int w = 1; w < kJoinWaves; ++w) sum += part[w][lane];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (c + j < a.cols) TO::store((char*)a.out.p, (int64_t)row * a.out.stride + c + j, sum[j] * a.scale);
    }
    __syncthreads();
  }
}

// Workspace: the number of kept entries, two (keys, positions) pairs, the tiles' histograms, the partial sums.
struct GradSpace {
  int32_t *keys[2], *pos[2], *counts, *nvalid;
  float* partial;
  size_t bytes;
};

GradSpace grad_space(char* base, int64_t ntokens, const SortPlan& s, const SumPlan& u) {
  GradSpace w;
  size_t at = 0;
  auto take = [&](size_t words) {
    char* p = base + at;
    at += ceil_div(words * 4, 16) * 16;
    return p;
  };
  w.nvalid = (int32_t*)take(1);
  for (int i = 0; i < 2; ++i) {
    w.keys[i] = (int32_t*)take((size_t)ntokens);
    w.pos[i] = (int32_t*)take((size_t)ntokens);
  }
  w.counts = (int32_t*)take((size_t)s.tiles << s.bits);
  w.partial = (float*)take(u.pieces > 1 ? (size_t)(2 * u.pieces * u.pitch) : 0);
  w.bytes = at;
  return w;
}

template <int TOKENS, typename TI>
auto lookup_of(Elem dtype) {
  return dtype == Elem::f32 ? lookup_kernel<TOKENS, TI, F32> : lookup_kernel<TOKENS, TI, B16>;
}

template <bool UNIFORM, typename TI>
auto sum_of(Elem dtype) {
  return dtype == Elem::f32 ? sum_kernel<UNIFORM, TI, F32> : sum_kernel<UNIFORM, TI, B16>;
}

}  // namespace

hipError_t launch_embedding(const void* tokens, int token_bytes, int64_t ntokens, Mat table, Elem table_dtype,
                            int64_t first, int64_t rows, int64_t cols, float scale, MatOut out, Elem dtype,
                            hipStream_t stream) {
  const int lanes = row_lanes((cols + 7) / 8, 256);
  // One token a lane where that leaves workgroups for the chip (1001 tokens of 333 columns: 63 of them with four).
  // Large: 153 us with two in turn, 157 with four, 161 with eight (65536 tokens of 4096 bfloat16 columns).
  const int tokens_each = ceil_div(ntokens, 2 * (256 / lanes)) < 1024 ? 1 : 2;
  const bool f32 = table_dtype == Elem::f32;
  const auto kernel = tokens_each == 1 ? (f32 ? lookup_of<1, F32>(dtype) : lookup_of<1, B16>(dtype))
                                       : (f32 ? lookup_of<2, F32>(dtype) : lookup_of<2, B16>(dtype));
  const size_t wgs = std::min<size_t>(ceil_div(ntokens, tokens_each * (256 / lanes)), 1 << 20);
  hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(256), 0, stream, (const char*)tokens, token_bytes, ntokens, table,
                     first, rows, cols, scale, out, lanes);
  return hipGetLastError();
}

size_t embedding_grad_workspace(int64_t ntokens, int64_t rows, int64_t cols) {
  if (few_tokens(ntokens, rows)) return 0;
  return grad_space(nullptr, ntokens, sort_plan(ntokens, rows), sum_plan(ntokens, rows, cols)).bytes;
}

hipError_t launch_embedding_grad(const void* tokens, int token_bytes, int64_t ntokens, Mat g, Elem g_dtype, int64_t first,
                                 int64_t rows, int64_t cols, float scale, MatOut out, Elem dtype, void* workspace,
                                 hipStream_t stream) {
  if (few_tokens(ntokens, rows)) {
    // rows a wave: as many as leave two workgroups a CU, to list and wait once for all
    const int each = (int)std::min<size_t>(ceil_div(rows, kFewWaves * 512), kFewMostEach);
    FewArgs a{(const char*)tokens, token_bytes, (int)ntokens, each, first, rows, cols, g, out, scale};
    const size_t blocks = ceil_div(rows, kFewWaves * each);
    // workgroups side by side in a row where the rows alone do not fill the chip
    const size_t side = std::min(ceil_div(cols, 512), ceil_div(512, blocks));
    const auto kernel = g_dtype == Elem::f32 ? (dtype == Elem::f32 ? few_kernel<F32, F32> : few_kernel<F32, B16>)
                                             : (dtype == Elem::f32 ? few_kernel<B16, F32> : few_kernel<B16, B16>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<size_t>(blocks, 1 << 20), (unsigned)side), dim3(kFewTokens), 0, stream,
                       a);
    return hipGetLastError();
  }
  const SortPlan plan = sort_plan(ntokens, rows);
  const SumPlan cut = sum_plan(ntokens, rows, cols);
  const GradSpace w = grad_space((char*)workspace, ntokens, plan, cut);
  SortArgs a{};
  a.tokens = (const char*)tokens;
  a.token_bytes = token_bytes;
  a.ntokens = ntokens;
  a.first = first;
  a.rows = rows;
  a.counts = w.counts;
  a.nvalid = w.nvalid;
  a.bits = plan.bits;
  a.tile = plan.tile;
  a.tiles = (int32_t)plan.tiles;
  const dim3 grid((unsigned)plan.tiles), block(kSortThreads);
  const bool small = ntokens <= kSmallTokens;
  int at = 0;
  if (small) {
    a.keys_out = w.keys[0];
    a.pos_out = w.pos[0];
    hipLaunchKernelGGL(small_sort_kernel, dim3(1), dim3(kSmallThreads), 0, stream, a, plan.passes);
  }
  for (int p = 0; p < plan.passes && !small; ++p) {
    a.shift = p * plan.bits;
    a.keys_in = w.keys[at];
    a.pos_in = w.pos[at];
    at ^= 1;
    a.keys_out = w.keys[at];
    a.pos_out = w.pos[at];
    if (p == 0) {
      hipLaunchKernelGGL(count_kernel<true>, grid, block, 0, stream, a);
      hipLaunchKernelGGL(scatter_kernel<true>, grid, block, 0, stream, a);
    } else {
      hipLaunchKernelGGL(count_kernel<false>, grid, block, 0, stream, a);
      hipLaunchKernelGGL(scatter_kernel<false>, grid, block, 0, stream, a);
    }
  }
  SumArgs u{};
  u.keys = w.keys[at];
  u.pos = w.pos[at];
  u.nvalid = w.nvalid;
  u.g = g;
  u.out = out;
  u.partial = w.partial;
  u.rows = rows;
  u.cols = cols;
  u.pitch = cut.pitch;
  u.scale = scale;
  u.piece = cut.piece;
  u.lanes = cut.lanes;
  u.sum_wgs = (int)cut.sum_wgs;
  u.zero_wgs = (int)cut.zero_wgs;
  const bool uniform = cut.lanes >= 64, f32 = g_dtype == Elem::f32;
  const auto kernel = uniform ? (f32 ? sum_of<true, F32>(dtype) : sum_of<true, B16>(dtype))
                              : (f32 ? sum_of<false, F32>(dtype) : sum_of<false, B16>(dtype));
  hipLaunchKernelGGL(kernel, dim3((unsigned)(cut.sum_wgs + cut.zero_wgs), (unsigned)cut.col_wgs), dim3(256), 0, stream, u);
  if (cut.pieces > 1) {
    const auto join = dtype == Elem::f32 ? join_kernel<F32> : join_kernel<B16>;
    hipLaunchKernelGGL(join, dim3((unsigned)ceil_div(cut.pieces - 1, kJoinPieces), (unsigned)ceil_div(cols, 256)), dim3(64 * kJoinWaves), 0,
                       stream, u);
  }
  return hipGetLastError();
}

}  // namespace pat
