// Embedding lookup with scaling, and its dense gradient by sorted tokens.
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

// One workgroup per token (in turn).
template <typename TI, typename TO>
__global__ __launch_bounds__(256) void lookup_kernel(const char* tokens, int token_bytes, int64_t ntokens, Mat table,
                                                     int64_t first, int64_t rows, int64_t cols, float scale, MatOut out) {
  for (int64_t t = blockIdx.x; t < ntokens; t += gridDim.x) {
    const int64_t row = token_row(tokens, token_bytes, t, first, rows);
    for (int64_t c = threadIdx.x; c < cols; c += 256)
      TO::store((char*)out.p, t * out.stride + c,
                row < 0 ? 0.0f : TI::load((const char*)table.p, row * table.stride + c) * scale);
  }
}

// ---- stable radix sort of (row, token index) by row -------------------------------------------------------
//
// A pass takes `bits` bits of the row, the low ones first.  Its input is cut into tiles of consecutive entries,
// one per workgroup: count_kernel writes each tile's histogram, scatter_kernel adds up what stands before
// its tile (smaller digits anywhere, equal digits in earlier tiles), then places its entries in order: its waves
// take consecutive sections, a wave 64 entries at a time, entries of one digit by their lane.  The first pass
// reads the tokens themselves and leaves out those the table does not hold.

constexpr int kSortThreads = 256, kSortWaves = kSortThreads / 64;
constexpr int kMaxBins = 1 << 10;

struct SortPlan {
  int bits, passes;
  int64_t tile, tiles;  // entries per workgroup, workgroups
};

SortPlan sort_plan(int64_t ntokens, int64_t rows) {
  int kb = 1;
  while (((int64_t)1 << kb) < rows) ++kb;
  SortPlan s;
  s.passes = (kb + 9) / 10;
  s.bits = (kb + s.passes - 1) / s.passes;
  s.tile = (int64_t)ceil_div(ceil_div(ntokens, 128), kSortThreads) * kSortThreads;
  if (s.tile < 1024) s.tile = 1024;
  s.tiles = (int64_t)ceil_div(ntokens, s.tile);
  return s;
}

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

// Entry i of a pass: its row (-1: none) and token index.
template <bool FIRST>
__device__ __forceinline__ int32_t entry(const SortArgs& a, int64_t i, int64_t n, int32_t* pos) {
  if (i >= n) return -1;
  if constexpr (FIRST) {
    *pos = (int32_t)i;
    return (int32_t)token_row(a.tokens, a.token_bytes, i, a.first, a.rows);
  } else {
    *pos = ldg<int32_t, false>((const char*)(a.pos_in + i));
    return ldg<int32_t, false>((const char*)(a.keys_in + i));
  }
}

template <bool FIRST>
__global__ __launch_bounds__(kSortThreads) void count_kernel(SortArgs a) {
  __shared__ int32_t hist[kMaxBins];
  const int bins = 1 << a.bits;
  for (int b = threadIdx.x; b < bins; b += kSortThreads) hist[b] = 0;
  __syncthreads();
  const int64_t n = FIRST ? a.ntokens : *a.nvalid, begin = blockIdx.x * a.tile;
  for (int64_t i = begin + threadIdx.x; i < begin + a.tile; i += kSortThreads) {
    int32_t pos;
    const int32_t key = entry<FIRST>(a, i, n, &pos);
    if (key >= 0) atomicAdd(&hist[key >> a.shift & (bins - 1)], 1);
  }
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += kSortThreads) a.counts[(int64_t)blockIdx.x * bins + b] = hist[b];
}

template <bool FIRST>
__global__ __launch_bounds__(kSortThreads) void scatter_kernel(SortArgs a) {
  __shared__ int32_t next[kSortWaves][kMaxBins];  // per wave and digit: where its next entry goes
  __shared__ int32_t sums[kSortThreads];
  const int bins = 1 << a.bits, t = threadIdx.x, wave = t / 64, lane = t % 64;
  const int64_t n = FIRST ? a.ntokens : *a.nvalid;
  const int64_t section = a.tile / kSortWaves, begin = blockIdx.x * a.tile + wave * section;

  for (int i = t; i < kSortWaves * bins; i += kSortThreads) next[i / bins][i % bins] = 0;
  __syncthreads();
  for (int64_t i = begin + lane; i < begin + section; i += 64) {
    int32_t pos;
    const int32_t key = entry<FIRST>(a, i, n, &pos);
    if (key >= 0) atomicAdd(&next[wave][key >> a.shift & (bins - 1)], 1);
  }

  // digits of lane t: consecutive ones, so that the scan over lanes is the scan over digits
  const int per = (bins + kSortThreads - 1) / kSortThreads;
  int32_t before[kMaxBins / kSortThreads], all = 0;
#pragma unroll
  for (int j = 0; j < kMaxBins / kSortThreads; ++j) {
    const int b = t * per + j;
    before[j] = 0;
    if (j >= per || b >= bins) continue;
    int32_t total = 0;
    for (int32_t w = 0; w < a.tiles; ++w) {
      const int32_t c = a.counts[(int64_t)w * bins + b];
      if (w < (int32_t)blockIdx.x) before[j] += c;
      total += c;
    }
    before[j] += all;
    all += total;
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

  for (int64_t i = begin + lane; i < begin + section; i += 64) {
    int32_t pos = 0;
    const int32_t key = entry<FIRST>(a, i, n, &pos);
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
      a.pos_out[at] = pos;
    }
  }
}

// First entry of keys[0, n) that is not below `key`.
__device__ __forceinline__ int32_t lower_bound(const int32_t* keys, int32_t n, int32_t key) {
  int32_t lo = 0, hi = n;
  while (lo < hi) {
    const int32_t mid = lo + (hi - lo) / 2;
    if (ldg<int32_t, false>((const char*)(keys + mid)) < key) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}

// One workgroup per row (in turn): the row's tokens are keys' run of its number.
template <typename TI, typename TO>
__global__ __launch_bounds__(256) void sum_kernel(const int32_t* keys, const int32_t* pos, const int32_t* nvalid, Mat g,
                                                  int64_t rows, int64_t cols, float scale, MatOut out) {
  const int32_t n = nvalid ? *nvalid : 0;
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const int32_t lo = lower_bound(keys, n, (int32_t)r), hi = lower_bound(keys, n, (int32_t)r + 1);
    for (int64_t c = threadIdx.x; c < cols; c += 256) {
      float s = 0.0f;
      for (int32_t i = lo; i < hi; ++i) s += TI::load((const char*)g.p, (int64_t)pos[i] * g.stride + c);
      TO::store((char*)out.p, r * out.stride + c, s * scale);
    }
  }
}

// Workspace: two (keys, positions) pairs, the tiles' histograms, the number of kept entries.
struct GradSpace {
  int32_t *keys[2], *pos[2], *counts, *nvalid;
  size_t bytes;
};

GradSpace grad_space(char* base, int64_t ntokens, const SortPlan& s) {
  GradSpace w;
  size_t at = 0;
  auto take = [&](size_t words) {
    int32_t* p = reinterpret_cast<int32_t*>(base + at);
    at += ceil_div(words * 4, 16) * 16;
    return p;
  };
  w.nvalid = take(1);
  for (int i = 0; i < 2; ++i) {
    w.keys[i] = take((size_t)ntokens);
    w.pos[i] = take((size_t)ntokens);
  }
  w.counts = take((size_t)s.tiles << s.bits);
  w.bytes = at;
  return w;
}

template <typename TI>
auto lookup_of(Elem dtype) {
  return dtype == Elem::f32 ? lookup_kernel<TI, F32> : lookup_kernel<TI, B16>;
}

template <typename TI>
auto sum_of(Elem dtype) {
  return dtype == Elem::f32 ? sum_kernel<TI, F32> : sum_kernel<TI, B16>;
}

}  // namespace

hipError_t launch_embedding(const void* tokens, int token_bytes, int64_t ntokens, Mat table, Elem table_dtype,
                            int64_t first, int64_t rows, int64_t cols, float scale, MatOut out, Elem dtype,
                            hipStream_t stream) {
  const auto kernel = table_dtype == Elem::f32 ? lookup_of<F32>(dtype) : lookup_of<B16>(dtype);
  hipLaunchKernelGGL(kernel, dim3((unsigned)(ntokens < (1 << 20) ? ntokens : 1 << 20)), dim3(256), 0, stream,
                     (const char*)tokens, token_bytes, ntokens, table, first, rows, cols, scale, out);
  return hipGetLastError();
}

size_t embedding_grad_workspace(int64_t ntokens, int64_t rows, int64_t) {
  return ntokens ? grad_space(nullptr, ntokens, sort_plan(ntokens, rows)).bytes : 0;
}

hipError_t launch_embedding_grad(const void* tokens, int token_bytes, int64_t ntokens, Mat g, Elem g_dtype, int64_t first,
                                 int64_t rows, int64_t cols, float scale, MatOut out, Elem dtype, void* workspace,
                                 hipStream_t stream) {
  const SortPlan plan = sort_plan(ntokens, rows);
  const GradSpace w = grad_space((char*)workspace, ntokens, plan);
  int at = 0;
  if (ntokens) {
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
    for (int p = 0; p < plan.passes; ++p) {
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
  }
  const auto kernel = g_dtype == Elem::f32 ? sum_of<F32>(dtype) : sum_of<B16>(dtype);
  hipLaunchKernelGGL(kernel, dim3((unsigned)(rows < (1 << 20) ? rows : 1 << 20)), dim3(256), 0, stream, w.keys[at],
                     w.pos[at], ntokens ? w.nvalid : nullptr, g, rows, cols, scale, out);
  return hipGetLastError();
}

}  // namespace pat
