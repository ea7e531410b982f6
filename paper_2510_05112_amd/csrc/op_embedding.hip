// Embedding lookup of a model's first stage, and the gradient of its table.
//
// Lookup: out[t] = scale table[tokens[t]].  A row is moved by a power of two of lanes, 16 bytes a lane, whatever its address; bound by memory for many tokens, by one load behind another (token, row) for few: 61 rows of
// 2,560 take 2.8 us.
//
// Gradient: dE[v] = scale sum over {t : tokens[t] = v} grad[t].  Adding rows with atomics would make the sums depend on
// their order; here the occurrences are sorted by token (a stable counting sort, 8 bits of the token a pass), so that each row of
// dE is the sum of a run of sorted occurrences.  Text repeats its few commonest tokens thousands of times: so that a
// run's length bounds nothing, the sorted occurrences are cut into blocks of 16 without regard to runs, each summed by
// workgroups of its own; a run inside one block is written where it belongs, one across blocks leaves its parts (32 bits) in the workspace, which
// another kernel adds up, of more than 16,384 tokens with sums over chunks of 64 blocks in between (131,072 tokens that are all the same, 1,024 wide: 767 us
// by one wavefront a run, 193 so).  Most rows of a large vocabulary have no token: all are filled with zeros by what the sort leaves of the chip.
// Floor: grad read once, dE written once.  Measured (bf16): 4,096 tokens into 65,536 x 4,096 sort and zeros 88 us (537 MB of zeros: 6.1 TB/s,
// and a fill by itself reaches 6.9), sums 25, runs across blocks 7; 16,384 into 262,144 x 2,560 224 us, 47 and 8.  (Zeros of some rows beside the sums of
// others instead, a quarter of the table: 134 against 119 us and 302 against 290.)
#include "ops_common.h"

#include <algorithm>

namespace fpsched {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kMaxWidth = 1 << 20, kMaxSummed = 1 << 30, kMostRows = 0x7fffffff;   // (places and tokens are 32-bit numbers)

// ---- lookup ----------------------------------------------------------------------------------------------------------

template <typename T>
__global__ __launch_bounds__(kThreads) void embedding_kernel(const T* table, int64_t table_stride, int64_t n_rows, int64_t width,
                                                            const void* tokens, int tokens64, int64_t n_tokens, float scale, T* out,
                                                            int64_t out_stride, int lanes_shift) {
  constexpr int N = kWide<T>;
  const int64_t step = (int64_t)gridDim.x << (8 - lanes_shift);   // (more than one each where a grid has no room for all)
  for (int64_t t = ((int64_t)blockIdx.x << (8 - lanes_shift)) + (threadIdx.x >> lanes_shift); t < n_tokens; t += step) {
    const int64_t token = token_at(tokens, tokens64, t);
    const bool real = token >= 0 && token < n_rows;
    const T* from = table + (real ? token * table_stride : 0);
    T* to = out + t * out_stride;
    const int lanes = 1 << lanes_shift;
    for (int64_t at = (int64_t)(threadIdx.x & (lanes - 1)) * N; at < width; at += (int64_t)lanes * N) {
      const int64_t c = width < N ? at : min(at, width - N);   // (the last piece's begin is another one's end, with the same values)
      if (c + N <= width) {
        Vec<T, N> v = {};
        if (real) {
          v = load_any<T, N>(from + c);
#pragma unroll
          for (int i = 0; i < N; ++i) v.at[i] = (T)((float)v.at[i] * scale);
        }
        store_any<T, N>(to + c, v);
      } else {
        for (int64_t i = c; i < width; ++i) to[i] = real ? (T)((float)from[i] * scale) : (T)0.f;
      }
    }
  }
}

// ---- zeros -------------------------------------------------------------------------------------------------------------

// A slice of the table's rows to be filled with zeros by the workgroups from `first` on (bytes of an element: 2 or 4).
struct Fill {
  char* out;              // NULL: nothing to fill
  int64_t rows, row_bytes, stride_bytes;   // adjacent rows are one row
  int wide;               // rows begin at multiples of 16 bytes
  int element;
  unsigned first;
  int slice, slices;

  __device__ __forceinline__ bool mine() const { return blockIdx.x >= first; }
  __device__ void run() const {
    if (!out) return;
    const int64_t at = (int64_t)(blockIdx.x - first) * blockDim.x + threadIdx.x, all = (int64_t)(gridDim.x - first) * blockDim.x;
    const int unit = wide ? 16 : element;
    const int64_t units = row_bytes / unit;
    auto put = [&](char* to) {
      if (wide) *reinterpret_cast<Vec<unsigned, 4>*>(to) = {};
      else if (element == 4) *reinterpret_cast<unsigned*>(to) = 0;
      else *reinterpret_cast<unsigned short*>(to) = 0;
    };
    if (rows == 1) {
      // (a workgroup's four stores are neighbours)
      const int64_t end = units * (slice + 1) / slices;
      for (int64_t i = units * slice / slices + (at - threadIdx.x) * 4 + threadIdx.x; i < end; i += all * 4)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (i + k * blockDim.x < end) put(out + (i + k * blockDim.x) * unit);
    } else {
      const int64_t end = rows * (slice + 1) / slices;
      for (int64_t r = rows * slice / slices + blockIdx.x - first; r < end; r += gridDim.x - first)
        for (int64_t i = threadIdx.x; i < units; i += blockDim.x) put(out + r * stride_bytes + i * unit);
    }
    // (what is left of rows that are no multiple of 16 bytes)
    const int left = (int)(row_bytes % unit);
    if (left && slice == slices - 1)
      for (int64_t i = at; i < rows * left; i += all) out[i / left * stride_bytes + units * unit + i % left] = 0;
  }
};

// ---- sorting the occurrences -------------------------------------------------------------------------------------------

constexpr int kDigits = 256;

struct Occurrence {
  unsigned token, at;
};

// The lanes with the same digit, among those that have one.
__device__ __forceinline__ unsigned long long same_digit(bool have, unsigned digit) {
  unsigned long long same = __ballot(have);
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    const unsigned long long ones = __ballot(have && (digit >> b & 1));
    same &= digit >> b & 1 ? ones : ~ones;
  }
  return same;
}
__device__ __forceinline__ unsigned lanes_in_front(unsigned long long of, int lane) { return __popcll(of & ((1ull << lane) - 1)); }

// Up to kOneSort occurrences, all passes by one workgroup in LDS, ROUNDS of 1,024 (as many as there are: with room for 16, 4,000 tokens took 28.6 us
// into a table of 5,000 x 512, and 22.7 with room for 4).  A wavefront has 64 `rounds` adjacent ones; a lane's place among those
// of its digit is counted wavefront by wavefront, then over the wavefronts, then over the digits.
constexpr unsigned kNone = ~0u;   // (a table has fewer rows)
constexpr int kMostRounds = 16, kOneSort = 1024 * kMostRounds;

template <int ROUNDS>
__global__ __launch_bounds__(1024) void sort_few_kernel(const void* tokens, int tokens64, int n_tokens, int64_t n_rows, Occurrence* sorted,
                                                       unsigned* total, Fill fill) {
  if (fill.mine()) return fill.run();
  __shared__ unsigned held_token[1024 * ROUNDS];
  __shared__ unsigned short held_at[1024 * ROUNDS];
  __shared__ unsigned short next[16][kDigits];
  __shared__ unsigned sums[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int rounds = (n_tokens + 1023) / 1024;
  int n = n_tokens;
  for (int shift = 0; shift == 0 || (n_rows - 1) >> shift != 0; shift += 8) {
    unsigned token[ROUNDS];     // kNone: none
    unsigned at_rank[ROUNDS];   // which occurrence it is; in the upper half, its place among those of its digit
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      const int i = (wave * rounds + r) * 64 + lane;
      token[r] = kNone, at_rank[r] = 0;
      if (r < rounds && i < n) {
        if (shift == 0) {
          const int64_t t = token_at(tokens, tokens64, i);
          if (t >= 0 && t < n_rows) token[r] = (unsigned)t, at_rank[r] = (unsigned)i;
        } else {
          token[r] = held_token[i], at_rank[r] = held_at[i];
        }
      }
    }
    for (int i = threadIdx.x; i < 16 * kDigits; i += 1024) next[0][i] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      if (r < rounds) {
        const bool have = token[r] != kNone;
        const unsigned digit = token[r] >> shift & (kDigits - 1);
        const unsigned long long same = same_digit(have, digit);
        const unsigned ahead = lanes_in_front(same, lane);
        unsigned base = 0;
        if (have) base = next[wave][digit];
        __builtin_amdgcn_wave_barrier();
        if (have && ahead == 0) next[wave][digit] = (unsigned short)(base + __popcll(same));
        __builtin_amdgcn_wave_barrier();
        at_rank[r] |= (base + ahead) << 16;
      }
    }
    __syncthreads();
    unsigned mine = 0, before = 0;
    if (threadIdx.x < kDigits) {
#pragma unroll
      for (int w = 0; w < 16; ++w) mine += next[w][threadIdx.x];
      unsigned incl = mine;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const unsigned other = __shfl_up(incl, d);
        incl += lane >= d ? other : 0u;
      }
      if (lane == 63) sums[wave] = incl;
      before = incl - mine;
    }
    __syncthreads();
    n = (int)(sums[0] + sums[1] + sums[2] + sums[3]);
    if (threadIdx.x < kDigits) {
      for (int w = 0; w < wave; ++w) before += sums[w];
#pragma unroll
      for (int w = 0; w < 16; ++w) {
        const unsigned c = next[w][threadIdx.x];
        next[w][threadIdx.x] = (unsigned short)before;
        before += c;
      }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r)
      if (token[r] != kNone) {
        const unsigned place = next[wave][token[r] >> shift & (kDigits - 1)] + (at_rank[r] >> 16);
        held_token[place] = token[r];
        held_at[place] = (unsigned short)at_rank[r];
      }
    __syncthreads();
  }
  for (int i = threadIdx.x; i < n; i += 1024) sorted[i] = {held_token[i], held_at[i]};
  if (threadIdx.x == 0) *total = (unsigned)n;
}

// More of them: three kernels a pass, over tiles of kSortTile.
constexpr int kSortRounds = 8, kSortTile = kThreads * kSortRounds;

// An occurrence to be sorted: of the first pass from the tokens (those outside the table are none), later of the pass before
// (`n` of them).
struct SortSource {
  const void* tokens;
  int tokens64;
  int64_t n_tokens, n_rows;
  const Occurrence* sorted;
  const unsigned* n;

  __device__ __forceinline__ bool get(int64_t i, Occurrence* o) const {
    o->token = o->at = 0;
    if (sorted) {
      if (i >= *n) return false;
      *o = sorted[i];
      return true;
    }
    if (i >= n_tokens) return false;
    const int64_t token = token_at(tokens, tokens64, i);
    o->token = (unsigned)token;
    o->at = (unsigned)i;
    return token >= 0 && token < n_rows;
  }
};

// counts[digit][workgroup]
__global__ __launch_bounds__(kThreads) void sort_count_kernel(SortSource src, int shift, unsigned* counts, Fill fill) {
  if (fill.mine()) return fill.run();
  __shared__ unsigned held[kDigits];
  held[threadIdx.x] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * kSortTile;
  for (int r = 0; r < kSortRounds; ++r) {
    Occurrence o;
    if (src.get(first + r * kThreads + threadIdx.x, &o)) atomicAdd(&held[(o.token >> shift) & (kDigits - 1)], 1u);
  }
  __syncthreads();
  counts[(int64_t)threadIdx.x * fill.first + blockIdx.x] = held[threadIdx.x];
}

// counts -> the place of the first occurrence of each (digit, workgroup); *total: how many there are
__global__ __launch_bounds__(1024) void sort_scan_kernel(unsigned* counts, int64_t n, unsigned* total, Fill fill) {
  if (fill.mine()) return fill.run();
  __shared__ unsigned waves[16];
  unsigned before = 0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  constexpr int kEach = 16;
  for (int64_t at = 0; at < n; at += 1024 * kEach) {
    const int64_t mine = at + threadIdx.x * kEach;
    unsigned c[kEach], sum = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      c[i] = mine + i < n ? counts[mine + i] : 0u;
      sum += c[i];
    }
    unsigned incl = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const unsigned other = __shfl_up(incl, d);
      incl += lane >= d ? other : 0u;
    }
    if (lane == 63) waves[wave] = incl;
    __syncthreads();
    unsigned base = before, all = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      base += w < wave ? waves[w] : 0u;
      all += waves[w];
    }
    base += incl - sum;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (mine + i < n) counts[mine + i] = base;
      base += c[i];
    }
    before += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) *total = before;
}

// Places a workgroup's occurrences in order.  Each wavefront takes a piece of them, counts its digits first, and places them behind
// those of the wavefronts in front of it.
__global__ __launch_bounds__(kThreads) void sort_place_kernel(SortSource src, int shift, const unsigned* places, Occurrence* out, Fill fill) {
  if (fill.mine()) return fill.run();
  __shared__ unsigned next[kThreads / 64][kDigits];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int w = 0; w < kThreads / 64; ++w) next[w][threadIdx.x] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * kSortTile + wave * 64 * kSortRounds + lane;
  Occurrence o[kSortRounds];
  unsigned rank[kSortRounds];
  bool have[kSortRounds];
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) have[r] = src.get(first + r * 64, &o[r]);
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const unsigned digit = (o[r].token >> shift) & (kDigits - 1);
    const unsigned long long same = same_digit(have[r], digit);
    const unsigned ahead = lanes_in_front(same, lane);
    unsigned base = 0;
    if (have[r]) base = next[wave][digit];
    __builtin_amdgcn_wave_barrier();
    if (have[r] && ahead == 0) next[wave][digit] = base + __popcll(same);
    __builtin_amdgcn_wave_barrier();
    rank[r] = base + ahead;
  }
  __syncthreads();
  unsigned at = places[(int64_t)threadIdx.x * fill.first + blockIdx.x];
  for (int w = 0; w < kThreads / 64; ++w) {
    const unsigned c = next[w][threadIdx.x];
    next[w][threadIdx.x] = at;
    at += c;
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r)
    if (have[r]) out[next[wave][(o[r].token >> shift) & (kDigits - 1)] + rank[r]] = o[r];
}

// ---- sums --------------------------------------------------------------------------------------------------------------

constexpr int kBlock = 16;   // sorted occurrences that are summed in one go

template <typename O, int N>
__device__ __forceinline__ void put_sum(O* out, const float* sum, float scale, int accumulate, int64_t c, int64_t width) {
  if (c + N <= width) {
    Vec<O, N> v = {};
    if (accumulate) v = load_any<O, N>(out + c);
#pragma unroll
    for (int i = 0; i < N; ++i) v.at[i] = (O)((accumulate ? (float)v.at[i] : 0.f) + sum[i] * scale);
    store_any<O, N>(out + c, v);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (c + i < width) out[c + i] = (O)((accumulate ? (float)out[c + i] : 0.f) + sum[i] * scale);
  }
}

// blockIdx.x: block of sorted occurrences behind first_block, blockIdx.y: piece of the width.  Part 2 b: of the run that block b begins in
// the middle of, 2 b + 1: of the run that goes on behind it.
template <typename T, typename O, int N>
__global__ __launch_bounds__(64) void row_sums_kernel(const T* __restrict__ grad, int64_t grad_stride, int64_t width,
                                                     const Occurrence* __restrict__ sorted, const unsigned* __restrict__ n, float scale,
                                                     O* __restrict__ out, int64_t out_stride, int accumulate, float* __restrict__ parts,
                                                     int64_t part_stride, unsigned first_block) {
  const unsigned block = first_block + blockIdx.x, first = block * (unsigned)kBlock, all = *n;
  if (first >= all) return;
  const unsigned end = min(first + kBlock, all);
  // A lane an occurrence, for all lanes to read: lanes behind the width stay, with the first column's addresses, and write nothing (a lane that
  // has returned loads nothing, and what others read of its registers is anything).
  const Occurrence mine = sorted[min(first + threadIdx.x % kBlock, end - 1)];
  const int64_t column = ((int64_t)blockIdx.y * 64 + threadIdx.x) * N;
  const bool live = column < width;
  const int64_t c = live ? column : 0;
  const bool whole = c + N <= width;
  float sum[N] = {};
  unsigned now = sorted[first].token;
  bool inside = first == 0 || sorted[first - 1].token != now;   // the run that is being summed begins in this block
  const bool goes_on = end < all && sorted[end].token == sorted[end - 1].token;
  auto flush = [&](bool ends) {
    if (!live) {
    } else if (inside && ends) {
      put_sum<O, N>(out + (int64_t)now * out_stride, sum, scale, accumulate, c, width);
    } else {
      float* part = parts + (2 * (int64_t)block + inside) * part_stride + c;   // (part_stride has room for whole vectors)
#pragma unroll
      for (int i = 0; i < N; ++i) part[i] = sum[i];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = 0.f;
  };
  constexpr int kAhead = 8;
  const int count = (int)(end - first);
#pragma unroll 1
  for (int b = 0; b < count; b += kAhead) {
    Vec<T, N> v[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const T* from = grad + (int64_t)__builtin_amdgcn_readlane(mine.at, b + i) * grad_stride + c;
      if (whole) {
        v[i] = load_any<T, N>(from);
      } else {
        v[i] = {};
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (c + e < width) v[i].at[e] = from[e];
      }
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (b + i < count) {
        const unsigned token = __builtin_amdgcn_readlane(mine.token, b + i);
        if (token != now) {
          flush(true);
          now = token;
          inside = true;
        }
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] += (float)v[i].at[e];
      }
    }
  }
  flush(!goes_on);
}

// The last of blocks low .. high that begins with `token`, which low does (they are in order).
__device__ __forceinline__ unsigned last_block_of(unsigned token, const Occurrence* sorted, unsigned low, unsigned high) {
  while (low < high) {
    const unsigned mid = (low + high + 1) >> 1;
    if (sorted[(int64_t)mid * kBlock].token == token) low = mid; else high = mid - 1;
  }
  return low;
}
// The sum of n parts, part_stride apart, from `from` on.
template <int N>
__device__ __forceinline__ void sum_parts(const float* from, int64_t part_stride, unsigned n, float (&sum)[N]) {
  constexpr unsigned kAhead = 8;
  unsigned b = 0;
  for (; b + kAhead <= n; b += kAhead) {
    float x[kAhead][N];
#pragma unroll
    for (unsigned j = 0; j < kAhead; ++j, from += part_stride)
#pragma unroll
      for (int i = 0; i < N; ++i) x[j][i] = from[i];
#pragma unroll
    for (unsigned j = 0; j < kAhead; ++j)
#pragma unroll
      for (int i = 0; i < N; ++i) sum[i] += x[j][i];
  }
  for (; b < n; ++b, from += part_stride)
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] += from[i];
}

// Long runs: what a run that comes into a chunk of kChunk blocks has in that chunk is summed into its first block's part.  blockIdx.x: chunk.
constexpr unsigned kChunk = 64;
template <int N>
__global__ __launch_bounds__(64) void chunk_sums_kernel(const Occurrence* __restrict__ sorted, const unsigned* __restrict__ n, int64_t width, float* parts, int64_t part_stride) {
  const unsigned first = blockIdx.x * kChunk, all = *n;
  if (first == 0 || (int64_t)first * kBlock >= all) return;
  const unsigned token = sorted[(int64_t)first * kBlock].token;
  if (sorted[(int64_t)first * kBlock - 1].token != token) return;
  const unsigned last = last_block_of(token, sorted, first, min((all - 1) / kBlock, first + kChunk - 1));
  const int64_t c = ((int64_t)blockIdx.y * 64 + threadIdx.x) * N;
  if (c >= width) return;
  float sum[N] = {};
  float* to = parts + 2 * (int64_t)first * part_stride + c;
  sum_parts<N>(to, 2 * part_stride, last - first + 1, sum);
#pragma unroll
  for (int i = 0; i < N; ++i) to[i] = sum[i];
}

// The runs across blocks: the workgroups of the block that one begins in add up its parts, each wavefront a share of them, put together in order.
// CHUNKS: of the chunks behind its own one, what each has of it.
constexpr int kJoinWaves = 4;
template <typename O, int N, bool CHUNKS>
__global__ __launch_bounds__(kJoinWaves * 64) void join_runs_kernel(const Occurrence* __restrict__ sorted, const unsigned* __restrict__ n, int64_t width,
                                                      const float* __restrict__ parts, int64_t part_stride, float scale,
                                                      O* __restrict__ out, int64_t out_stride, int accumulate, unsigned first_block) {
  __shared__ float shares[kJoinWaves][64][N + 1];   // (N + 1: lanes' numbers in different banks)
  const unsigned block = first_block + blockIdx.x, first = block * (unsigned)kBlock, all = *n, end = first + kBlock;
  if (end >= all) return;
  const unsigned token = sorted[end - 1].token;
  if (sorted[end].token != token) return;
  if (sorted[first].token == token && first > 0 && sorted[first - 1].token == token) return;   // (it begins further in front)
  // the last block that has some of it (its tokens begin blocks up to there)
  const unsigned next = block + 1, last = last_block_of(token, sorted, next, (all - 1) / kBlock);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t column = ((int64_t)blockIdx.y * 64 + lane) * N;
  const bool live = column < width;
  const int64_t c = live ? column : 0;
  float sum[N] = {};
  auto add = [&](unsigned at, unsigned step, unsigned count) {   // parts of blocks at, at + step, ...: a share for each wavefront
    const unsigned share = (count + kJoinWaves - 1) / kJoinWaves, begin = min(wave * share, count);
    sum_parts<N>(parts + 2 * ((int64_t)at + (int64_t)begin * step) * part_stride + c, 2 * (int64_t)step * part_stride, min(share, count - begin), sum);
  };
  if (!CHUNKS) {
    add(next, 1, last - block);
  } else {
    const unsigned chunk = (next + kChunk - 1) / kChunk;   // the first one that it comes into
    add(next, 1, min(last + 1, chunk * kChunk) - next);
    if (last >= chunk * kChunk) add(chunk * kChunk, kChunk, last / kChunk - chunk + 1);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) shares[wave][lane][i] = sum[i];
  __syncthreads();
  if (wave || !live) return;
#pragma unroll
  for (int i = 0; i < N; ++i) sum[i] = parts[(2 * (int64_t)block + 1) * part_stride + c + i];
#pragma unroll
  for (int w = 0; w < kJoinWaves; ++w)
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] += shares[w][lane][i];
  put_sum<O, N>(out + (int64_t)token * out_stride, sum, scale, accumulate, c, width);
}

// lanes for a row: the power of two of them, at most a workgroup's, that a row of `vectors` has work for
int row_lanes_shift(int64_t vectors) {
  int shift = 0;
  while (shift < 8 && (1ll << shift) < vectors) ++shift;
  return shift;
}

// From here on chunks are summed in a launch of their own.
constexpr int64_t kManyBlocks = 1024;

struct GradWorkspace {
  size_t sorted[2], counts, parts, total, bytes;
  int64_t part_stride, tiles, blocks;
};

GradWorkspace grad_workspace(int64_t width, int64_t n_tokens) {
  GradWorkspace w;
  w.tiles = std::max<int64_t>(1, ceil_div(n_tokens, kSortTile));
  w.blocks = ceil_div(n_tokens, kBlock);
  w.part_stride = (int64_t)round_up((size_t)width, 8);
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t here = at; at = round_up(at + bytes, 256); return here; };
  for (size_t& s : w.sorted) s = take((size_t)n_tokens * sizeof(Occurrence));
  w.counts = take((size_t)w.tiles * kDigits * 4);
  w.total = take(4);
  w.parts = take((size_t)w.blocks * 2 * w.part_stride * 4);
  w.bytes = at;
  return w;
}

}  // namespace
}  // namespace fpsched

using namespace fpsched;

extern "C" {

int fpsched_op_embedding(int device_id, int type, const void* table, int64_t table_stride, int64_t n_rows, int64_t width,
                         const void* tokens, int tokens64, int64_t n_tokens, float scale, void* out, int64_t out_stride,
                         void* hip_stream) {
  if (type < FPSCHED_BF16 || type > FPSCHED_F32 || n_rows < 0 || width < 0 || width > kMaxWidth || n_tokens < 0 || n_tokens > 0x7fffffffll) return FPSCHED_EINVAL;
  if (table_stride < width || out_stride < width) return FPSCHED_EINVAL;
  if (device_id < 0) return FPSCHED_ENODEV;
  if (n_tokens == 0 || width == 0) return FPSCHED_OK;
  const size_t element = type == FPSCHED_F32 ? 4 : 2;
  if ((n_rows > 0 && !table) || !tokens || !out || !aligned(table, element) || !aligned(out, element)) return FPSCHED_EINVAL;
  OpsDevice g(device_id);
  if (!g.ok) return FPSCHED_EHIP;
  return with_type(type, [&](auto zero) {
    using T = decltype(zero);
    const int shift = row_lanes_shift(ceil_div(width, kWide<T>));
    embedding_kernel<T><<<dim3((unsigned)std::min(kMostGroups, ceil_div(n_tokens, kThreads >> shift))), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream)>>>(
        static_cast<const T*>(table), table_stride, n_rows, width, tokens, tokens64, n_tokens, scale, static_cast<T*>(out), out_stride, shift);
    return launched();
  });
}

size_t fpsched_op_embedding_grad_workspace_bytes(int64_t n_rows, int64_t width, int64_t n_tokens) {
  if (n_rows < 0 || width < 0 || width > kMaxWidth || n_tokens < 0 || n_rows > kMostRows || n_tokens >= kMaxSummed) return 0;
  return grad_workspace(width, n_tokens).bytes;
}

int fpsched_op_embedding_grad(int device_id, int type, const void* grad, int64_t grad_stride, int64_t n_rows, int64_t width,
                              const void* tokens, int tokens64, int64_t n_tokens, float scale, int out_type, void* out,
                              int64_t out_stride, int accumulate, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  if (type < FPSCHED_BF16 || type > FPSCHED_F32 || (out_type != type && out_type != FPSCHED_F32)) return FPSCHED_EINVAL;
  if (accumulate && out_type != FPSCHED_F32) return FPSCHED_EINVAL;
  if (n_rows < 0 || width < 0 || width > kMaxWidth || n_tokens < 0 || n_rows > kMostRows || n_tokens >= kMaxSummed) return FPSCHED_EINVAL;
  if (grad_stride < width || out_stride < width) return FPSCHED_EINVAL;
  if (device_id < 0) return FPSCHED_ENODEV;
  if (n_rows == 0 || width == 0) return FPSCHED_OK;
  if (!out || (n_tokens > 0 && (!grad || !tokens)) || !d_workspace || !aligned(d_workspace, 16)) return FPSCHED_EINVAL;
  if (!aligned(out, out_type == FPSCHED_F32 ? 4 : 2) || !aligned(grad, type == FPSCHED_F32 ? 4 : 2)) return FPSCHED_EINVAL;
  const GradWorkspace w = grad_workspace(width, n_tokens);
  if (workspace_bytes < w.bytes) return FPSCHED_ENOMEM;
  OpsDevice g(device_id);
  if (!g.ok) return FPSCHED_EHIP;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  char* base = static_cast<char*>(d_workspace);
  unsigned *counts = reinterpret_cast<unsigned*>(base + w.counts), *total = reinterpret_cast<unsigned*>(base + w.total);
  float* parts = reinterpret_cast<float*>(base + w.parts);
  // zeros everywhere, in slices beside the kernels that sort
  const int out_size = out_type == FPSCHED_F32 ? 4 : 2;
  Fill fill = {};
  if (!accumulate) {
    fill.out = static_cast<char*>(out);
    const bool adjacent = out_stride == width || n_rows == 1;
    fill.rows = adjacent ? 1 : n_rows;
    fill.row_bytes = (adjacent ? n_rows : 1) * width * out_size;
    fill.stride_bytes = out_stride * out_size;
    fill.wide = aligned(out, 16) && (adjacent || out_stride * out_size % 16 == 0);
    fill.element = out_size;
  }
  auto grid = [&](int64_t groups, int threads) {   // the kernel's own workgroups and those that fill
    fill.first = (unsigned)groups;
    const int64_t fillers = !fill.out ? 0 : std::min<int64_t>(2048 * 256 / threads, ceil_div(fill.rows * ceil_div(fill.row_bytes, 16), (int64_t)threads * 4 * fill.slices) + 1);
    return dim3((unsigned)(groups + fillers));
  };
  const Occurrence* sorted = reinterpret_cast<const Occurrence*>(base + w.sorted[0]);
  // (Of more than 8,192 one workgroup takes longer than many in several launches, 57 and 45 us for 16,000 tokens into 5,000 x 512, but where it is done before
  // the zeros are, those go faster in one launch: 281 and 324 us for 16,384 into 262,144 x 2,560, 55 and 71 for 8,300 into 70,000 x 512 of 32 bits.)
  const bool many_zeros = fill.out && n_rows * width * out_size >= 64 << 20;
  if (n_tokens <= (many_zeros ? kOneSort : kOneSort / 2)) {
    fill.slices = 1;
    const dim3 groups = grid(1, 1024);
    auto sort = [&](auto rounds) {
      sort_few_kernel<decltype(rounds)::value><<<groups, dim3(1024), 0, stream>>>(tokens, tokens64, (int)n_tokens, n_rows, reinterpret_cast<Occurrence*>(base + w.sorted[0]), total, fill);
    };
    if (n_tokens <= 1024 * 4) sort(std::integral_constant<int, 4>());
    else if (n_tokens <= 1024 * 8) sort(std::integral_constant<int, 8>());
    else sort(std::integral_constant<int, kMostRounds>());
  } else {
    int passes = 1;
    while ((n_rows - 1) >> 8 * passes) ++passes;
    fill.slices = 3 * passes;
    SortSource src{tokens, tokens64, n_tokens, n_rows, nullptr, total};
    for (int pass = 0; pass < passes; ++pass) {
      Occurrence* placed = reinterpret_cast<Occurrence*>(base + w.sorted[pass & 1]);
      const dim3 many = grid(w.tiles, kThreads);
      sort_count_kernel<<<many, dim3(kThreads), 0, stream>>>(src, 8 * pass, counts, fill);
      ++fill.slice;
      const dim3 one = grid(1, 1024);
      sort_scan_kernel<<<one, dim3(1024), 0, stream>>>(counts, w.tiles * kDigits, total, fill);
      ++fill.slice;
      fill.first = (unsigned)w.tiles;
      sort_place_kernel<<<many, dim3(kThreads), 0, stream>>>(src, 8 * pass, counts, placed, fill);
      ++fill.slice;
      src.sorted = sorted = placed;
    }
  }
  return with_type(type, [&](auto zero) {
    using T = decltype(zero);
    return with_type(out_type, [&](auto zero_out) {
      using O = decltype(zero_out);
      if constexpr (!std::is_same<O, T>::value && !std::is_same<O, float>::value) {
        return (int)FPSCHED_EINVAL;
      } else {
        constexpr int N = kWide<T>;
        if (w.blocks) {
          const unsigned pieces = (unsigned)ceil_div(width, 64 * N);
          for (int64_t at = 0; at < w.blocks; at += kMostWaves)
            row_sums_kernel<T, O, N><<<dim3((unsigned)std::min(kMostWaves, w.blocks - at), pieces), dim3(64), 0, stream>>>(
                static_cast<const T*>(grad), grad_stride, width, sorted, total, scale, static_cast<O*>(out), out_stride, accumulate, parts, w.part_stride, (unsigned)at);
          auto join = [&](auto chunks) {
            for (int64_t at = 0; at < w.blocks; at += kMostGroups)
              join_runs_kernel<O, N, decltype(chunks)::value><<<dim3((unsigned)std::min(kMostGroups, w.blocks - at), pieces), dim3(kJoinWaves * 64), 0, stream>>>(
                  sorted, total, width, parts, w.part_stride, scale, static_cast<O*>(out), out_stride, accumulate, (unsigned)at);
          };
          if (w.blocks > kManyBlocks) {
            chunk_sums_kernel<N><<<dim3((unsigned)ceil_div(w.blocks, kChunk), pieces), dim3(64), 0, stream>>>(sorted, total, width, parts, w.part_stride);
            join(std::true_type());
          } else {
            join(std::false_type());
          }
        }
        return launched();
      }
    });
  });
}

}  // extern "C"
