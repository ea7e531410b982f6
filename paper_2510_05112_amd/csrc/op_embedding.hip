// Embedding lookup of a model's first stage, and the gradient of its table.
//
// Lookup: out[t] = scale table[tokens[t]].  A row is moved by a power of two of lanes, 16 bytes a lane where rows are
// 16-byte aligned (else an element a lane); bound by memory for many tokens, by one load behind another (token, row) for few.
//
// Gradient: dE[v] = scale sum over {t : tokens[t] = v} grad[t].  Adding rows with atomics would make the sums depend on
// their order; here the occurrences are sorted by token (a stable counting sort, 8 bits of the token a pass), so that each row of
// dE is the sum of a run of sorted occurrences, and every row is written once.  Text repeats its few commonest tokens thousands of times: so that a
// run's length bounds nothing, the sorted occurrences are cut into blocks of 32 without regard to runs, each summed by
// workgroups of its own; a run inside one block is written where it belongs, one across blocks leaves its part (32 bits) in the workspace, and the pass
// that writes the rows without a token adds the parts up.  Floor: grad read once, dE written once.
#include "ops_common.h"

namespace fpsched {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kMaxWidth = 1 << 20;   // (what the grids have room for)

// ---- lookup ----------------------------------------------------------------------------------------------------------

template <typename T, int N>
__global__ __launch_bounds__(kThreads) void embedding_kernel(const T* table, int64_t table_stride, int64_t n_rows, int64_t width,
                                                            const void* tokens, int tokens64, int64_t n_tokens, float scale, T* out,
                                                            int64_t out_stride, int lanes_shift) {
  const int64_t t = ((int64_t)blockIdx.x << (8 - lanes_shift)) + (threadIdx.x >> lanes_shift);
  if (t >= n_tokens) return;
  const int64_t token = token_at(tokens, tokens64, t);
  const bool real = token >= 0 && token < n_rows;
  const T* from = table + (real ? token * table_stride : 0);
  T* to = out + t * out_stride;
  const int lanes = 1 << lanes_shift;
  for (int64_t c = (int64_t)(threadIdx.x & (lanes - 1)) * N; c < width; c += (int64_t)lanes * N) {
    if (c + N <= width) {
      Vec<T, N> v = {};
      if (real) {
        v = load_vec<T, N>(from + c);
#pragma unroll
        for (int i = 0; i < N; ++i) v.at[i] = (T)((float)v.at[i] * scale);
      }
      store_vec<T, N>(to + c, v);
    } else {
      for (int64_t i = c; i < width; ++i) to[i] = real ? (T)((float)from[i] * scale) : (T)0.f;
    }
  }
}

// ---- sorting the occurrences -------------------------------------------------------------------------------------------

constexpr int kDigits = 256, kSortRounds = 8;
constexpr int kSortTile = kThreads * kSortRounds;   // occurrences a workgroup places

struct Occurrence {
  unsigned token, at;
};

// An occurrence to be sorted: of the first pass from the tokens (those outside the table are none), later of the pass before
// (`n` of them).
struct SortSource {
  const void* tokens;
  int tokens64;
  int64_t n_tokens, n_rows;
  const Occurrence* sorted;
  const unsigned* n;

  __device__ __forceinline__ bool get(int64_t i, Occurrence* o) const {
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
__global__ __launch_bounds__(kThreads) void sort_count_kernel(SortSource src, int shift, unsigned* counts) {
  __shared__ unsigned held[kDigits];
  held[threadIdx.x] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * kSortTile;
  for (int r = 0; r < kSortRounds; ++r) {
    Occurrence o;
    if (src.get(first + r * kThreads + threadIdx.x, &o)) atomicAdd(&held[(o.token >> shift) & (kDigits - 1)], 1u);
  }
  __syncthreads();
  counts[(int64_t)threadIdx.x * gridDim.x + blockIdx.x] = held[threadIdx.x];
}

// counts -> the place of the first occurrence of each (digit, workgroup); *total: how many there are
__global__ __launch_bounds__(1024) void sort_scan_kernel(unsigned* counts, int64_t n, unsigned* total) {
  __shared__ unsigned waves[16];
  unsigned before = 0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t at = 0; at < n; at += 4096) {
    const int64_t mine = at + threadIdx.x * 4;
    unsigned c[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
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
    for (int i = 0; i < 4; ++i) {
      if (mine + i < n) counts[mine + i] = base;
      base += c[i];
    }
    before += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) *total = before;
}

// Places a workgroup's occurrences in order.  Each wavefront takes a piece of them, counts its digits first (lanes with one
// digit find each other by eight ballots), and places them behind those of the wavefronts in front of it.
__global__ __launch_bounds__(kThreads) void sort_place_kernel(SortSource src, int shift, const unsigned* places, Occurrence* out) {
  __shared__ unsigned next[kThreads / 64][kDigits];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int w = 0; w < kThreads / 64; ++w) next[w][threadIdx.x] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * kSortTile + wave * 64 * kSortRounds + lane;
  Occurrence o[kSortRounds];
  unsigned rank[kSortRounds];
  bool have[kSortRounds];
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    have[r] = src.get(first + r * 64, &o[r]);
    const unsigned digit = (o[r].token >> shift) & (kDigits - 1);
    unsigned long long same = __ballot(have[r]);
#pragma unroll
    for (int b = 0; b < 8; ++b) {
      const unsigned long long ones = __ballot(have[r] && (digit >> b & 1));
      same &= digit >> b & 1 ? ones : ~ones;
    }
    const int ahead = __popcll(same & ((1ull << lane) - 1));
    unsigned base = 0;
    if (have[r]) base = next[wave][digit];
    __builtin_amdgcn_wave_barrier();
    if (have[r] && ahead == 0) next[wave][digit] = base + __popcll(same);
    __builtin_amdgcn_wave_barrier();
    rank[r] = base + ahead;
  }
  __syncthreads();
  unsigned at = places[(int64_t)threadIdx.x * gridDim.x + blockIdx.x];
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

// starts[v]: the first sorted occurrence of a token >= v
__global__ __launch_bounds__(kThreads) void row_starts_kernel(const Occurrence* sorted, const unsigned* n, int64_t n_rows, unsigned* starts) {
  const int64_t v = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (v > n_rows) return;
  unsigned low = 0, high = *n;
  while (low < high) {
    const unsigned mid = (low + high) >> 1;
    if (sorted[mid].token < (unsigned)v) low = mid + 1; else high = mid;
  }
  starts[v] = low;
}

// ---- sums --------------------------------------------------------------------------------------------------------------

constexpr int kBlock = 32;   // sorted occurrences that are summed in one go

template <typename O, int N>
__device__ __forceinline__ void put_sum(O* out, const float* sum, float scale, int accumulate, int64_t c, int64_t width) {
  if (c + N <= width) {
    Vec<O, N> v = {};
    if (accumulate) v = load_vec<O, N>(out + c);
#pragma unroll
    for (int i = 0; i < N; ++i) v.at[i] = (O)((accumulate ? (float)v.at[i] : 0.f) + sum[i] * scale);
    store_vec<O, N>(out + c, v);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (c + i < width) out[c + i] = (O)((accumulate ? (float)out[c + i] : 0.f) + sum[i] * scale);
  }
}

// blockIdx.x: block of sorted occurrences, blockIdx.y: piece of the width.  Part 2 b: of the run that block b begins in
// the middle of, 2 b + 1: of the run that goes on behind it.
template <typename T, typename O, int N>
__global__ __launch_bounds__(64) void row_sums_kernel(const T* grad, int64_t grad_stride, int64_t width, const Occurrence* sorted,
                                                     const unsigned* n, const unsigned* starts, float scale, O* out, int64_t out_stride,
                                                     int accumulate, float* parts, int64_t part_stride) {
  const unsigned first = blockIdx.x * (unsigned)kBlock, all = *n;
  if (first >= all) return;
  const unsigned end = min(first + kBlock, all);
  const int64_t c = ((int64_t)blockIdx.y * 64 + threadIdx.x) * N;
  if (c >= width) return;
  const bool whole = c + N <= width;
  float sum[N] = {};
  auto flush = [&](unsigned token) {
    const unsigned from = starts[token], to = starts[token + 1];
    if (from >= first && to <= end) {
      put_sum<O, N>(out + (int64_t)token * out_stride, sum, scale, accumulate, c, width);
    } else {
      float* part = parts + (2 * (int64_t)blockIdx.x + (from >= first)) * part_stride + c;   // (part_stride has room for whole vectors)
#pragma unroll
      for (int i = 0; i < N; ++i) part[i] = sum[i];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = 0.f;
  };
  unsigned now = sorted[first].token;
  constexpr int kAhead = 8;
  for (unsigned at = first; at < end; at += kAhead) {
    Occurrence o[kAhead];
    Vec<T, N> v[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      o[i] = sorted[min(at + i, end - 1)];
      const T* from = grad + (int64_t)o[i].at * grad_stride + c;
      if (whole) {
        v[i] = load_vec<T, N>(from);
      } else {
        v[i] = {};
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (c + e < width) v[i].at[e] = from[e];
      }
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (at + i >= end) break;
      if (o[i].token != now) {
        flush(now);
        now = o[i].token;
      }
#pragma unroll
      for (int e = 0; e < N; ++e) sum[e] += (float)v[i].at[e];
    }
  }
  flush(now);
}

// The rows that no block wrote: without a token, or with a run across blocks, whose parts are added up.
template <typename O, int N>
__global__ __launch_bounds__(kThreads) void row_rest_kernel(const unsigned* starts, int64_t n_rows, int64_t width, const float* parts,
                                                           int64_t part_stride, float scale, O* out, int64_t out_stride, int accumulate,
                                                           int lanes_shift) {
  const int64_t v = ((int64_t)blockIdx.x << (8 - lanes_shift)) + (threadIdx.x >> lanes_shift);
  if (v >= n_rows) return;
  const unsigned from = starts[v], to = starts[v + 1];
  const int lanes = 1 << lanes_shift;
  const bool none = from == to;
  if (none ? accumulate != 0 : from / kBlock == (to - 1) / kBlock) return;
  for (int64_t c = (int64_t)(threadIdx.x & (lanes - 1)) * N; c < width; c += (int64_t)lanes * N) {
    float sum[N] = {};
    if (!none) {
      const unsigned b0 = from / kBlock, b1 = (to - 1) / kBlock;
      for (unsigned b = b0; b <= b1; ++b) {
        const float* part = parts + (2 * (int64_t)b + (b == b0)) * part_stride + c;
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] += part[i];
      }
    }
    put_sum<O, N>(out + v * out_stride, sum, scale, accumulate, c, width);
  }
}

// lanes for a row: the power of two of them, at most a workgroup's, that a row of `vectors` has work for
int row_lanes_shift(int64_t vectors) {
  int shift = 0;
  while (shift < 8 && (1ll << shift) < vectors) ++shift;
  return shift;
}

struct GradWorkspace {
  size_t sorted[2], counts, starts, parts, total, bytes;
  int64_t part_stride, tiles, blocks;
};

GradWorkspace grad_workspace(int64_t n_rows, int64_t width, int64_t n_tokens) {
  GradWorkspace w;
  w.tiles = ceil_div(n_tokens, kSortTile);
  w.blocks = ceil_div(n_tokens, kBlock);
  w.part_stride = (int64_t)round_up((size_t)width, 8);
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t here = at; at = round_up(at + bytes, 256); return here; };
  for (size_t& s : w.sorted) s = take((size_t)n_tokens * sizeof(Occurrence));
  w.counts = take((size_t)w.tiles * kDigits * 4);
  w.total = take(4);
  w.starts = take((size_t)(n_rows + 1) * 4);
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
  if ((n_rows > 0 && !table) || !tokens || !out) return FPSCHED_EINVAL;
  OpsDevice g(device_id);
  if (!g.ok) return FPSCHED_EHIP;
  return with_type(type, [&](auto zero) {
    using T = decltype(zero);
    auto go = [&](auto n) {
      constexpr int N = decltype(n)::value;
      const int shift = row_lanes_shift(ceil_div(width, N));
      embedding_kernel<T, N><<<dim3((unsigned)ceil_div(n_tokens, kThreads >> shift)), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream)>>>(
          static_cast<const T*>(table), table_stride, n_rows, width, tokens, tokens64, n_tokens, scale, static_cast<T*>(out), out_stride, shift);
      return launched();
    };
    if (wide_rows(table, table_stride, sizeof(T)) && wide_rows(out, out_stride, sizeof(T))) return go(std::integral_constant<int, kWide<T>>());
    return go(std::integral_constant<int, 1>());
  });
}

size_t fpsched_op_embedding_grad_workspace_bytes(int64_t n_rows, int64_t width, int64_t n_tokens) {
  if (n_rows < 0 || width < 0 || width > kMaxWidth || n_tokens < 0 || n_rows > 0x7ffffffell || n_tokens > 0x7fffffffll) return 0;
  return grad_workspace(n_rows, width, n_tokens).bytes;
}

int fpsched_op_embedding_grad(int device_id, int type, const void* grad, int64_t grad_stride, int64_t n_rows, int64_t width,
                              const void* tokens, int tokens64, int64_t n_tokens, float scale, int out_type, void* out,
                              int64_t out_stride, int accumulate, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  if (type < FPSCHED_BF16 || type > FPSCHED_F32 || (out_type != type && out_type != FPSCHED_F32)) return FPSCHED_EINVAL;
  if (accumulate && out_type != FPSCHED_F32) return FPSCHED_EINVAL;
  if (n_rows < 0 || width < 0 || width > kMaxWidth || n_tokens < 0 || n_rows > 0x7ffffffell || n_tokens > 0x7fffffffll) return FPSCHED_EINVAL;
  if (grad_stride < width || out_stride < width) return FPSCHED_EINVAL;
  if (device_id < 0) return FPSCHED_ENODEV;
  if (n_rows == 0 || width == 0) return FPSCHED_OK;
  if (!out || (n_tokens > 0 && (!grad || !tokens)) || !d_workspace || !aligned(d_workspace, 16)) return FPSCHED_EINVAL;
  const GradWorkspace w = grad_workspace(n_rows, width, n_tokens);
  if (workspace_bytes < w.bytes) return FPSCHED_ENOMEM;
  OpsDevice g(device_id);
  if (!g.ok) return FPSCHED_EHIP;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  char* base = static_cast<char*>(d_workspace);
  unsigned *counts = reinterpret_cast<unsigned*>(base + w.counts), *total = reinterpret_cast<unsigned*>(base + w.total);
  unsigned* starts = reinterpret_cast<unsigned*>(base + w.starts);
  float* parts = reinterpret_cast<float*>(base + w.parts);
  SortSource src{tokens, tokens64, n_tokens, n_rows, nullptr, total};
  int which = 0;
  for (int shift = 0; shift == 0 || (n_rows - 1) >> shift != 0; shift += 8, which ^= 1) {
    if (w.tiles) sort_count_kernel<<<dim3((unsigned)w.tiles), dim3(kThreads), 0, stream>>>(src, shift, counts);
    sort_scan_kernel<<<dim3(1), dim3(1024), 0, stream>>>(counts, w.tiles * kDigits, total);
    Occurrence* placed = reinterpret_cast<Occurrence*>(base + w.sorted[which]);
    if (w.tiles) sort_place_kernel<<<dim3((unsigned)w.tiles), dim3(kThreads), 0, stream>>>(src, shift, counts, placed);
    src.sorted = placed;
  }
  row_starts_kernel<<<dim3((unsigned)ceil_div(n_rows + 1, kThreads)), dim3(kThreads), 0, stream>>>(src.sorted, total, n_rows, starts);
  return with_type(type, [&](auto zero) {
    using T = decltype(zero);
    return with_type(out_type, [&](auto zero_out) {
      using O = decltype(zero_out);
      if constexpr (!std::is_same<O, T>::value && !std::is_same<O, float>::value) {
        return (int)FPSCHED_EINVAL;
      } else {
        auto go = [&](auto n) {
          constexpr int N = decltype(n)::value;
          if (w.blocks)
            row_sums_kernel<T, O, N><<<dim3((unsigned)w.blocks, (unsigned)ceil_div(width, 64 * N)), dim3(64), 0, stream>>>(
                static_cast<const T*>(grad), grad_stride, width, src.sorted, total, starts, scale, static_cast<O*>(out), out_stride, accumulate,
                parts, w.part_stride);
          const int shift = row_lanes_shift(ceil_div(width, N));
          row_rest_kernel<O, N><<<dim3((unsigned)ceil_div(n_rows, kThreads >> shift)), dim3(kThreads), 0, stream>>>(
              starts, n_rows, width, parts, w.part_stride, scale, static_cast<O*>(out), out_stride, accumulate, shift);
          return launched();
        };
        // (16 bytes of the gradient a lane, and as many elements of the output: of 32 bits two pieces of 16 bytes)
        if (wide_rows(grad, grad_stride, sizeof(T)) && aligned(out, sizeof(O) * kWide<T>) && out_stride % kWide<T> == 0)
          return go(std::integral_constant<int, kWide<T>>());
        return go(std::integral_constant<int, 1>());
      }
    });
  });
}

}  // extern "C"
