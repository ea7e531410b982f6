// Log probabilities of given tokens, the entropy and the likeliest alternatives, in one pass over the logits, and the gradient.
//
// With m the largest logit of what was seen, s = sum e^(x - m) and w = sum e^(x - m) (x - m), what is asked for is
//   log p[token] = (x[token] - m) - log s,   entropy = log s - w / s,
// and two parts of a row are put together by multiplying s by e^(m1 - m) and adding s (m1 - m) to w.  A lane looks at 16
// bytes of logits at a time and changes its m only where one of them is larger.  Rows are cut into parts where there are fewer rows than
// the chip has room for; a second kernel puts the parts together.  Bound by memory for many rows (4,096 x 65,536 bf16: 105 us, 5.1 TB/s), for few by
// ten instructions a logit and by what each part costs beside its logits (61 x 262,144: 15.5 us and 4.9 for the parts).
//
// Alternatives: of 32 groups of lanes each has a largest logit, and k logits at least are
// not below the k-th of these, the bar; each lane knows the largest of each of its pieces, and the pieces with one that is not below the bar are
// read once more (from cache: there are about as many as alternatives) and those logits collected in LDS.  Each finds its place by counting the larger
// ones.  Equal logits come by ascending id: a candidate is the logit's bits, in an order in which they compare as integers, with the id behind.
// Where too many are not below the bar (a row of one value) the k-th largest is found digit by digit (509 x 100,003 equal f16 logits: 258 us, and
// 514 where the k were found one by one).  The parts' candidates, which are in order, are put together by a bar of their own (1 x 4,500,000 f16, k 32: 31 us,
// and 2,030 without).  (With the pieces kept in registers instead, there was room for five wavefronts a SIMD and twice the code: 18.5 against 14.8 us for
// 61 x 262,144 bf16, 43.8 against 35.3 for 509 x 100,003 f16, 164 against 93 for 1,000 x 128,000 f32.)
//
// Masked logits are minus infinity, and x - m = -infinity gives e = 0, but 0 times it is NaN: factors are held at -1000.  m begins at the
// type's lowest number and not at minus infinity, so that a row of masks needs no branch: its s stays 0.
//
// Gradient: one pass, element by element, bound by memory (4,096 x 65,536 bf16: 180 us, 6.0 TB/s).
#include "ops_common.h"

#include <float.h>

#include <algorithm>

namespace fpsched {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMostAlternatives = 32;
constexpr int kHeld = 64;                              // logits of a lane where alternatives are wanted (32: 149 against 131 us for 2,000 x 50,257 f16, k 32)
constexpr int64_t kHeldPart = (int64_t)kThreads * kHeld;

__device__ __forceinline__ float held_back(float x) { return fmaxf(x, -1000.f); }   // (of what is no number -1000, and its e^x none)

struct Stats {
  float m, s, w;

  __device__ __forceinline__ void raise(float to) {
    const float d = held_back(m - to), f = fast_exp(d);
    w = f * (w + s * d);
    s *= f;
    m = to;
  }
  __device__ __forceinline__ void add(float x) {   // x <= m, or not a number
    const float e = fast_exp(x - m);
    s += e;
    w += e * held_back(x - m);
  }
};

__device__ __forceinline__ Stats nothing() { return {-FLT_MAX, 0.f, 0.f}; }

// The value of the lane across: of steps 1, 2, 4, ... in turn, where the values of each group of STEP lanes are the same already, lanes of the
// other group of STEP.
template <int STEP>
__device__ __forceinline__ float across(float x) {
  const int i = __float_as_int(x);
  if constexpr (STEP == 1) return __int_as_float(__builtin_amdgcn_update_dpp(i, i, 0xb1, 0xf, 0xf, false));        // neighbours in pairs
  else if constexpr (STEP == 2) return __int_as_float(__builtin_amdgcn_update_dpp(i, i, 0x4e, 0xf, 0xf, false));   // pairs in fours
  else if constexpr (STEP == 4) return __int_as_float(__builtin_amdgcn_update_dpp(i, i, 0x141, 0xf, 0xf, false));  // eights mirrored
  else if constexpr (STEP == 8) return __int_as_float(__builtin_amdgcn_update_dpp(i, i, 0x140, 0xf, 0xf, false));  // sixteens mirrored
  else if constexpr (STEP == 16) return __int_as_float(__builtin_amdgcn_ds_swizzle(i, 0x401f));
  else return __shfl_xor(x, 32);
}
template <typename F>
__device__ __forceinline__ float over_lanes(float x, F f) {
  x = f(x, across<1>(x));
  x = f(x, across<2>(x));
  x = f(x, across<4>(x));
  x = f(x, across<8>(x));
  x = f(x, across<16>(x));
  return f(x, across<32>(x));
}
// The lanes' sums put together.
__device__ __forceinline__ Stats wave_stats(Stats a) {
  auto add = [](float x, float y) { return x + y; };
  a.raise(over_lanes(a.m, [](float x, float y) { return fmaxf(x, y); }));
  a.s = over_lanes(a.s, add);
  a.w = over_lanes(a.w, add);
  return a;
}
// The sums of WAVES wavefronts, by each lane.
template <int WAVES>
__device__ __forceinline__ Stats put_together(const Stats* wave_sums, int lane) {
  static_assert(WAVES == 1 || WAVES == 4, "the lanes are taken in fours");
  if (WAVES == 1) return wave_sums[0];
  Stats a = wave_sums[lane & 3];
  float most = fmaxf(a.m, across<1>(a.m));
  a.raise(fmaxf(most, across<2>(most)));
  a.s += across<1>(a.s);
  a.s += across<2>(a.s);
  a.w += across<1>(a.w);
  a.w += across<2>(a.w);
  return a;
}
// A number that is larger for a larger x (not 0 for any that is a number).
__device__ __forceinline__ unsigned in_order(float x) {
  const unsigned bits = __float_as_uint(x);
  return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}
__device__ __forceinline__ float out_of_order(unsigned order) { return __uint_as_float(order & 0x80000000u ? order & 0x7fffffffu : ~order); }

// A logit and its id as one number: larger for a larger logit, then for a smaller id.  0: none.
__device__ __forceinline__ unsigned long long ranked(float x, unsigned id) { return (unsigned long long)in_order(x) << 32 | (unsigned)~id; }
__device__ __forceinline__ float logit_of(unsigned long long r) { return out_of_order((unsigned)(r >> 32)); }
__device__ __forceinline__ unsigned long long wave_most(unsigned long long a) {
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    const unsigned long long o = __shfl_xor(a, d);
    a = o > a ? o : a;
  }
  return a;
}

constexpr int kGroups = 32;   // of the lanes of one number modulo 32: neighbouring logits are in different ones, and a part of 256 has some in each
static_assert(kMostAlternatives <= kGroups, "as many groups of lanes as alternatives");
constexpr int kRoom = 512;   // candidates in LDS
constexpr int kDigits = 256;

// put(place, candidate) if the at-th of n distinct candidates in LDS is one of the k largest.
template <typename P>
__device__ __forceinline__ void by_rank(const unsigned long long* candidates, int n, int k, int at, P put) {
  const unsigned long long mine = at < n ? candidates[at] : 0;
  int larger = 0;
#pragma unroll 16
  for (int i = 0; i < n; ++i) larger += candidates[i] > mine;
  if (mine && larger < k) put(larger, mine);
}

struct PartOut {          // [row][part]
  Stats* stats;
  unsigned long long* best;   // [row][part][k], descending
  int parts;
};

// -0 and 0 are equal logits
template <typename T>
__device__ __forceinline__ float logit(T x) { return (float)x + 0.f; }

template <typename T>
struct RowOut {
  const T* logits;
  int64_t stride, vocab;
  const void* tokens;
  int tokens64, k;
  float *logprob, *entropy, *lse;
  int32_t* ids;
  float* alternatives;

  RowOut behind(int64_t rows) const {
    RowOut r = *this;
    r.logits += rows * stride;
    r.tokens = static_cast<const char*>(tokens) + rows * (tokens64 ? 8 : 4);
    r.logprob += rows, r.entropy += rows, r.lse += 2 * rows;
    if (k) r.ids += rows * k, r.alternatives += rows * k;
    return r;
  }
  // the given token's logit; 0 and false if it has none
  __device__ __forceinline__ float given(int64_t row, bool* is) const {
    const int64_t token = token_at(tokens, tokens64, row);
    *is = token >= 0 && token < vocab;
    return *is ? logit(logits[row * stride + token]) : 0.f;
  }
  __device__ __forceinline__ void put(int64_t row, const Stats& a, float x, bool is) const {
    const float ln = fast_log(a.s);
    const bool none = a.s == 0.f;
    float lp = 0.f;
    if (is) lp = none ? -INFINITY : (x - a.m) - ln;
    logprob[row] = a.s != a.s ? a.s : lp;
    entropy[row] = none ? 0.f : ln - a.w / a.s;
    lse[2 * row] = none ? 0.f : a.m;
    lse[2 * row + 1] = none ? -INFINITY : ln;
  }
  __device__ __forceinline__ void put_alternative(int64_t row, int i, unsigned long long r, const Stats& a) const {
    const float x = logit_of(r);
    const bool masked = r == 0 || x == -INFINITY, wrong = a.s != a.s;
    ids[row * k + i] = masked || wrong ? -1 : (int32_t)~(unsigned)r;
    alternatives[row * k + i] = wrong ? a.s : masked ? -INFINITY : (x - a.m) - fast_log(a.s);
  }
};

// One part of a row, by WAVES wavefronts.  blockIdx.x: row * parts + part.  ALT: with alternatives, of at most kHeld logits a lane.
template <typename T, bool ALT, int WAVES>
__global__ __launch_bounds__(WAVES * 64, sizeof(T) == 4 ? 5 : 6) void logprobs_kernel(RowOut<T> row_out, PartOut part_out, int64_t part_length) {
  constexpr int N = kWide<T>, kLanes = WAVES * 64;
  __shared__ Stats wave_sums[WAVES];
  __shared__ unsigned long long candidates[ALT ? kRoom : 1];
  __shared__ struct { unsigned digit, count, larger; } chosen;
  __shared__ unsigned group_tops[ALT ? WAVES : 1][kGroups];
  __shared__ int collected;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), k = row_out.k;
  const int64_t row = blockIdx.x / part_out.parts, part = blockIdx.x % part_out.parts;
  const T* logits = row_out.logits + row * row_out.stride;
  bool is_given = false;
  const float given = part_out.parts == 1 ? row_out.given(row, &is_given) : 0.f;   // (on its way while the row is read)
  // Pieces of 16 bytes that are aligned as such, from `inner` on, and up to N - 1 logits in front of them and behind them, one a lane.
  const int64_t begin = part * part_length, end = min(begin + part_length, row_out.vocab);
  const int64_t skew = (int64_t)((0 - reinterpret_cast<uintptr_t>(logits + begin)) % 16 / sizeof(T));
  const int64_t inner = min(begin + skew, end);
  const unsigned length = (unsigned)((end - inner) / N * N), mine_at = threadIdx.x * N;
  const int64_t outer = threadIdx.x < N ? begin + threadIdx.x : inner + length + threadIdx.x - N;
  const bool has_outer = threadIdx.x < N ? outer < inner : threadIdx.x < 2 * N && outer < end;
  const float x_outer = has_outer ? (float)logits[outer] : -INFINITY;
  auto get = [&](unsigned at) {
    Vec<T, N> v;
    if (at < length) {
      v = load_vec<T, N>(logits + inner + at);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) v.at[i] = (T)-INFINITY;
    }
    return v;
  };
  Stats mine = nothing();
  auto take = [&](const Vec<T, N>& v) {   // returns the largest
    float x[N], most = -INFINITY;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = (float)v.at[i];
      most = fmaxf(most, x[i]);
    }
    if (most > mine.m) mine.raise(most);
#pragma unroll
    for (int i = 0; i < N; ++i) mine.add(x[i]);
    return most;
  };
  constexpr int kPieces = kHeld / N;
  float tops[ALT ? kPieces : 1];   // the pieces' largest logits
  if constexpr (ALT) {
    Vec<T, N> v[kPieces];
#pragma unroll
    for (int p = 0; p < kPieces; ++p) v[p] = get(mine_at + p * kLanes * N);
#pragma unroll
    for (int p = 0; p < kPieces; ++p) tops[p] = (unsigned)(p * kLanes * N) < length ? take(v[p]) : -INFINITY;
  } else {
    constexpr int kAhead = 4;
    for (unsigned at = mine_at; at < length; at += kAhead * kLanes * N) {
      Vec<T, N> v[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) v[i] = get(at + i * kLanes * N);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) take(v[i]);
    }
  }
  if (wave == 0) {
    if (x_outer > mine.m) mine.raise(x_outer);
    mine.add(x_outer);
  }
  if constexpr (ALT) {
    const float most = fmaxf(mine.m, across<32>(mine.m));   // (the last bits give way to the group's number, so that no two are equal)
    if (lane < kGroups) group_tops[wave][lane] = (in_order(most) & ~(kGroups - 1u)) | lane;
    if (threadIdx.x == 0) collected = 0;
  }
  const Stats sums = wave_stats(mine);
  if (lane == 0) wave_sums[wave] = sums;
  __syncthreads();
  if constexpr (ALT) {
    unsigned mine_of_groups = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) mine_of_groups = max(mine_of_groups, group_tops[w][lane & (kGroups - 1)]);
    int larger = 0;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) larger += (unsigned)__builtin_amdgcn_readlane(mine_of_groups, g) > mine_of_groups;
    const unsigned long long at_bar = __ballot(larger == k - 1);
    // (at or a little below the k-th largest, and not below the lowest number: with no piece above that, the largest is taken as that)
    const float bar = out_of_order(__builtin_amdgcn_readlane(mine_of_groups, __builtin_ctzll(at_bar)) & ~(kGroups - 1u));
    unsigned again = 0;   // pieces of which a lane has one
#pragma unroll
    for (int p = 0; p < kPieces; ++p) again |= (unsigned)(__any(tops[p] >= bar) != 0) << p;
    auto add = [&](unsigned long long r) {
      const int place = atomicAdd(&collected, 1);   // (in any order: places among them are found by value)
      if (place < kRoom) candidates[place] = r;
    };
    auto collect = [&](float x, int64_t id) {
      if (x >= bar) add(ranked(x + 0.f, (unsigned)id));   // (what is masked or outside the part is minus infinity)
    };
    if (wave == 0) collect(x_outer, outer);
    for (; again; again &= again - 1) {
      const unsigned at = mine_at + __builtin_ctz(again) * kLanes * N;
      const Vec<T, N> v = get(at);
#pragma unroll
      for (int i = 0; i < N; ++i) collect((float)v.at[i], inner + at + i);
    }
    __syncthreads();
    if (collected > kRoom) {
      // Too many (more than kRoom equal logits, say): the k-th largest candidate's digits of eight bits are counted out, from the first on in which the
      // largest and the smallest that there can be differ, until few enough are not below what is known of it.
      auto all_of_part = [&](auto f) {
        auto one = [&](float x, int64_t id) {
          if (x > -INFINITY) f(ranked(x + 0.f, (unsigned)id));
        };
        if (wave == 0) one(x_outer, outer);
        for (unsigned at = mine_at; at < length; at += kLanes * N) {
          const Vec<T, N> v = get(at);
#pragma unroll
          for (int i = 0; i < N; ++i) one((float)v.at[i], inner + at + i);
        }
      };
      unsigned* counts = reinterpret_cast<unsigned*>(candidates);
      static_assert(!ALT || sizeof(candidates) >= kDigits * 4, "they fit");
      const unsigned long long largest = ranked(put_together<WAVES>(wave_sums, lane).m + 0.f, (unsigned)begin), smallest = ranked(bar, (unsigned)(end - 1));
      int shift = (63 - __builtin_clzll((largest ^ smallest) | 1)) & ~7;
      unsigned long long known = shift == 56 ? 0 : largest >> (shift + 8) << (shift + 8);
      unsigned wanted = k;   // of those that begin with what is known
      for (; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int d = threadIdx.x; d < kDigits; d += kLanes) counts[d] = 0;
        __syncthreads();
        all_of_part([&](unsigned long long r) {
          if (shift == 56 || (r ^ known) >> (shift + 8) == 0) {
            const unsigned digit = (unsigned)(r >> shift) & 255, of_first = __builtin_amdgcn_readfirstlane(digit);
            const unsigned long long here = __ballot(1);
            if (__ballot(digit == of_first) == here) {   // (as digits of equal logits are: one addition for all lanes)
              if (__builtin_ctzll(here) == lane) atomicAdd(&counts[digit], (unsigned)__popcll(here));
            } else {
              atomicAdd(&counts[digit], 1u);
            }
          }
        });
        __syncthreads();
        for (int digit = threadIdx.x; digit < kDigits; digit += kLanes) {
          unsigned larger = 0;
          for (int d = kDigits - 1; d >= 0; --d) larger += d > digit ? counts[d] : 0u;
          const unsigned count = counts[digit];
          if (larger < wanted && larger + count >= wanted) chosen = {(unsigned)digit, count, larger};
        }
        __syncthreads();
        known |= (unsigned long long)chosen.digit << shift;
        wanted -= chosen.larger;
        if (k - wanted + chosen.count <= kRoom) break;
      }
      if (threadIdx.x == 0) collected = 0;
      __syncthreads();
      all_of_part([&](unsigned long long r) {
        if (r >= known) add(r);
      });
      __syncthreads();
    }
  }
  const bool whole = part_out.parts == 1;
  const int64_t at = row * part_out.parts + part;
  const Stats all = whole || wave == 0 ? put_together<WAVES>(wave_sums, lane) : nothing();
  if (threadIdx.x == 0) {
    if (whole) row_out.put(row, all, given, is_given);
    else part_out.stats[at] = all;
  }
  if constexpr (ALT) {
    const int n = collected;
    auto put = [&](int i, unsigned long long r) {
      if (whole) row_out.put_alternative(row, i, r, all);
      else part_out.best[at * k + i] = r;
    };
    for (int first = wave * 64; first < n; first += kLanes) by_rank(candidates, n, k, first + lane, put);
    if ((int)threadIdx.x >= n && (int)threadIdx.x < k) put(threadIdx.x, 0);
  }
}

// The parts of a row put together.
template <typename T>
__global__ __launch_bounds__(kThreads) void logprobs_join_kernel(RowOut<T> row_out, PartOut part_out) {
  constexpr int kRoomOfParts = 1024;
  __shared__ unsigned long long candidates[kRoomOfParts];
  __shared__ unsigned long long tops[kThreads], bar;
  __shared__ Stats all;
  __shared__ int collected;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, k = row_out.k;
  const int64_t row = blockIdx.x;
  const int n = part_out.parts * k;
  const unsigned long long* best = part_out.best + row * n;
  if (threadIdx.x == 0) collected = 0;
  __syncthreads();
  auto add = [&](unsigned long long r) {
    if (r == 0) return;
    const int place = atomicAdd(&collected, 1);
    if (place < kRoomOfParts) candidates[place] = r;
  };
  if (n <= kThreads || part_out.parts < k) {   // (fewer parts than alternatives have fewer candidates than kMostAlternatives^2)
    for (int i = threadIdx.x; i < n; i += kThreads) add(best[i]);
  } else {
    // The parts' candidates are in order, so a part whose first one is below the bar has none; the bar is the k-th of the largest ones of the lanes' parts.
    // Up to kThreads parts, k of them at most are not below it.
    unsigned long long most = 0;
    for (int p = threadIdx.x; p < part_out.parts; p += kThreads) {
      const unsigned long long r = best[(int64_t)p * k];
      most = r > most ? r : most;
    }
    tops[threadIdx.x] = most;
    if (threadIdx.x == 0) bar = 1;
    __syncthreads();
    int larger = 0;
#pragma unroll 16
    for (int i = 0; i < kThreads; ++i) larger += tops[i] > most;
    if (most && larger == k - 1) bar = most;   // (fewer lanes that have one: all candidates, fewer than kMostAlternatives^2 up to kThreads parts)
    __syncthreads();
    for (int p = threadIdx.x; p < part_out.parts; p += kThreads) {
      for (int i = 0; i < k; ++i) {
        const unsigned long long r = best[(int64_t)p * k + i];
        if (r < bar) break;
        add(r);
      }
    }
  }
  if (wave == 0) {
    bool is_given;
    const float given = row_out.given(row, &is_given);
    Stats mine = nothing();
    for (int p = lane; p < part_out.parts; p += 64) {
      Stats other = part_out.stats[row * part_out.parts + p];
      const float most = fmaxf(mine.m, other.m);
      mine.raise(most);
      other.raise(most);
      mine.s += other.s;
      mine.w += other.w;
    }
    mine = wave_stats(mine);
    if (lane == 0) {
      all = mine;
      row_out.put(row, mine, given, is_given);
    }
  }
  __syncthreads();
  if (collected <= kRoomOfParts) {
    const int found = collected;
    for (int first = wave * 64; first < found; first += kThreads)
      by_rank(candidates, found, k, first + lane, [&](int i, unsigned long long r) { row_out.put_alternative(row, i, r, all); });
    if ((int)threadIdx.x >= found && (int)threadIdx.x < k) row_out.put_alternative(row, threadIdx.x, 0, all);
  } else if (wave == 0) {
    unsigned long long below = ~0ull;
    for (int i = 0; i < k; ++i) {
      unsigned long long most = 0;
      for (int j = lane; j < n; j += 64) {
        const unsigned long long r = best[j];
        if (r < below && r > most) most = r;
      }
      below = wave_most(most);
      if (lane == 0) row_out.put_alternative(row, i, below, all);
    }
  }
}

constexpr int kGradRounds = 4;
template <typename T>
__global__ __launch_bounds__(kThreads) void logprobs_grad_kernel(const T* logits, int64_t stride, int64_t vocab, const void* tokens,
                                                                int tokens64, const float* lse, const float* entropy,
                                                                const float* grad_logprob, const float* grad_entropy, T* out,
                                                                int64_t out_stride, int pieces, int64_t first_row) {
  const int64_t row = first_row + blockIdx.x / pieces;
  const int64_t token = token_at(tokens, tokens64, row);
  const bool given = token >= 0 && token < vocab;
  const float m = lse[2 * row], ln = lse[2 * row + 1];
  const float gl = given && grad_logprob ? grad_logprob[row] : 0.f, ge = grad_entropy ? grad_entropy[row] : 0.f, h = entropy[row];
  const T* from = logits + row * stride;
  T* to = out + row * out_stride;
  const bool none = ln == -INFINITY;
  auto gradient = [&](T x, bool is_token) {
    const float lp = ((float)x - m) - ln;
    const float p = fast_exp(lp);
    const float d = (is_token ? gl : 0.f) - p * (gl + ge * (held_back(lp) + h));
    return (T)(none ? 0.f : d);
  };
  // Pieces of 16 bytes that are aligned as such in the logits, and up to N - 1 elements in front of them and behind them, by the row's first workgroup
  // (509 x 100,003 f16: 34 us, and 56 an element a lane).
  constexpr int N = kWide<T>;
  const unsigned piece = blockIdx.x % pieces;
  const int64_t inner = min((int64_t)((0 - reinterpret_cast<uintptr_t>(from)) % 16 / sizeof(T)), vocab), length = (vocab - inner) / N * N;
  if (piece == 0 && threadIdx.x < 2 * N) {
    const int64_t i = threadIdx.x < N ? threadIdx.x : inner + length + threadIdx.x - N;
    if (threadIdx.x < N ? i < inner : i < vocab) to[i] = gradient(from[i], i == token);
  }
  const int64_t first = ((int64_t)piece * kGradRounds * kThreads + threadIdx.x) * N;
#pragma unroll
  for (int r = 0; r < kGradRounds; ++r) {
    const int64_t c = first + (int64_t)r * kThreads * N;
    if (c < length) {
      Vec<T, N> v = load_vec<T, N>(from + inner + c);
      const int64_t behind = token - inner - c;
      const int at = behind >= 0 && behind < N ? (int)behind : -1;   // the token's place in the piece
#pragma unroll
      for (int i = 0; i < N; ++i) v.at[i] = gradient(v.at[i], i == at);
      store_any<T, N>(to + inner + c, v);
    }
  }
}

// Rows that one wavefront takes, of more than kFewRows (4,096 x 4,000 bf16: 9.9 us, and 14.0 by four wavefronts a row; 4,096 x 1,500 f16, k 20: 12.1 and 18.3;
// but 300 x 3,000 f32, k 4: 7.1 and 6.3).
constexpr int64_t kShortRow = 4096, kFewRows = 512;
static_assert(kShortRow <= 64 * kHeld, "a wavefront holds a short row");

struct Parts {
  int64_t length;
  int parts;
};

// Parts of a row: with alternatives kHeld logits a lane, fewer where there are few rows (1,024 workgroups
// fill the chip), but 4,096 at least.
Parts parts_of(int64_t n_rows, int64_t vocab, int k) {
  const int64_t wanted = std::max<int64_t>(1, ceil_div(1024, std::max<int64_t>(1, n_rows)));
  int64_t length = std::max<int64_t>(4096, ceil_div(vocab, wanted));
  if (k > 0) length = std::min<int64_t>(length, kHeldPart);
  length = (int64_t)round_up((size_t)length, 64);
  Parts p;
  p.length = length;
  p.parts = (int)std::max<int64_t>(1, ceil_div(vocab, length));
  return p;
}

bool sizes_fit(int64_t n_rows, int64_t vocab, int k) {
  if (n_rows < 0 || n_rows > 0x7fffffffll || vocab < 1 || vocab > 0x7fffffffll || k < 0 || k > kMostAlternatives) return false;
  return n_rows * parts_of(n_rows, vocab, k).parts <= 0x7fffffffll;
}

}  // namespace
}  // namespace fpsched

using namespace fpsched;

extern "C" {

size_t fpsched_op_logprobs_workspace_bytes(int64_t n_rows, int64_t vocab, int n_alternatives) {
  if (!sizes_fit(n_rows, vocab, n_alternatives)) return 0;
  const Parts p = parts_of(n_rows, vocab, n_alternatives);
  if (p.parts == 1) return 16;
  return round_up((size_t)n_rows * p.parts * sizeof(Stats), 16) + (size_t)n_rows * p.parts * n_alternatives * 8;
}

int fpsched_op_logprobs(int device_id, int type, int64_t n_rows, int64_t vocab, const void* logits, int64_t logits_stride,
                        const void* tokens, int tokens64, int n_alternatives, float* logprob, float* entropy, float* lse,
                        int32_t* ids, float* alternatives, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  if (type < FPSCHED_BF16 || type > FPSCHED_F32 || !sizes_fit(n_rows, vocab, n_alternatives) || logits_stride < vocab) return FPSCHED_EINVAL;
  if (device_id < 0) return FPSCHED_ENODEV;
  if (n_rows == 0) return FPSCHED_OK;
  if (!logits || !tokens || !logprob || !entropy || !lse || (n_alternatives > 0 && (!ids || !alternatives))) return FPSCHED_EINVAL;
  if (!aligned(logits, type == FPSCHED_F32 ? 4 : 2)) return FPSCHED_EINVAL;
  const Parts p = parts_of(n_rows, vocab, n_alternatives);
  if (p.parts > 1) {
    if (!d_workspace || !aligned(d_workspace, 16)) return FPSCHED_EINVAL;
    if (workspace_bytes < fpsched_op_logprobs_workspace_bytes(n_rows, vocab, n_alternatives)) return FPSCHED_ENOMEM;
  }
  OpsDevice g(device_id);
  if (!g.ok) return FPSCHED_EHIP;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  return with_type(type, [&](auto zero) {
    using T = decltype(zero);
    RowOut<T> row{static_cast<const T*>(logits), logits_stride, vocab, tokens, tokens64, n_alternatives, logprob, entropy, lse, ids, alternatives};
    PartOut part{static_cast<Stats*>(d_workspace), nullptr, p.parts};
    if (p.parts > 1)
      part.best = reinterpret_cast<unsigned long long*>(static_cast<char*>(d_workspace) + round_up((size_t)n_rows * p.parts * sizeof(Stats), 16));
    const int64_t most = kMostGroups / p.parts;   // rows of a launch
    for (int64_t at = 0; at < n_rows; at += most) {
      const int64_t n = std::min(most, n_rows - at);
      const dim3 grid((unsigned)(n * p.parts));
      auto go = [&](auto waves) {
        constexpr int W = decltype(waves)::value;
        if (n_alternatives > 0) logprobs_kernel<T, true, W><<<grid, dim3(W * 64), 0, stream>>>(row, part, p.length);
        else logprobs_kernel<T, false, W><<<grid, dim3(W * 64), 0, stream>>>(row, part, p.length);
      };
      if (vocab <= kShortRow && n_rows > kFewRows) go(std::integral_constant<int, 1>());
      else go(std::integral_constant<int, kWaves>());
      if (p.parts > 1) logprobs_join_kernel<T><<<dim3((unsigned)n), dim3(kThreads), 0, stream>>>(row, part);
      row = row.behind(n);
    }
    return launched();
  });
}

int fpsched_op_logprobs_grad(int device_id, int type, int64_t n_rows, int64_t vocab, const void* logits, int64_t logits_stride,
                             const void* tokens, int tokens64, const float* lse, const float* entropy, const float* grad_logprob,
                             const float* grad_entropy, void* out, int64_t out_stride, void* hip_stream) {
  if (type < FPSCHED_BF16 || type > FPSCHED_F32 || !sizes_fit(n_rows, vocab, 0) || logits_stride < vocab || out_stride < vocab) return FPSCHED_EINVAL;
  if (device_id < 0) return FPSCHED_ENODEV;
  if (n_rows == 0) return FPSCHED_OK;
  const size_t element = type == FPSCHED_F32 ? 4 : 2;
  if (!logits || !tokens || !lse || !entropy || !out || (out == logits && out_stride != logits_stride)) return FPSCHED_EINVAL;
  if (!aligned(logits, element) || !aligned(out, element)) return FPSCHED_EINVAL;
  OpsDevice g(device_id);
  if (!g.ok) return FPSCHED_EHIP;
  return with_type(type, [&](auto zero) {
    using T = decltype(zero);
    const int64_t pieces = ceil_div(vocab, kGradRounds * kThreads * kWide<T>), most = kMostGroups / pieces;   // rows of a launch
    for (int64_t at = 0; at < n_rows; at += most)
      logprobs_grad_kernel<T><<<dim3((unsigned)(std::min(most, n_rows - at) * pieces)), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream)>>>(
          static_cast<const T*>(logits), logits_stride, vocab, tokens, tokens64, lse, entropy, grad_logprob, grad_entropy, static_cast<T*>(out),
          out_stride, (int)pieces, at);
    return launched();
  });
}

}  // extern "C"
