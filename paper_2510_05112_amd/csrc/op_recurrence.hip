// Gated linear recurrence:  h[t] = a[t] h[t-1] + (1 - a[t]) v[t],  a = sigmoid(gate), for each sequence and channel.
//
// A step is an affine map of the state, and maps compose: of a run of steps (A, S) with h_end = A h_begin + S, two runs one after the other
// have (A2 A1, A2 S1 + S2).  A workgroup walks a sequence in blocks of 64 steps for 64 lanes' channels (two adjacent ones a lane
// where strides allow): each wavefront loads a run of 16 steps (8 in the backward pass), works out its map, the maps go round through LDS, and
// each wavefront then takes its steps from the state that those in front of it leave.
//
// Few sequences of few channels leave most of the chip idle that way; they are cut into segments, whose maps
// a first kernel works out, and each segment's workgroup begins by composing those in front of it, a share a wavefront (one after the other, the thousand
// maps of 65,536 steps of 64 channels took 261 us with everything, and 66 so).  That reads gate and value twice, and is what
// bounds a few long sequences: 65,536 steps of 2,560 in 16 bits 156 us for the maps (4.3 TB/s) and 205 for the walk (4.9).  Without segments, 16
// sequences of 1,024 steps of 4,096 take 210 us for both passes (5.1 TB/s).  (One reading, workgroups waiting for the states that others make known: 311 us
// for the first, but 122 against 81 for 4 sequences of 1,021 steps of 4,096 both ways.)
//
// The backward pass is the same walk from the end, of e[t-1] = a[t] (grad[t] + e[t]), where e is the gradient of the state from
// what follows.  It needs h[t-1] to 32 bits: the forward pass leaves the state in front of every block
// of 64 steps (1/64 of gate and value in 16 bits), and the wavefronts work out the rest again from gate and value, which the backward pass reads anyway.
#include "ops_common.h"

#include <algorithm>
#include <cmath>

namespace fpsched {
namespace {

constexpr int kBlock = FPSCHED_RECURRENCE_BLOCK;
constexpr int kSteps = 16, kWaves = kBlock / kSteps;            // of a wavefront and of a workgroup, forward
constexpr int kGradSteps = 8, kGradWaves = kBlock / kGradSteps;   // backward, which holds more of each step
constexpr int kFewSteps = 16;

// a = sigmoid(gate) and 1 - a.  The smaller one is worked out (a gate of 20 has 1 - a = 2e-9) and the other one rounded once from
// it: a state is multiplied by a as many times as it has steps, and an error of the reciprocal in a would add up.
__device__ __forceinline__ void gates(float gate, float* a, float* b) {
  const float e = fast_exp(-__builtin_fabsf(gate)), small = e * __builtin_amdgcn_rcpf(1.f + e), large = 1.f - small;
  *a = gate >= 0.f ? large : small;   // (a gate that is no number makes both none)
  *b = gate >= 0.f ? small : large;
}

// (the steps and sequences of a tensor, in elements)
struct Strides {
  int64_t batch, step;
};

template <typename T>
struct RecurrenceArgs {
  const T *gate, *value, *grad;
  T *out, *d_gate, *d_value;
  Strides s_gate, s_value, s_grad, s_out, s_d_gate, s_d_value;
  const float *state;      // where the walk begins: in front of the first step; backward, the gradient behind the last
  float *final_state;      // where it ends
  float *kept;             // [batch][blocks][width]
  const int32_t* lengths;
  float* segment_maps;     // [batch][segment][2][width]
  float* state_copy;       // [batch][width]
  int64_t steps, width;
  int blocks, segment_blocks;   // of a sequence, of a segment
};

__device__ __forceinline__ int64_t end_of(const int32_t* lengths, int64_t b, int64_t steps) {
  return lengths ? min(max((int64_t)lengths[b], (int64_t)0), steps) : steps;
}

// Rows first ... of a tensor, a lane's channels from c on; of those from `end` on the last one in front of it (what is loaded is not used).
// Rows are the same for all lanes.
template <typename T, int N, int STEPS>
__device__ __forceinline__ void load_steps(Vec<T, N> (&to)[STEPS], const T* from, int64_t step_stride, int64_t first, int64_t end, unsigned c) {
#pragma unroll
  for (int i = 0; i < STEPS; ++i) to[i] = load_vec<T, N>(from + max(min(first + i, end - 1), (int64_t)0) * step_stride + c);
}

enum { kForward, kBackward };

// The maps of segments: forward (A, S) of its steps in order, backward (A, E) of them from the end.  Of the walk's segments but the last.
template <typename T, int N, int DIR>
__global__ __launch_bounds__(kWaves * 64) void segment_maps_kernel(RecurrenceArgs<T> args) {
  __shared__ Vec<float, 2 * N> maps[2][kWaves][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t b = blockIdx.y;
  const int turn = blockIdx.z;   // segments in the order of the walk
  const int segments = gridDim.z + 1;
  const unsigned at = (blockIdx.x * 64 + lane) * N;
  const bool live = at < args.width;
  const unsigned c = live ? at : 0;
  if (turn == 0 && wave == 0 && live) {   // (the caller may have the walk's result where its start is: other segments' workgroups read a copy)
#pragma unroll
    for (int k = 0; k < N; ++k) args.state_copy[b * args.width + c + k] = args.state ? args.state[b * args.width + c + k] : 0.f;
  }
  const int64_t end = end_of(args.lengths, b, args.steps);
  const T* gate = args.gate + b * args.s_gate.batch;
  const T* other = DIR == kForward ? args.value + b * args.s_value.batch : args.grad + b * args.s_grad.batch;
  const int64_t other_step = DIR == kForward ? args.s_value.step : args.s_grad.step;
  const int segment = DIR == kForward ? turn : segments - 1 - turn;
  const int first_block = segment * args.segment_blocks, last_block = min(first_block + args.segment_blocks, args.blocks);
  float A[N], S[N];
#pragma unroll
  for (int k = 0; k < N; ++k) A[k] = 1.f, S[k] = 0.f;
  for (int j = 0; j < last_block - first_block; ++j) {
    // (the walk itself begins where this one ends, with what is still in cache)
    const int block = DIR == kForward ? last_block - 1 - j : first_block + j;
    const int64_t first = (int64_t)block * kBlock + wave * kSteps;
    Vec<T, N> g[kSteps], v[kSteps];
    load_steps<T, N, kSteps>(g, gate, args.s_gate.step, first, end, c);
    load_steps<T, N, kSteps>(v, other, other_step, first, end, c);
    Vec<float, 2 * N> m;
#pragma unroll
    for (int k = 0; k < N; ++k) m.at[k] = 1.f, m.at[N + k] = 0.f;
#pragma unroll
    for (int n = 0; n < kSteps; ++n) {
      const int i = DIR == kForward ? n : kSteps - 1 - n;
      if (first + i < end) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
          float a, na;
          gates((float)g[i].at[k], &a, &na);
          if (DIR == kForward) m.at[N + k] = a * m.at[N + k] + na * (float)v[i].at[k];
          else m.at[N + k] = a * (m.at[N + k] + (float)v[i].at[k]);
          m.at[k] *= a;
        }
      }
    }
    maps[j & 1][wave][lane] = m;
    __syncthreads();   // (the next block's maps go to the other half)
#pragma unroll
    for (int n = 0; n < kWaves; ++n) {   // (in front of what is composed already)
      const Vec<float, 2 * N> o = maps[j & 1][DIR == kForward ? kWaves - 1 - n : n][lane];
#pragma unroll
      for (int k = 0; k < N; ++k) {
        S[k] += A[k] * o.at[N + k];
        A[k] *= o.at[k];
      }
    }
  }
  if (live && wave == 0) {
    float* to = args.segment_maps + (b * segments + turn) * 2 * args.width + c;
#pragma unroll
    for (int k = 0; k < N; ++k) to[k] = A[k], to[args.width + k] = S[k];
  }
}

// A lane's channels of the walk's state in front of its turn-th segment.  Each wavefront composes a share of the maps in front, in order; the shares go
// round through LDS (`maps`: a half of it that the walk's first block does not use).
template <typename T, int N, int WAVES>
__device__ __forceinline__ void begin_walk(const RecurrenceArgs<T>& args, int64_t b, int turn, int segments, unsigned c, int lane, int wave,
                                           Vec<float, 2 * N> (&maps)[WAVES][64], float (&h)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) h[k] = args.state ? args.state[b * args.width + c + k] : 0.f;
  if (turn == 0) return;
  const int share = (turn + WAVES - 1) / WAVES, first = min(wave * share, turn), last = min(first + share, turn);
  const float* m = args.segment_maps + (b * segments + first) * 2 * args.width + c;
  Vec<float, 2 * N> mine;
#pragma unroll
  for (int k = 0; k < N; ++k) mine.at[k] = 1.f, mine.at[N + k] = 0.f;
  constexpr int kAhead = 8;
  for (int s = first; s < last; s += kAhead) {
    float A[kAhead][N], S[kAhead][N];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const float* at = m + (int64_t)min(i, last - 1 - s) * 2 * args.width;
#pragma unroll
      for (int k = 0; k < N; ++k) A[i][k] = at[k], S[i][k] = at[args.width + k];
    }
    m += (int64_t)kAhead * 2 * args.width;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (s + i < last) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
          mine.at[N + k] = A[i][k] * mine.at[N + k] + S[i][k];
          mine.at[k] *= A[i][k];
        }
      }
    }
  }
  maps[wave][lane] = mine;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    const Vec<float, 2 * N> o = maps[w][lane];
#pragma unroll
    for (int k = 0; k < N; ++k) h[k] = o.at[k] * h[k] + o.at[N + k];
  }
}

template <typename T, int N, bool KEEP>
__global__ __launch_bounds__(kWaves * 64, 4) void recurrence_kernel(RecurrenceArgs<T> args) {
  __shared__ Vec<float, 2 * N> maps[2][kWaves][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t b = blockIdx.y;
  const int segment = blockIdx.z, segments = gridDim.z;
  const unsigned at = (blockIdx.x * 64 + lane) * N;
  const bool live = at < args.width;
  const unsigned c = live ? at : 0;
  const int64_t end = end_of(args.lengths, b, args.steps);
  const T *gate = args.gate + b * args.s_gate.batch, *value = args.value + b * args.s_value.batch;
  T* out = args.out + b * args.s_out.batch;
  float h[N];   // the state in front of the block
  const int first_block = segment * args.segment_blocks, last_block = min(first_block + args.segment_blocks, args.blocks);
  begin_walk<T, N, kWaves>(args, b, segment, segments, c, lane, wave, maps[(first_block + 1) & 1], h);
  for (int block = first_block; block < last_block; ++block) {
    const int64_t first = (int64_t)block * kBlock + wave * kSteps;
    float a[kSteps][N], s[kSteps][N];
    {
      Vec<T, N> g[kSteps], v[kSteps];
      load_steps<T, N, kSteps>(g, gate, args.s_gate.step, first, end, c);
      load_steps<T, N, kSteps>(v, value, args.s_value.step, first, end, c);
      if (KEEP && live && wave == 0) {
        float* to = args.kept + (b * args.blocks + block) * args.width + c;
#pragma unroll
        for (int k = 0; k < N; ++k) to[k] = h[k];
      }
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
          float na;
          gates((float)g[i].at[k], &a[i][k], &na);
          s[i][k] = na * (float)v[i].at[k];
        }
      }
    }
    if (first + kSteps > end) {
#pragma unroll
      for (int i = 0; i < kSteps; ++i)
        if (first + i >= end) {
#pragma unroll
          for (int k = 0; k < N; ++k) a[i][k] = 1.f, s[i][k] = 0.f;
        }
    }
    Vec<float, 2 * N> m;
#pragma unroll
    for (int k = 0; k < N; ++k) m.at[k] = 1.f, m.at[N + k] = 0.f;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        m.at[N + k] = a[i][k] * m.at[N + k] + s[i][k];
        m.at[k] *= a[i][k];
      }
    }
    maps[block & 1][wave][lane] = m;
    __syncthreads();   // (the next block's maps go to the other half: one barrier a block)
    float mine[N];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const Vec<float, 2 * N> o = maps[block & 1][w][lane];
#pragma unroll
      for (int k = 0; k < N; ++k) {
        if (w == wave) mine[k] = h[k];
        h[k] = o.at[k] * h[k] + o.at[N + k];
      }
    }
    T* row = out + first * args.s_out.step;
    if (first + kSteps <= end) {
#pragma unroll
      for (int i = 0; i < kSteps; ++i, row += args.s_out.step) {
        Vec<T, N> o;
#pragma unroll
        for (int k = 0; k < N; ++k) {
          mine[k] = a[i][k] * mine[k] + s[i][k];
          o.at[k] = (T)mine[k];
        }
        if (live) store_vec<T, N>(row + c, o);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kSteps; ++i, row += args.s_out.step) {
        if (first + i >= args.steps) break;
        Vec<T, N> o;
#pragma unroll
        for (int k = 0; k < N; ++k) {
          mine[k] = a[i][k] * mine[k] + s[i][k];
          o.at[k] = (T)(first + i < end ? mine[k] : 0.f);
        }
        if (live) store_vec<T, N>(row + c, o);
      }
    }
  }
  if (live && wave == 0 && segment == segments - 1) {
#pragma unroll
    for (int k = 0; k < N; ++k) args.final_state[b * args.width + c + k] = h[k];
  }
}

// At most kFewSteps steps: a lane takes its channels from first to last.  (64 sequences of 9 steps of 4,096: 5.8 us, and 17.2 in a block of 64.)
template <typename T, int N>
__global__ __launch_bounds__(256) void few_steps_kernel(RecurrenceArgs<T> args) {
  const int64_t b = blockIdx.y;
  const unsigned c = (blockIdx.x * 256 + threadIdx.x) * N;
  if (c >= args.width) return;
  const int64_t end = end_of(args.lengths, b, args.steps);
  const T *gate = args.gate + b * args.s_gate.batch, *value = args.value + b * args.s_value.batch;
  T* out = args.out + b * args.s_out.batch;
  Vec<float, N> h = {};
  if (args.state) {
#pragma unroll
    for (int k = 0; k < N; ++k) h.at[k] = args.state[b * args.width + c + k];
  }
  if (args.kept) {
#pragma unroll
    for (int k = 0; k < N; ++k) args.kept[b * args.width + c + k] = h.at[k];
  }
  constexpr int kAhead = 8;
  for (int64_t first = 0; first < args.steps; first += kAhead) {
    Vec<T, N> g[kAhead], v[kAhead];
    load_steps<T, N, kAhead>(g, gate, args.s_gate.step, first, end, c);
    load_steps<T, N, kAhead>(v, value, args.s_value.step, first, end, c);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (first + i >= args.steps) break;
      Vec<T, N> o = {};
      if (first + i < end) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
          float a, na;
          gates((float)g[i].at[k], &a, &na);
          h.at[k] = a * h.at[k] + na * (float)v[i].at[k];
          o.at[k] = (T)h.at[k];
        }
      }
      store_vec<T, N>(out + (first + i) * args.s_out.step + c, o);
    }
  }
#pragma unroll
  for (int k = 0; k < N; ++k) args.final_state[b * args.width + c + k] = h.at[k];
}

// Its backward pass: the states in front of the steps once more, then the steps from last to first.  (64 sequences of one step of 4,096: 3.9 us,
// and 18.9 in blocks of 64 steps; of 16 steps 11.2 and 22.7.)
template <typename T, int N, int STEPS>
__global__ __launch_bounds__(256) void few_steps_grad_kernel(RecurrenceArgs<T> args) {
  const int64_t b = blockIdx.y;
  const unsigned c = (blockIdx.x * 256 + threadIdx.x) * N;
  if (c >= args.width) return;
  const int steps = (int)args.steps, end = (int)end_of(args.lengths, b, args.steps);
  const T *gate = args.gate + b * args.s_gate.batch + c, *value = args.value + b * args.s_value.batch + c, *grad = args.grad + b * args.s_grad.batch + c;
  T *d_gate = args.d_gate + b * args.s_d_gate.batch + c, *d_value = args.d_value + b * args.s_d_value.batch + c;
  float h[N], e[N], a[STEPS][N], na[STEPS][N], before[STEPS][N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    h[k] = args.kept[b * args.width + c + k];
    e[k] = args.state ? args.state[b * args.width + c + k] : 0.f;
  }
#pragma unroll
  for (int t = 0; t < STEPS; ++t) {
    if (t < end) {
      const Vec<T, N> g = load_vec<T, N>(gate + t * args.s_gate.step), v = load_vec<T, N>(value + t * args.s_value.step);
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float x = (float)v.at[k];
        gates((float)g.at[k], &a[t][k], &na[t][k]);
        before[t][k] = h[k] - x;
        h[k] = a[t][k] * h[k] + na[t][k] * x;
      }
    }
  }
#pragma unroll
  for (int t = STEPS - 1; t >= 0; --t) {
    if (t < steps) {
      Vec<T, N> dg = {}, dv = {};
      if (t < end) {
        const Vec<T, N> d = load_vec<T, N>(grad + t * args.s_grad.step);
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const float now = (float)d.at[k] + e[k];
          dv.at[k] = (T)(na[t][k] * now);
          dg.at[k] = (T)(now * before[t][k] * (a[t][k] * na[t][k]));
          e[k] = a[t][k] * now;
        }
      }
      store_vec<T, N>(d_value + t * args.s_d_value.step, dv);
      store_vec<T, N>(d_gate + t * args.s_d_gate.step, dg);
    }
  }
  if (args.final_state) {
#pragma unroll
    for (int k = 0; k < N; ++k) args.final_state[b * args.width + c + k] = e[k];
  }
}

template <typename T, int N>
__global__ __launch_bounds__(kGradWaves * 64) void recurrence_grad_kernel(RecurrenceArgs<T> args) {
  __shared__ Vec<float, 2 * N> maps[2][kGradWaves][64];
  __shared__ Vec<float, N> map_grads[2][kGradWaves][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t b = blockIdx.y;
  const int segments = gridDim.z, segment = blockIdx.z;
  const unsigned at = (blockIdx.x * 64 + lane) * N;
  const bool live = at < args.width;
  const unsigned c = live ? at : 0;
  const int64_t end = end_of(args.lengths, b, args.steps);
  const T *gate = args.gate + b * args.s_gate.batch, *value = args.value + b * args.s_value.batch, *grad = args.grad + b * args.s_grad.batch;
  T *d_gate = args.d_gate + b * args.s_d_gate.batch, *d_value = args.d_value + b * args.s_d_value.batch;
  float e[N];   // the gradient of the state behind the block
  const int first_block = segment * args.segment_blocks, last_block = min(first_block + args.segment_blocks, args.blocks);
  begin_walk<T, N, kGradWaves>(args, b, segments - 1 - segment, segments, c, lane, wave, maps[last_block & 1], e);
  for (int block = last_block - 1; block >= first_block; --block) {
    const int64_t first = (int64_t)block * kBlock + wave * kGradSteps;
    Vec<T, N> g[kGradSteps], v[kGradSteps], d[kGradSteps];
    load_steps<T, N, kGradSteps>(g, gate, args.s_gate.step, first, end, c);
    load_steps<T, N, kGradSteps>(v, value, args.s_value.step, first, end, c);
    load_steps<T, N, kGradSteps>(d, grad, args.s_grad.step, first, end, c);
    float h[N];
#pragma unroll
    for (int k = 0; k < N; ++k) h[k] = args.kept[(b * args.blocks + block) * args.width + c + k];
    const bool whole = first + kGradSteps <= end;
    float a[kGradSteps][N], na[kGradSteps][N];
#pragma unroll
    for (int i = 0; i < kGradSteps; ++i) {
#pragma unroll
      for (int k = 0; k < N; ++k) gates((float)g[i].at[k], &a[i][k], &na[i][k]);
    }
    if (!whole) {
#pragma unroll
      for (int i = 0; i < kGradSteps; ++i)
        if (first + i >= end) {
          v[i] = {}, d[i] = {};
#pragma unroll
          for (int k = 0; k < N; ++k) a[i][k] = 1.f, na[i][k] = 0.f;
        }
    }
    Vec<float, 2 * N> m;
    Vec<float, N> E = {};
#pragma unroll
    for (int k = 0; k < N; ++k) m.at[k] = 1.f, m.at[N + k] = 0.f;
#pragma unroll
    for (int i = 0; i < kGradSteps; ++i) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        m.at[N + k] = a[i][k] * m.at[N + k] + na[i][k] * (float)v[i].at[k];
        m.at[k] *= a[i][k];
      }
    }
#pragma unroll
    for (int i = kGradSteps - 1; i >= 0; --i) {
#pragma unroll
      for (int k = 0; k < N; ++k) E.at[k] = a[i][k] * ((float)d[i].at[k] + E.at[k]);
    }
    maps[block & 1][wave][lane] = m;
    map_grads[block & 1][wave][lane] = E;
    __syncthreads();
    float behind[N];
    for (int w = 0; w < wave; ++w) {
      const Vec<float, 2 * N> o = maps[block & 1][w][lane];
#pragma unroll
      for (int k = 0; k < N; ++k) h[k] = o.at[k] * h[k] + o.at[N + k];
    }
#pragma unroll
    for (int w = kGradWaves - 1; w >= 0; --w) {
      const Vec<float, 2 * N> o = maps[block & 1][w][lane];
      const Vec<float, N> og = map_grads[block & 1][w][lane];
#pragma unroll
      for (int k = 0; k < N; ++k) {
        if (w == wave) behind[k] = e[k];
        e[k] = o.at[k] * e[k] + og.at[k];
      }
    }
    float before[kGradSteps][N];   // the state in front of each step, less its value
#pragma unroll
    for (int i = 0; i < kGradSteps; ++i) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float x = (float)v[i].at[k];
        before[i][k] = h[k] - x;
        h[k] = a[i][k] * h[k] + na[i][k] * x;
      }
    }
#pragma unroll
    for (int i = kGradSteps - 1; i >= 0; --i) {
      Vec<T, N> dg, dv;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float now = (float)d[i].at[k] + behind[k];
        dv.at[k] = (T)(na[i][k] * now);
        dg.at[k] = (T)(now * before[i][k] * (a[i][k] * na[i][k]));
        behind[k] = a[i][k] * now;
      }
      if (!whole && first + i >= end) dg = {}, dv = {};   // (a state that is infinite makes 0 times it no number)
      if (live && first + i < args.steps) {
        store_vec<T, N>(d_value + (first + i) * args.s_d_value.step + c, dv);
        store_vec<T, N>(d_gate + (first + i) * args.s_d_gate.step + c, dg);
      }
    }
  }
  if (live && wave == 0 && segment == 0 && args.final_state) {
#pragma unroll
    for (int k = 0; k < N; ++k) args.final_state[b * args.width + c + k] = e[k];
  }
}

// Segments of a sequence: enough for four workgroups a compute unit, and none where there are two each without (a segment's steps are read
// twice).  65,536 steps of 2,560 forward, 4 x 1,021 of 4,096 in both directions: for two workgroups a compute unit 380 and 84 us, for four 347
// and 78, for six 368 and 78.  But a segment costs those behind it a hundredth of what a block of steps costs it, so that no more than sqrt(128 blocks) are
// worth it: 65,536 steps of 64 channels forward take 68 us in 1,024 segments, 39 in 342, 53 in 128.
struct Cut {
  int blocks, segment_blocks, segments;
};

Cut cut(int64_t n_batch, int64_t n_steps, int64_t width) {
  Cut s;
  s.blocks = (int)ceil_div(n_steps, kBlock);
  const int64_t groups = std::max<int64_t>(1, n_batch * ceil_div(width, 128));
  s.segment_blocks = std::max(s.blocks, 1);
  if (groups < 512 && s.blocks > 1) {
    const int64_t most = (int64_t)std::sqrt(128. * s.blocks) + 1;
    s.segment_blocks = (int)ceil_div(s.blocks, std::min<int64_t>({ceil_div(1024, groups), most, s.blocks}));
  }
  s.segments = (int)std::max<int64_t>(1, ceil_div(s.blocks, s.segment_blocks));
  return s;
}

constexpr int64_t kMostStride = 1ll << 31;   // (times a count of steps far from what 64 bits hold)

bool sizes_fit(int64_t n_batch, int64_t n_steps, int64_t width) {
  return n_batch >= 0 && n_batch <= 65535 && n_steps >= 0 && n_steps <= 0x7fffffffll && width >= 0 && width <= (1 << 24);
}

// Both kernels, maps(args, grid) and then walk(args, grid), or the walk alone.
template <typename T, typename M, typename W>
void run_walk(RecurrenceArgs<T> a, const Cut& s, int64_t n_batch, unsigned x, float* workspace, M maps, W walk) {
  a.blocks = s.blocks;
  a.segment_blocks = s.segment_blocks;
  if (s.segments > 1) {
    a.segment_maps = workspace;
    a.state_copy = workspace + n_batch * s.segments * 2 * a.width;
    maps(a, dim3(x, (unsigned)n_batch, s.segments - 1));
    a.state = a.state_copy;
  }
  walk(a, dim3(x, (unsigned)n_batch, s.segments));
}

// Whether no two elements of an output share memory: the steps of a sequence behind one another, or the sequences of a step.  (Of no elements none do,
// whatever the strides: those of packed sequences of no steps are 0.)
bool apart(int64_t n_batch, int64_t n_steps, int64_t width, int64_t batch, int64_t step) {
  if (n_batch == 0 || n_steps == 0 || width == 0) return true;
  if (n_batch <= 1) return n_steps <= 1 || step >= width;
  if (n_steps <= 1) return batch >= width;
  return (step >= width && batch >= (n_steps - 1) * step + width) || (batch >= width && step >= (n_batch - 1) * batch + width);
}

// f(N): two channels a lane where every tensor's place and strides are even
template <typename T, typename F>
int with_channels(int64_t width, std::initializer_list<const void*> tensors, std::initializer_list<int64_t> strides, F f) {
  bool two = width % 2 == 0;
  for (const void* p : tensors) two = two && aligned(p, 2 * sizeof(T));
  for (int64_t s : strides) two = two && s % 2 == 0;
  return two ? f(std::integral_constant<int, 2>()) : f(std::integral_constant<int, 1>());
}

}  // namespace
}  // namespace fpsched

using namespace fpsched;

extern "C" {

size_t fpsched_op_recurrence_workspace_bytes(int64_t n_batch, int64_t n_steps, int64_t width) {
  if (!sizes_fit(n_batch, n_steps, width)) return 0;
  const Cut s = cut(n_batch, n_steps, width);
  return s.segments > 1 ? (size_t)n_batch * (s.segments * 2 + 1) * width * sizeof(float) : 16;
}

int fpsched_op_recurrence(int device_id, int type, int64_t n_batch, int64_t n_steps, int64_t width, const void* gate,
                          const void* value, const int64_t* strides, const float* state, const int32_t* lengths, void* out,
                          float* final_state, float* kept, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  if (type < FPSCHED_BF16 || type > FPSCHED_F32 || !sizes_fit(n_batch, n_steps, width) || !strides) return FPSCHED_EINVAL;
  for (int i = 0; i < 6; ++i)
    if (strides[i] < 0 || strides[i] > kMostStride) return FPSCHED_EINVAL;
  if (!apart(n_batch, n_steps, width, strides[4], strides[5])) return FPSCHED_EINVAL;
  if (device_id < 0) return FPSCHED_ENODEV;
  if (n_batch == 0 || width == 0) return FPSCHED_OK;
  if (!final_state || (n_steps > 0 && (!gate || !value || !out))) return FPSCHED_EINVAL;
  for (const void* p : {gate, value, static_cast<const void*>(out)})
    if (!aligned(p, type == FPSCHED_F32 ? 4 : 2)) return FPSCHED_EINVAL;
  const Cut s = cut(n_batch, n_steps, width);
  if (s.segments > 1) {
    if (!d_workspace || !aligned(d_workspace, 16)) return FPSCHED_EINVAL;
    if (workspace_bytes < fpsched_op_recurrence_workspace_bytes(n_batch, n_steps, width)) return FPSCHED_ENOMEM;
  }
  OpsDevice g(device_id);
  if (!g.ok) return FPSCHED_EHIP;
  return with_type(type, [&](auto zero) {
    using T = decltype(zero);
    RecurrenceArgs<T> a = {};
    a.gate = static_cast<const T*>(gate); a.value = static_cast<const T*>(value); a.out = static_cast<T*>(out);
    a.s_gate = {strides[0], strides[1]}; a.s_value = {strides[2], strides[3]}; a.s_out = {strides[4], strides[5]};
    a.state = state; a.final_state = final_state; a.kept = n_steps > 0 ? kept : nullptr;   // (no steps: no blocks, and no room for a state in front of one)
    a.lengths = lengths; a.steps = n_steps; a.width = width;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return with_channels<T>(width, {gate, value, out}, {strides[0], strides[1], strides[2], strides[3], strides[4], strides[5]}, [&](auto n) {
      constexpr int N = decltype(n)::value;
      if (n_steps <= kFewSteps) {
        few_steps_kernel<T, N><<<dim3((unsigned)ceil_div(width, 256 * N), (unsigned)n_batch), dim3(256), 0, stream>>>(a);
        return launched();
      }
      run_walk(a, s, n_batch, (unsigned)ceil_div(width, 64 * N), static_cast<float*>(d_workspace),
                  [&](const RecurrenceArgs<T>& m, dim3 grid) { segment_maps_kernel<T, N, kForward><<<grid, dim3(kWaves * 64), 0, stream>>>(m); },
                  [&](const RecurrenceArgs<T>& w, dim3 grid) {
                    if (kept) recurrence_kernel<T, N, true><<<grid, dim3(kWaves * 64), 0, stream>>>(w);
                    else recurrence_kernel<T, N, false><<<grid, dim3(kWaves * 64), 0, stream>>>(w);
                  });
      return launched();
    });
  });
}

int fpsched_op_recurrence_grad(int device_id, int type, int64_t n_batch, int64_t n_steps, int64_t width, const void* grad,
                               const void* gate, const void* value, const int64_t* strides, const float* kept,
                               const float* grad_state, const int32_t* lengths, void* d_gate, void* d_value, float* d_state,
                               void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  if (type < FPSCHED_BF16 || type > FPSCHED_F32 || !sizes_fit(n_batch, n_steps, width) || !strides) return FPSCHED_EINVAL;
  for (int i = 0; i < 10; ++i)
    if (strides[i] < 0 || strides[i] > kMostStride) return FPSCHED_EINVAL;
  for (int i = 6; i < 10; i += 2)
    if (!apart(n_batch, n_steps, width, strides[i], strides[i + 1])) return FPSCHED_EINVAL;
  if (device_id < 0) return FPSCHED_ENODEV;
  if (n_batch == 0 || width == 0) return FPSCHED_OK;
  if (n_steps > 0 && (!grad || !gate || !value || !kept || !d_gate || !d_value)) return FPSCHED_EINVAL;
  for (const void* p : {grad, gate, value, static_cast<const void*>(d_gate), static_cast<const void*>(d_value)})
    if (!aligned(p, type == FPSCHED_F32 ? 4 : 2)) return FPSCHED_EINVAL;
  const Cut s = cut(n_batch, n_steps, width);
  if (s.segments > 1) {
    if (!d_workspace || !aligned(d_workspace, 16)) return FPSCHED_EINVAL;
    if (workspace_bytes < fpsched_op_recurrence_workspace_bytes(n_batch, n_steps, width)) return FPSCHED_ENOMEM;
  }
  OpsDevice g(device_id);
  if (!g.ok) return FPSCHED_EHIP;
  return with_type(type, [&](auto zero) {
    using T = decltype(zero);
    RecurrenceArgs<T> a = {};
    a.grad = static_cast<const T*>(grad); a.gate = static_cast<const T*>(gate); a.value = static_cast<const T*>(value);
    a.d_gate = static_cast<T*>(d_gate); a.d_value = static_cast<T*>(d_value);
    a.s_grad = {strides[0], strides[1]}; a.s_gate = {strides[2], strides[3]}; a.s_value = {strides[4], strides[5]};
    a.s_d_gate = {strides[6], strides[7]}; a.s_d_value = {strides[8], strides[9]};
    a.state = grad_state; a.final_state = d_state; a.kept = const_cast<float*>(kept); a.lengths = lengths;
    a.steps = n_steps; a.width = width;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return with_channels<T>(width, {grad, gate, value, d_gate, d_value},
                            {strides[0], strides[1], strides[2], strides[3], strides[4], strides[5], strides[6], strides[7], strides[8], strides[9]},
                            [&](auto n) {
      constexpr int N = decltype(n)::value;
      const dim3 few((unsigned)ceil_div(width, 256 * N), (unsigned)n_batch);
      if (n_steps > 0 && n_steps <= kFewSteps / 2) {
        few_steps_grad_kernel<T, N, kFewSteps / 2><<<few, dim3(256), 0, stream>>>(a);
        return launched();
      }
      // (few channels leave a lane's steps one after the other to its latency: one sequence of 16 steps of 4,096 8.7 us so and 5.3 in a block)
      if (n_steps > 0 && n_steps <= kFewSteps && n_batch * ceil_div(width, 128) >= 256) {
        few_steps_grad_kernel<T, N, kFewSteps><<<few, dim3(256), 0, stream>>>(a);
        return launched();
      }
      run_walk(a, s, n_batch, (unsigned)ceil_div(width, 64 * N), static_cast<float*>(d_workspace),
                  [&](const RecurrenceArgs<T>& m, dim3 grid) { segment_maps_kernel<T, N, kBackward><<<grid, dim3(kWaves * 64), 0, stream>>>(m); },
                  [&](const RecurrenceArgs<T>& w, dim3 grid) { recurrence_grad_kernel<T, N><<<grid, dim3(kGradWaves * 64), 0, stream>>>(w); });
      return launched();
    });
  });
}

}  // extern "C"
