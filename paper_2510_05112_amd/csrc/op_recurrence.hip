// Gated linear recurrence:  h[t] = a[t] h[t-1] + (1 - a[t]) v[t],  a = sigmoid(gate), for each sequence and channel.
//
// A step is an affine map of the state, and maps compose: of a run of steps (A, S) with h_end = A h_begin + S, two runs one after the other
// have (A2 A1, A2 S1 + S2).  A workgroup walks a sequence in blocks of kWaves x kSteps = 128 steps for 64 lanes' channels (two adjacent ones a lane
// where strides allow): each wavefront loads kSteps of them, works out its run's map from registers, the maps go round through LDS, and
// each wavefront then takes its steps from the state that those in front of it leave.  Everything is read once and written once, the next block's
// loads under way meanwhile.
//
// Few sequences of few channels leave most of the chip idle that way; they are cut into segments, whose maps
// a first kernel works out (it reads gate and value once more), and each segment's workgroup begins by composing those in front of it.
//
// The backward pass is the same walk from the end, of e[t-1] = a[t] (grad[t] + e[t]), where e is the gradient of the state from
// what follows.  It needs h[t-1] to 32 bits: the forward pass leaves the state in front of every block
// of 128 steps (at most 1/32 of what it reads), and the wavefronts work out the rest again from gate and value, which the backward pass reads anyway.
#include "ops_common.h"

namespace fpsched {
namespace {

constexpr int kWaves = 8, kSteps = 16, kBlock = FPSCHED_RECURRENCE_BLOCK;
static_assert(kWaves * kSteps == kBlock, "a workgroup's steps are a block");

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
  const float *state;      // of the forward pass: in front of the first step; of the backward pass: the gradient behind the last
  float *final_state;      // ... behind the last; the gradient in front of the first
  float *kept;             // [batch][blocks][width]
  const int32_t* lengths;
  float* segment_maps;     // [batch][segment][2][width]
  float* state_copy;       // [batch][width]
  int64_t steps, width;
  int blocks, segment_blocks, segments;
};

// One block of steps of a lane's channels in registers, steps [first, first + kSteps) of this wavefront.
template <typename T, int N>
__device__ __forceinline__ void load_steps(Vec<T, N> (&to)[kSteps], const T* from, int64_t step_stride, int64_t first, int64_t end) {
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    to[i] = {};
    if (first + i < end) to[i] = load_vec<T, N>(from + (first + i) * step_stride);
  }
}

enum { kForward, kBackward };

// The maps of segments: forward (A, S) of its steps in order, backward (A, E) of them from the end.
template <typename T, int N, int DIR>
__global__ __launch_bounds__(kWaves * 64) void segment_maps_kernel(RecurrenceArgs<T> args) {
  __shared__ float maps[kWaves][2][64 * N];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t b = blockIdx.y, segment = DIR == kForward ? blockIdx.z : blockIdx.z + 1;   // (nothing follows the walk's last)
  const int64_t c = ((int64_t)blockIdx.x * 64 + lane) * N;
  const bool live = c < args.width;
  const int64_t cc = live ? c : 0;
  if (blockIdx.z == 0 && wave == 0 && live) {   // (the caller may have the walk's result where its start is: other segments' workgroups read a copy)
#pragma unroll
    for (int k = 0; k < N; ++k) args.state_copy[b * args.width + c + k] = args.state ? args.state[b * args.width + c + k] : 0.f;
  }
  const int64_t end = args.lengths ? min(max((int64_t)args.lengths[b], (int64_t)0), args.steps) : args.steps;
  const T* gate = args.gate + b * args.s_gate.batch + cc;
  const T* other = DIR == kForward ? args.value + b * args.s_value.batch + cc : args.grad + b * args.s_grad.batch + cc;
  const int64_t other_step = DIR == kForward ? args.s_value.step : args.s_grad.step;
  float A[N], S[N];
#pragma unroll
  for (int k = 0; k < N; ++k) A[k] = 1.f, S[k] = 0.f;
  const int64_t first_block = segment * args.segment_blocks, last_block = min(first_block + args.segment_blocks, (int64_t)args.blocks);
  // (each wavefront its share of the segment's blocks' steps, block by block: the maps of a wavefront's runs in different blocks are not
  // adjacent, so they are composed block by block)
  for (int64_t j = 0; j < last_block - first_block; ++j) {
    const int64_t block = DIR == kForward ? first_block + j : last_block - 1 - j;
    if (block * kBlock >= end) continue;
    const int64_t first = block * kBlock + wave * kSteps;
    Vec<T, N> g[kSteps], v[kSteps];
    load_steps<T, N>(g, gate, args.s_gate.step, first, end);
    load_steps<T, N>(v, other, other_step, first, end);
    float a1[N], s1[N];
#pragma unroll
    for (int k = 0; k < N; ++k) a1[k] = 1.f, s1[k] = 0.f;
#pragma unroll
    for (int n = 0; n < kSteps; ++n) {
      const int i = DIR == kForward ? n : kSteps - 1 - n;
      if (first + i < end) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
          float a, na;
          gates((float)g[i].at[k], &a, &na);
          if (DIR == kForward) s1[k] = a * s1[k] + na * (float)v[i].at[k];
          else s1[k] = a * (s1[k] + (float)v[i].at[k]);
          a1[k] *= a;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) maps[wave][0][lane * N + k] = a1[k], maps[wave][1][lane * N + k] = s1[k];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < kWaves; ++n) {
      const int w = DIR == kForward ? n : kWaves - 1 - n;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float a2 = maps[w][0][lane * N + k];
        S[k] = a2 * S[k] + maps[w][1][lane * N + k];
        A[k] *= a2;
      }
    }
    __syncthreads();
  }
  if (live && wave == 0) {
    float* to = args.segment_maps + ((b * args.segments + segment) * 2) * args.width + c;
#pragma unroll
    for (int k = 0; k < N; ++k) to[k] = A[k], to[args.width + k] = S[k];
  }
}

template <typename T, int N, bool KEEP>
__global__ __launch_bounds__(kWaves * 64) void recurrence_kernel(RecurrenceArgs<T> args) {
  __shared__ float maps[2][kWaves][2][64 * N];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t b = blockIdx.y, segment = blockIdx.z;
  const int64_t c = ((int64_t)blockIdx.x * 64 + lane) * N;
  const bool live = c < args.width;
  const int64_t cc = live ? c : 0;
  const int64_t end = args.lengths ? min(max((int64_t)args.lengths[b], (int64_t)0), args.steps) : args.steps;
  const T* gate = args.gate + b * args.s_gate.batch + cc;
  const T* value = args.value + b * args.s_value.batch + cc;
  T* out = args.out + b * args.s_out.batch + cc;
  float h[N];   // the state in front of the block
#pragma unroll
  for (int k = 0; k < N; ++k) h[k] = args.state ? args.state[b * args.width + cc + k] : 0.f;
  for (int64_t s = 0; s < segment; ++s) {
    const float* m = args.segment_maps + ((b * args.segments + s) * 2) * args.width + cc;
#pragma unroll
    for (int k = 0; k < N; ++k) h[k] = m[k] * h[k] + m[args.width + k];
  }
  const int64_t first_block = segment * args.segment_blocks, last_block = min(first_block + args.segment_blocks, (int64_t)args.blocks);
  Vec<T, N> g[kSteps], v[kSteps];
  load_steps<T, N>(g, gate, args.s_gate.step, first_block * kBlock + wave * kSteps, end);
  load_steps<T, N>(v, value, args.s_value.step, first_block * kBlock + wave * kSteps, end);
  for (int64_t block = first_block; block < last_block; ++block) {
    if (KEEP && live && wave == 0) {
      float* to = args.kept + (b * args.blocks + block) * args.width + c;
#pragma unroll
      for (int k = 0; k < N; ++k) to[k] = h[k];
    }
    const int64_t first = block * kBlock + wave * kSteps;
    float a[kSteps][N], s[kSteps][N], A[N], S[N];
#pragma unroll
    for (int k = 0; k < N; ++k) A[k] = 1.f, S[k] = 0.f;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        float na;
        gates((float)g[i].at[k], &a[i][k], &na);
        s[i][k] = na * (float)v[i].at[k];
        if (first + i >= end) a[i][k] = 1.f, s[i][k] = 0.f;
        S[k] = a[i][k] * S[k] + s[i][k];
        A[k] *= a[i][k];
      }
    }
    if (block + 1 < last_block) {
      load_steps<T, N>(g, gate, args.s_gate.step, first + kBlock, end);
      load_steps<T, N>(v, value, args.s_value.step, first + kBlock, end);
    }
    float(&m)[kWaves][2][64 * N] = maps[block & 1];
#pragma unroll
    for (int k = 0; k < N; ++k) m[wave][0][lane * N + k] = A[k], m[wave][1][lane * N + k] = S[k];
    __syncthreads();   // (the other half of `maps` is the next block's: one barrier a block)
    float mine[N];
#pragma unroll
    for (int k = 0; k < N; ++k) mine[k] = h[k];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        if (w == wave) mine[k] = h[k];
        h[k] = m[w][0][lane * N + k] * h[k] + m[w][1][lane * N + k];
      }
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      if (first + i >= args.steps) break;
      Vec<T, N> o;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        mine[k] = a[i][k] * mine[k] + s[i][k];
        o.at[k] = (T)(first + i < end ? mine[k] : 0.f);
      }
      if (live) store_vec<T, N>(out + (first + i) * args.s_out.step, o);
    }
  }
  if (live && wave == 0 && segment == args.segments - 1) {
#pragma unroll
    for (int k = 0; k < N; ++k) args.final_state[b * args.width + c + k] = h[k];
  }
}

template <typename T, int N>
__global__ __launch_bounds__(kWaves * 64) void recurrence_grad_kernel(RecurrenceArgs<T> args) {
  __shared__ float maps[2][kWaves][4][64 * N];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t b = blockIdx.y, segment = blockIdx.z;
  const int64_t c = ((int64_t)blockIdx.x * 64 + lane) * N;
  const bool live = c < args.width;
  const int64_t cc = live ? c : 0;
  const int64_t end = args.lengths ? min(max((int64_t)args.lengths[b], (int64_t)0), args.steps) : args.steps;
  const T* gate = args.gate + b * args.s_gate.batch + cc;
  const T* value = args.value + b * args.s_value.batch + cc;
  const T* grad = args.grad + b * args.s_grad.batch + cc;
  T* d_gate = args.d_gate + b * args.s_d_gate.batch + cc;
  T* d_value = args.d_value + b * args.s_d_value.batch + cc;
  float e[N];   // the gradient of the state behind the block
#pragma unroll
  for (int k = 0; k < N; ++k) e[k] = args.state ? args.state[b * args.width + cc + k] : 0.f;
  for (int64_t s = args.segments - 1; s > segment; --s) {
    const float* m = args.segment_maps + ((b * args.segments + s) * 2) * args.width + cc;
#pragma unroll
    for (int k = 0; k < N; ++k) e[k] = m[k] * e[k] + m[args.width + k];
  }
  const int64_t first_block = segment * args.segment_blocks, last_block = min(first_block + args.segment_blocks, (int64_t)args.blocks);
  Vec<T, N> g[kSteps], v[kSteps], d[kSteps];
  auto load = [&](int64_t block) {
    const int64_t first = block * kBlock + wave * kSteps;
    load_steps<T, N>(g, gate, args.s_gate.step, first, end);
    load_steps<T, N>(v, value, args.s_value.step, first, end);
    load_steps<T, N>(d, grad, args.s_grad.step, first, end);
  };
  if (last_block > first_block) load(last_block - 1);
  for (int64_t block = last_block - 1; block >= first_block; --block) {
    const int64_t first = block * kBlock + wave * kSteps;
    float h[N];
#pragma unroll
    for (int k = 0; k < N; ++k) h[k] = args.kept[(b * args.blocks + block) * args.width + cc + k];
    float A[N], S[N], E[N];
#pragma unroll
    for (int k = 0; k < N; ++k) A[k] = 1.f, S[k] = 0.f, E[k] = 0.f;
    float a[kSteps][N], na[kSteps][N];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        gates((float)g[i].at[k], &a[i][k], &na[i][k]);
        if (first + i >= end) a[i][k] = 1.f, na[i][k] = 0.f;   // (value and grad are zero there)
        S[k] = a[i][k] * S[k] + na[i][k] * (float)v[i].at[k];
        A[k] *= a[i][k];
      }
    }
#pragma unroll
    for (int i = kSteps - 1; i >= 0; --i) {
#pragma unroll
      for (int k = 0; k < N; ++k) E[k] = a[i][k] * ((float)d[i].at[k] + E[k]);
    }
    float(&m)[kWaves][4][64 * N] = maps[block & 1];
#pragma unroll
    for (int k = 0; k < N; ++k) m[wave][0][lane * N + k] = A[k], m[wave][1][lane * N + k] = S[k], m[wave][2][lane * N + k] = E[k];
    __syncthreads();
    float behind[N];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w >= wave) break;
#pragma unroll
      for (int k = 0; k < N; ++k) h[k] = m[w][0][lane * N + k] * h[k] + m[w][1][lane * N + k];
    }
#pragma unroll
    for (int w = kWaves - 1; w >= 0; --w) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        if (w == wave) behind[k] = e[k];
        e[k] = m[w][0][lane * N + k] * e[k] + m[w][2][lane * N + k];
      }
    }
    float before[kSteps][N];   // the state in front of each step, less its value
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float x = (float)v[i].at[k];
        before[i][k] = h[k] - x;
        h[k] = a[i][k] * h[k] + na[i][k] * x;
      }
    }
#pragma unroll
    for (int i = kSteps - 1; i >= 0; --i) {
      Vec<T, N> dg, dv;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float now = (float)d[i].at[k] + behind[k];
        const bool in = first + i < end;
        dv.at[k] = (T)(in ? na[i][k] * now : 0.f);
        dg.at[k] = (T)(in ? now * before[i][k] * (a[i][k] * na[i][k]) : 0.f);
        behind[k] = a[i][k] * now;
      }
      if (live && first + i < args.steps) {
        store_vec<T, N>(d_value + (first + i) * args.s_d_value.step, dv);
        store_vec<T, N>(d_gate + (first + i) * args.s_d_gate.step, dg);
      }
    }
    if (block > first_block) load(block - 1);
  }
  if (live && wave == 0 && segment == 0 && args.final_state) {
#pragma unroll
    for (int k = 0; k < N; ++k) args.final_state[b * args.width + c + k] = e[k];
  }
}

// Segments of a sequence: enough for two workgroups a compute unit, of four blocks at least (what a segment
// costs is the second reading of its steps, and its turn in the composition that every later segment begins with).
struct Cut {
  int blocks, segment_blocks, segments;
};

Cut cut(int64_t n_batch, int64_t n_steps, int64_t width) {
  Cut s;
  s.blocks = (int)ceil_div(n_steps, kBlock);
  const int64_t groups = std::max<int64_t>(1, n_batch * ceil_div(width, 128));
  const int64_t wanted = std::min<int64_t>(ceil_div(512, groups), ceil_div(s.blocks, 4));
  s.segment_blocks = (int)std::max<int64_t>(1, ceil_div(s.blocks, std::max<int64_t>(1, wanted)));
  s.segments = (int)std::max<int64_t>(1, ceil_div(s.blocks, s.segment_blocks));
  return s;
}

constexpr int64_t kMostStride = 1ll << 31;   // (times a count of steps far from what 64 bits hold)

bool sizes_fit(int64_t n_batch, int64_t n_steps, int64_t width) {
  return n_batch >= 0 && n_batch <= 65535 && n_steps >= 0 && n_steps <= 0x7fffffffll && width >= 0 && width <= (1 << 24);
}

// Whether no two elements of an output share memory: the steps of a sequence behind one another, or the sequences of a step.
bool apart(int64_t n_batch, int64_t n_steps, int64_t width, int64_t batch, int64_t step) {
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
    a.state = state; a.final_state = final_state; a.kept = kept; a.lengths = lengths;
    a.segment_maps = static_cast<float*>(d_workspace);
    a.state_copy = a.segment_maps + n_batch * s.segments * 2 * width;
    a.steps = n_steps; a.width = width; a.blocks = s.blocks; a.segment_blocks = s.segment_blocks; a.segments = s.segments;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return with_channels<T>(width, {gate, value, out}, {strides[0], strides[1], strides[2], strides[3], strides[4], strides[5]}, [&](auto n) {
      constexpr int N = decltype(n)::value;
      const unsigned x = (unsigned)ceil_div(width, 64 * N);
      if (s.segments > 1) {
        segment_maps_kernel<T, N, kForward><<<dim3(x, (unsigned)n_batch, s.segments - 1), dim3(kWaves * 64), 0, stream>>>(a);
        a.state = a.state_copy;
      }
      if (kept) recurrence_kernel<T, N, true><<<dim3(x, (unsigned)n_batch, s.segments), dim3(kWaves * 64), 0, stream>>>(a);
      else recurrence_kernel<T, N, false><<<dim3(x, (unsigned)n_batch, s.segments), dim3(kWaves * 64), 0, stream>>>(a);
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
    a.segment_maps = static_cast<float*>(d_workspace);
    a.state_copy = a.segment_maps + n_batch * s.segments * 2 * width;
    a.steps = n_steps; a.width = width; a.blocks = s.blocks; a.segment_blocks = s.segment_blocks; a.segments = s.segments;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return with_channels<T>(width, {grad, gate, value, d_gate, d_value},
                            {strides[0], strides[1], strides[2], strides[3], strides[4], strides[5], strides[6], strides[7], strides[8], strides[9]},
                            [&](auto n) {
      constexpr int N = decltype(n)::value;
      const unsigned x = (unsigned)ceil_div(width, 64 * N);
      if (s.segments > 1) {
        segment_maps_kernel<T, N, kBackward><<<dim3(x, (unsigned)n_batch, s.segments - 1), dim3(kWaves * 64), 0, stream>>>(a);
        a.state = a.state_copy;
      }
      recurrence_grad_kernel<T, N><<<dim3(x, (unsigned)n_batch, s.segments), dim3(kWaves * 64), 0, stream>>>(a);
      return launched();
    });
  });
}

}  // extern "C"
