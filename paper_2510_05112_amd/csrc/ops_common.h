// What the stage operators share: element types, vectors of them, reductions over a wavefront, and the host side of a call.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/fpsched_ops.h"

namespace fpsched {

template <typename T, int N>
struct alignas(sizeof(T) * N) Vec {
  T at[N];
};

template <typename T, int N>
__device__ __forceinline__ Vec<T, N> load_vec(const T* from) {
  return *reinterpret_cast<const Vec<T, N>*>(from);
}
template <typename T, int N>
__device__ __forceinline__ void store_vec(T* to, const Vec<T, N>& v) {
  *reinterpret_cast<Vec<T, N>*>(to) = v;
}

// The same from and to any element's address in global memory (one access of 16 bytes nevertheless).
template <typename T, int N>
__device__ __forceinline__ Vec<T, N> load_any(const T* from) {
  Vec<T, N> v;
  __builtin_memcpy(&v, from, sizeof(v));
  return v;
}
template <typename T, int N>
__device__ __forceinline__ void store_any(T* to, const Vec<T, N>& v) {
  __builtin_memcpy(to, &v, sizeof(v));
}

// elements of 16 bytes
template <typename T>
constexpr int kWide = 16 / (int)sizeof(T);

__device__ __forceinline__ int64_t token_at(const void* tokens, int tokens64, int64_t i) {
  return tokens64 ? static_cast<const int64_t*>(tokens)[i] : (int64_t)static_cast<const int32_t*>(tokens)[i];
}

// exp and log by the hardware's base-2 forms (an error of about 2^-23 in the result, 2^-24 times the argument in exp's; what exp gives below 2^-126 is 0)
__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f); }
__device__ __forceinline__ float fast_log(float x) { return __logf(x); }

// ---- host --------------------------------------------------------------------------------------------------------------

struct OpsDevice {   // makes a GPU the current one for a call's launches
  int prev = -1;
  bool ok = false;
  explicit OpsDevice(int dev) {
    if (hipGetDevice(&prev) != hipSuccess) { prev = -1; return; }
    ok = prev == dev || hipSetDevice(dev) == hipSuccess;
    if (prev == dev) prev = -1;
  }
  ~OpsDevice() {
    if (prev >= 0) (void)hipSetDevice(prev);
  }
};

constexpr int64_t kMostGroups = (1 << 24) - 1, kMostWaves = (1 << 26) - 1;   // workgroups of 256 and of 64 along a grid's x, which has room for 2^32 - 1 lanes

inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t round_up(size_t n, size_t to) { return (n + to - 1) / to * to; }
inline int launched() { return hipGetLastError() == hipSuccess ? FPSCHED_OK : FPSCHED_EHIP; }

// f(T()) with the element type of `type`; FPSCHED_EINVAL for another number
template <typename F>
int with_type(int type, F f) {
  switch (type) {
    case FPSCHED_BF16: return f(__bf16());
    case FPSCHED_F16: return f(_Float16());
    case FPSCHED_F32: return f(float());
  }
  return FPSCHED_EINVAL;
}

}  // namespace fpsched
