// Gated feed-forward block:  [g u] = x w_in^T,  hidden = act(g) u,  out = hidden w_out^T, and its B and W items.
//
// All products go through one kernel on the matrix cores.  out[m][n] = sum over k of M(m, k) N(n, k); either operand lies in memory
// with k running along its rows (kAlong) or down them (kDown):
//   F:  x w_in^T (both along; both projections in one tile, act and product in its epilogue),  hidden w_out^T (both along)
//   B:  grad w_out (N down; the derivative of the gate in its epilogue),  d_pre w_in (N down: one product over gate and up together)
//   W:  d_pre^T x,  grad^T hidden (both down)
// so that nothing is transposed in memory.  A tile of 64 k of either operand goes to LDS without passing registers, 16 bytes a lane;
// what is past an operand's end arrives as zeros (buffer loads check the range), so that sizes need not fit tiles.  Of an operand
// along k a lane reads its 8 k as they lie there; of one down k the transposing LDS read hands every lane 4 k of its column.  Pieces of 16 bytes are
// placed crosswise (xor with the row) so that a read meets every bank once.
//
// The N operand is the matrix instruction's first, so that a lane holds four neighbouring n of one m, which is how rows are written.
//
// Measured, bf16 8,192 x 4,096 x 10,752 (in PFLOP/s; a large library product 1.1 to 1.6): x w_in^T 1.17, hidden w_out^T 1.28, grad w_out 0.97 (it
// moves 1.06 GB of kept numbers and gradients besides, 215 us of 747), d_pre w_in 1.34, d_pre^T x 1.28, grad^T hidden 1.20, with the sums of shared tiles.  The
// matrix cores are busy two thirds of the time at 1.7 GHz: the card's power bounds it.
#include "ops_common.h"

#include <algorithm>

namespace fpsched {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

template <typename T>
struct Frag;
template <>
struct Frag<__bf16> {
  typedef __bf16 type __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x16 mul(type a, type b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Frag<_Float16> {
  typedef _Float16 type __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x16 mul(type a, type b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

enum { kAlong, kDown };                        // how k lies in an operand
enum { kStore, kGated, kGatedGrad };           // what becomes of a tile
constexpr int kDepth = 64;                     // k of a tile in LDS
constexpr unsigned kOutside = 0x80000000u;     // an offset behind the end of every tile's buffer

struct Operand {
  const void* data;
  int64_t stride;      // between rows, in elements
  int64_t extent;      // m or n
};

struct Gemm {
  Operand m, n;
  int64_t depth;             // k
  int64_t n_half;            // kGated, kGatedGrad: columns of the gate's half
  void* out;
  int64_t out_stride;
  int accumulate;
  int act;
  void* kept;                // kGated: written unless NULL; kGatedGrad: read, and written in its place
  int tiles_m, tiles_n;
  int whole, parts;          // tiles that one workgroup each works on; of the others, workgroups that share k
  int64_t part_depth;        // a share of k
  float* sums;               // their sums: [tile - whole][part][row][column]
};

// ---- activations: the value, and with it the derivative ----------------------------------------------------------------

__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.f + fast_exp(-x)); }

constexpr float kGeluScale = 1.5957691216057308f, kGeluCube = 0.044715f;   // 2 sqrt(2 / pi); (1 + tanh y) / 2 = sigmoid(2 y)

// act(g) and act'(g).  Of |g| beyond 40 the sigmoid is 0 or 1 to the last bit of what it is added to, and what else the derivative has of g is held there (squares
// would overflow, and 0 times infinity is none).
template <int ACT>
struct Activation {
  float value, slope;
  __device__ __forceinline__ explicit Activation(float g) {
    if constexpr (ACT == FPSCHED_RELU) {
      value = g < 0.f ? 0.f : g;   // (and none of what is none)
      slope = g > 0.f ? 1.f : 0.f;
    } else {
      const float p = sigmoid(ACT == FPSCHED_SILU ? g : kGeluScale * (g + kGeluCube * g * g * g)), c = fminf(fmaxf(g, -40.f), 40.f), rest = c * p * (1.f - p);
      value = g * p;
      slope = p + (ACT == FPSCHED_SILU ? rest : rest * kGeluScale * (1.f + 3.f * kGeluCube * c * c));
    }
  }
};
// f(Activation<act>'s number): the choice is made once for all elements that a lane has, so that their exponentials do not wait one for another
template <typename F>
__device__ __forceinline__ void with_activation(int act, F f) {
  if (act == FPSCHED_SILU) f(std::integral_constant<int, FPSCHED_SILU>());
  else if (act == FPSCHED_GELU) f(std::integral_constant<int, FPSCHED_GELU>());
  else f(std::integral_constant<int, FPSCHED_RELU>());
}

// ---- tiles in LDS --------------------------------------------------------------------------------------------------------

typedef __attribute__((address_space(3))) char lds_char;

// A tile of ROWS m (or n) by kDepth k.  kAlong: [row][8 pieces of 8 k], piece p of row r in place p ^ (r / 2 % 8): of 16
// rows that a read takes one piece each, no two are in the same banks.  kDown: [k][ROWS / 8 pieces of 8 rows], piece p of k in place p ^ (k % 4 * 4): the
// four k of a transposing read are in different quarters of the banks.
//
// A thread loads kLoads pieces of it; they are the same number of rows (or k) apart, so that one offset serves all, and what differs is the
// same for all lanes.  HALVES: rows from ROWS / 2 on are those of another place, n_half rows on.
template <int LAYOUT, int ROWS, int THREADS, bool HALVES>
struct Tile {
  static constexpr int kBytes = ROWS * kDepth * 2, kLoads = kBytes / 16 / THREADS;
  static constexpr int kPieces = LAYOUT == kAlong ? kDepth / 8 : ROWS / 8;       // in a row of LDS
  static constexpr int kApart = THREADS / kPieces;                               // rows of LDS between a thread's loads
  static constexpr int kHalfLoads = HALVES ? kLoads / 2 : kLoads;
  static_assert(kLoads * kApart == (LAYOUT == kAlong ? ROWS : kDepth) && (LAYOUT == kAlong ? kApart % 16 == 0 : kApart % 4 == 0), "places do not depend on the load");

  const char *base, *half_base;   // of the next tile to load
  int records;                    // bytes from there to the operand's end, as far as this tile's rows go
  int64_t step;                   // bytes to the tile behind it
  int apart, last_records;
  unsigned offset, last_offset;

  __device__ __forceinline__ void begin(const Operand& o, int64_t row0, int64_t n_half, int64_t depth, int thread) {
    const int r = thread / kPieces, place = thread % kPieces;
    const int stride = (int)o.stride, last_k = (int)((depth - 1) % kDepth) + 1;
    apart = kApart * stride * 2;
    if constexpr (LAYOUT == kAlong) {
      const int piece = place ^ (r >> 1 & 7);
      base = static_cast<const char*>(o.data) + row0 * o.stride * 2;
      half_base = base + n_half * o.stride * 2;
      const int64_t end = HALVES ? n_half : o.extent;
      const int rows = (int)min(end - row0, (int64_t)(HALVES ? ROWS / 2 : ROWS));
      records = ((rows - 1) * stride + (int)depth) * 2;
      step = kDepth * 2;
      last_records = 0;
      offset = (unsigned)(r * stride + piece * 8) * 2;
      last_offset = piece * 8 < last_k ? offset : kOutside;
    } else {
      const int piece = place ^ ((r & 3) << 2);
      const int left = (int)min(o.extent - row0, (int64_t)ROWS);
      base = half_base = static_cast<const char*>(o.data) + row0 * 2;
      records = ((kDepth - 1) * stride + left) * 2;
      last_records = ((last_k - 1) * stride + left) * 2;
      step = (int64_t)kDepth * stride * 2;
      offset = last_offset = piece * 8 < left ? (unsigned)(r * stride + piece * 8) * 2 : kOutside;
    }
  }

  __amdgpu_buffer_rsrc_t rsrc, half_rsrc;   // of the tile that is being loaded
  unsigned from;

  // Goes on to the next tile to load.  last: it is the last one; none: there is none, and what is loaded is zeros.
  __device__ __forceinline__ void next(bool last, bool none) {
    const int bytes = none ? 0 : LAYOUT == kDown && last ? last_records : records;
    from = last ? last_offset : offset;
    rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, bytes, 0x00027000);
    base += step;
    if constexpr (HALVES) {
      half_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(half_base), 0, bytes, 0x00027000);
      half_base += step;
    }
    if constexpr (LAYOUT == kAlong) records -= kDepth * 2;
  }
  // One of its kLoads pieces for each thread.
  __device__ __forceinline__ void load(lds_char* lds, int wave, int i) {
    if (HALVES && i >= kHalfLoads)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(half_rsrc, lds + (i * THREADS + wave * 64) * 16, 16, (int)from, (i - kHalfLoads) * apart, 0, 0);
    else
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, lds + (i * THREADS + wave * 64) * 16, 16, (int)from, i * apart, 0, 0);
  }

  // A lane's 8 k (16 step + 8 (lane / 32) ...) of row first + lane % 32.
  template <typename T>
  static __device__ __forceinline__ typename Frag<T>::type frag(const lds_char* lds, int first, int step, int lane) {
    if constexpr (LAYOUT == kAlong) {
      const int r = first + (lane & 31), piece = step * 2 + (lane >> 5);
      typedef __attribute__((address_space(3))) const typename Frag<T>::type lds_frag;
      return *(lds_frag*)(lds + r * (kDepth * 2) + ((piece ^ (r >> 1 & 7)) << 4));
    } else {
      const int k = step * 16 + (lane >> 5) * 8 + (lane >> 2 & 3), column = first + (lane >> 4 & 1) * 16 + (lane & 3) * 4;
      const int place = ((column >> 3) ^ ((k & 3) << 2)) * 16 + (column & 7) * 2;
      typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
      const s16x4 low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + k * (ROWS * 2) + place));
      const s16x4 high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + (k + 4) * (ROWS * 2) + place));
      const s16x8 both = __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7);
      return __builtin_bit_cast(typename Frag<T>::type, both);
    }
  }
};

// Tiles in an order in which those of one XCD (every eighth workgroup) are neighbours, eight rows of tiles high, for its L2.
__device__ __forceinline__ void tile_of(unsigned id, int tiles_m, int tiles_n, int* tm, int* tn) {
  const unsigned all = (unsigned)tiles_m * tiles_n, each = all >> 3, more = all & 7, xcd = id & 7, at = id >> 3;
  const unsigned place = xcd * each + min(xcd, more) + at;
  const unsigned strip = place / (8u * tiles_n), in = place - strip * 8u * tiles_n;
  const unsigned high = min(8u, tiles_m - strip * 8u);
  *tm = strip * 8 + in % high;
  *tn = in / high;
}

// What the forward pass keeps: g and u in 24 bits (a 32-bit number's first 24, rounded), off by 2^-16 of themselves at most.  In 16 bits they would
// add as much to the gradients' error as rounding d_pre does (bfloat16, 8,192 x 4,096 x 10,752: 3.0e-3 of the gradients' norm, and 2.4e-3 so).  The
// first 16 of all are [m][2 n_half], as d_pre will be; the last 8 of g and u are side by side in [m][n_half][2], where the same element of
// hidden will be: the backward pass writes the three in the place of the two, whose memory then lasts until the weights' gradients.
template <int N>
struct Kept {
  static_assert(N % 2 == 0, "two elements a word");
  Vec<unsigned, N / 2> g, u, last;

  static __device__ __forceinline__ unsigned bits(float x) { return x == x ? __float_as_uint(x) + 0x80u : 0x7fc00000u; }
  __device__ __forceinline__ void set(int pair, float gate0, float gate1, float up0, float up1) {
    const unsigned g0 = bits(gate0), g1 = bits(gate1), u0 = bits(up0), u1 = bits(up1);
    g.at[pair] = g0 >> 16 | (g1 & 0xffff0000u);
    u.at[pair] = u0 >> 16 | (u1 & 0xffff0000u);
    last.at[pair] = (g0 >> 8 & 0xff) | (u0 & 0xff00) | (g1 << 8 & 0xff0000) | (u1 << 16 & 0xff000000u);
  }
  // (the bytes of an element from its two words, and 0 for the last one)
  __device__ __forceinline__ float gate(int e) const {
    return __uint_as_float(__builtin_amdgcn_perm(g.at[e / 2], last.at[e / 2], e % 2 ? 0x0706020c : 0x0504000c));
  }
  __device__ __forceinline__ float up(int e) const {
    return __uint_as_float(__builtin_amdgcn_perm(u.at[e / 2], last.at[e / 2], e % 2 ? 0x0706030c : 0x0504010c));
  }

  static __device__ __forceinline__ unsigned short* first_of(const Gemm& a, int64_t m, int64_t n) {
    return static_cast<unsigned short*>(a.kept) + m * 2 * a.n_half + n;
  }
  static __device__ __forceinline__ unsigned char* last_of(const Gemm& a, int64_t m, int64_t n) {
    return static_cast<unsigned char*>(a.kept) + (a.m.extent * 2 + m) * 2 * a.n_half + 2 * n;
  }
  static __device__ __forceinline__ unsigned* words(void* p) { return static_cast<unsigned*>(p); }
  __device__ __forceinline__ void store(const Gemm& a, int64_t m, int64_t n) const {
    store_vec<unsigned, N / 2>(words(first_of(a, m, n)), g);
    store_vec<unsigned, N / 2>(words(first_of(a, m, n) + a.n_half), u);
    store_vec<unsigned, N / 2>(words(last_of(a, m, n)), last);
  }
  __device__ __forceinline__ void load(const Gemm& a, int64_t m, int64_t n) {
    g = load_vec<unsigned, N / 2>(words(first_of(a, m, n)));
    u = load_vec<unsigned, N / 2>(words(first_of(a, m, n) + a.n_half));
    last = load_vec<unsigned, N / 2>(words(last_of(a, m, n)));
  }
};

// What becomes of N neighbouring columns of a row, of the gate's half and the other one.  Hidden is rounded to the operands' type here, for the matrix
// cores' second product: relative to 64 bits, out is off by 2.3e-3 of its norm so (bfloat16; 2.9e-4 in float16), and by 1.64e-3 (2.07e-4) where only out itself
// is rounded.  (With what the rounding leaves off as a second operand, 1 to 16 tokens of 4,096 x 10,752 took 10 to 25 % longer; many tokens would take
// the second product twice.)
template <typename T, int N>
__device__ __forceinline__ void put_gated(const Gemm& a, int64_t m, int64_t n, const Vec<float, N>& gate, const Vec<float, N>& up) {
  Vec<T, N> h;
  Kept<N> kept;
  with_activation(a.act, [&](auto act) {
#pragma unroll
    for (int e = 0; e < N; ++e) h.at[e] = (T)(Activation<decltype(act)::value>(gate.at[e]).value * up.at[e]);
  });
#pragma unroll
  for (int e = 0; e < N; e += 2) kept.set(e / 2, gate.at[e], gate.at[e + 1], up.at[e], up.at[e + 1]);
  store_vec<T, N>(static_cast<T*>(a.out) + m * a.out_stride + n, h);
  if (a.kept) kept.store(a, m, n);
}

// What is read of 8 neighbouring columns of a row's place before they are written, where there are no halves.
template <int EPILOGUE, typename O>
struct Before {
  static constexpr bool kAny = std::is_same<O, float>::value;
  Vec<O, 8> v;
  __device__ __forceinline__ void load(const Gemm& a, int64_t m, int64_t n) {
    if (!kAny || !a.accumulate) return;
    const O* out = static_cast<const O*>(a.out) + m * a.out_stride + n;
    const Vec<O, 4> low = load_vec<O, 4>(out), high = load_vec<O, 4>(out + 4);   // (rows begin at 16 bytes)
#pragma unroll
    for (int e = 0; e < 4; ++e) v.at[e] = low.at[e], v.at[e + 4] = high.at[e];
  }
};
template <typename O>
struct Before<kGatedGrad, O> {
  static constexpr bool kAny = true;
  Kept<8> kept;
  __device__ __forceinline__ void load(const Gemm& a, int64_t m, int64_t n) { kept.load(a, m, n); }
};

// What becomes of them.
template <typename T, int EPILOGUE, typename O>
__device__ __forceinline__ void put_columns(const Gemm& a, int64_t m, int64_t n, const Vec<float, 8>& x, const Before<EPILOGUE, O>& before) {
  if constexpr (EPILOGUE == kGatedGrad) {
    // (d_pre is rounded to the operands' type, and hidden once more, for the matrix cores: the three gradients are off by as much as out is)
    asm volatile("" : : : "memory");   // (what is written below is of another type, in the place that `before` was read from)
    Vec<T, 8> dg, du, h;
    with_activation(a.act, [&](auto act) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const Activation<decltype(act)::value> of(before.kept.gate(e));
        const float up = before.kept.up(e);
        dg.at[e] = (T)(x.at[e] * up * of.slope);
        du.at[e] = (T)(x.at[e] * of.value);
        h.at[e] = (T)(of.value * up);
      }
    });
    T* out = reinterpret_cast<T*>(Kept<8>::first_of(a, m, n));
    store_vec<T, 8>(out, dg);
    store_vec<T, 8>(out + a.n_half, du);
    store_vec<T, 8>(reinterpret_cast<T*>(Kept<8>::last_of(a, m, n)), h);
  } else {
    O* out = static_cast<O*>(a.out) + m * a.out_stride + n;
    Vec<O, 8> v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v.at[e] = (O)(Before<EPILOGUE, O>::kAny && a.accumulate ? (float)before.v.at[e] + x.at[e] : x.at[e]);
    if constexpr (std::is_same<O, float>::value) {
      store_vec<O, 4>(out, {v.at[0], v.at[1], v.at[2], v.at[3]});
      store_vec<O, 4>(out + 4, {v.at[4], v.at[5], v.at[6], v.at[7]});
    } else {
      store_vec<O, 8>(out, v);
    }
  }
}

// All wavefronts of a workgroup have read what they read of LDS, and their loads to it have arrived but for the last ON_THEIR_WAY.
template <int ON_THEIR_WAY = 0>
__device__ __forceinline__ void meet() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "i"(ON_THEIR_WAY) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" : : : "memory");
}

template <typename T, int LM, int LN, int EPILOGUE, typename O, int BM, int BN, int kWavesM, int kWavesN, int kPlaces>
__global__ __launch_bounds__(kWavesM * kWavesN * 64) void gemm_kernel(Gemm a) {
  constexpr int kThreads = kWavesM * kWavesN * 64;
  constexpr int MF = BM / kWavesM / 32, NF = BN / kWavesN / 32, kStepsOfTile = kDepth / 16;
  constexpr bool kHalves = EPILOGUE == kGated;
  using TileM = Tile<LM, BM, kThreads, false>;
  using TileN = Tile<LN, BN, kThreads, kHalves>;
  constexpr int kTile = TileM::kBytes + TileN::kBytes;
  __shared__ __align__(1024) char lds[kPlaces * kTile];
  const int thread = threadIdx.x, lane = thread & 63, wave = __builtin_amdgcn_readfirstlane(thread >> 6);
  const int wave_m = wave / kWavesN, wave_n = wave % kWavesN;
  int tm, tn;
  const bool shared = (int)blockIdx.x >= a.whole;
  float* sums = nullptr;
  if (shared) {
    const int of = blockIdx.x - a.whole, part = of % a.parts;
    tile_of(a.whole + of / a.parts, a.tiles_m, a.tiles_n, &tm, &tn);
    sums = a.sums + (int64_t)of * BM * BN;
    const int64_t k0 = part * a.part_depth;
    a.m.data = static_cast<const T*>(a.m.data) + k0 * (LM == kAlong ? 1 : a.m.stride);
    a.n.data = static_cast<const T*>(a.n.data) + k0 * (LN == kAlong ? 1 : a.n.stride);
    a.depth = min(a.part_depth, a.depth - k0);
  } else {
    tile_of(blockIdx.x, a.tiles_m, a.tiles_n, &tm, &tn);
  }
  const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * (kHalves ? BN / 2 : BN);
  f32x16 acc[MF][NF] = {};
  const int tiles = (int)((a.depth + kDepth - 1) / kDepth);
  TileM tile_m;
  TileN tile_n;
  tile_m.begin(a.m, m0, 0, a.depth, thread);
  tile_n.begin(a.n, n0, a.n_half, a.depth, thread);
  typename Frag<T>::type fm[2][MF] = {}, fn[2][NF] = {};
  constexpr int kLoads = TileM::kLoads + TileN::kLoads;
  auto load = [&](lds_char* to, int i) {
    if (i < TileM::kLoads) tile_m.load(to, wave, i);
    else tile_n.load(to + TileM::kBytes, wave, i - TileM::kLoads);
  };
  auto next_tile = [&](int t) {
    tile_m.next(t == tiles - 1, t >= tiles);
    tile_n.next(t == tiles - 1, t >= tiles);
  };
  // A step's fragments are read between the products of the one in front of it, the first ones of a tile between the last products of the
  // tile before, and the next tile's loads are issued between the first of a tile's products: any of them by itself would keep a wavefront from
  // its products for as long as the wavefronts of the compute unit need to issue theirs.
  // (That the two places are different ones is said by __restrict: the compiler would else wait for what is on its way to one in front of
  // each transposing read of the other.)
  auto work_on = [&](int t, lds_char* __restrict place, lds_char* __restrict other) __attribute__((always_inline)) {
    next_tile(t + kPlaces - 1);
#pragma unroll
    for (int step = 0; step < kStepsOfTile; ++step) {
      const int to = step & 1, of = to ^ 1;   // fragments to read, to multiply (in the first tile's first step, zeros)
#pragma unroll
      for (int j = 0; j < NF; ++j)
        fn[to][j] = TileN::template frag<T>(place + TileM::kBytes, kHalves ? j / (NF / 2) * (BN / 2) + (wave_n * (NF / 2) + j % (NF / 2)) * 32 : (wave_n * NF + j) * 32, step, lane);
#pragma unroll
      for (int i = 0; i < MF; ++i) {
        fm[to][i] = TileM::template frag<T>(place, (wave_m * MF + i) * 32, step, lane);
#pragma unroll
        for (int j = 0; j < NF; ++j) acc[i][j] = Frag<T>::mul(fn[of][j], fm[of][i], acc[i][j]);
        constexpr int kTurns = MF;   // of products among which the loads are spread: a step's (over a tile's they come late: 7 % slower)
        const int turn = step * MF + i;
#pragma unroll
        for (int l = turn * kLoads / kTurns; l < (turn + 1) * kLoads / kTurns && l < kLoads; ++l) load(other, l);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  lds_char* const room = (lds_char*)lds;
#pragma unroll
  for (int p = 0; p < kPlaces - 1; ++p) {
    next_tile(p);
#pragma unroll
    for (int l = 0; l < kLoads; ++l) load(room + p * kTile, l);
  }
  for (int t = 0; t < tiles; ++t) {
    meet<kLoads * (kPlaces - 2)>();
    work_on(t, room + t % kPlaces * kTile, room + (t + kPlaces - 1) % kPlaces * kTile);
  }
#pragma unroll
  for (int i = 0; i < MF; ++i)
#pragma unroll
    for (int j = 0; j < NF; ++j) acc[i][j] = Frag<T>::mul(fn[(kStepsOfTile - 1) & 1][j], fm[(kStepsOfTile - 1) & 1][i], acc[i][j]);
  // A wavefront's 32 rows at a time go through LDS, so that rows are read and written 8 columns a lane.
  constexpr int kPad = NF * 32 + 4;   // floats between rows: 16 rows' pieces of 16 bytes are in different banks
  meet();   // (the loads of the tile behind the last one, zeros, among them)
  float* mine = reinterpret_cast<float*>(lds) + wave * 32 * kPad;
  static_assert(kThreads / 64 * 32 * kPad * 4 <= kPlaces * kTile, "the rows fit");
  constexpr int kColumns = (kHalves ? NF / 2 : NF) * 32, kLanes = kColumns / 8, kRows = 64 / kLanes;   // of the output; lanes of a row, rows at a time
  const int64_t n = n0 + wave_n * kColumns + lane % kLanes * 8;
  // What is read there is on its way 32 rows ahead.  (Read where it is needed, one wait after another: the gate's gradient of 8,192 x 10,752 x 4,096
  // 799 us, and 778 so; weights' gradients added to what is there, 2,048 x 4,096 x 10,752, 685 and 648.)
  using Ahead = Before<EPILOGUE, O>;
  Ahead before[32 / kRows];
  auto read_ahead = [&](int i, int p) {
    const int64_t m = m0 + (wave_m * MF + i) * 32 + p * kRows + lane / kLanes;
    if (Ahead::kAny && !kHalves && !shared && m < a.m.extent && n < a.n.extent) before[p].load(a, m, n);
  };
#pragma unroll
  for (int p = 0; p < 32 / kRows; ++p) read_ahead(0, p);
#pragma unroll
  for (int i = 0; i < MF; ++i) {
#pragma unroll
    for (int j = 0; j < NF; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        store_vec<float, 4>(mine + (lane & 31) * kPad + j * 32 + q * 8 + (lane >> 5) * 4,
                            {acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]});
    __builtin_amdgcn_wave_barrier();
    const int64_t rows = m0 + (wave_m * MF + i) * 32;
#pragma unroll
    for (int p = 0; p < 32 / kRows; ++p) {
      const int r = p * kRows + lane / kLanes;
      const int64_t m = rows + r;
      const float* from = mine + r * kPad + lane % kLanes * 8;
      if (shared) {   // (a tile's own rows and columns, the other half's behind the gate's)
        if (m >= a.m.extent) continue;
        float* to = sums + ((wave_m * MF + i) * 32 + r) * BN + wave_n * kColumns + lane % kLanes * 8;
        store_vec<float, 4>(to, load_vec<float, 4>(from));
        store_vec<float, 4>(to + 4, load_vec<float, 4>(from + 4));
        if constexpr (kHalves) {
          store_vec<float, 4>(to + BN / 2, load_vec<float, 4>(from + kColumns));
          store_vec<float, 4>(to + BN / 2 + 4, load_vec<float, 4>(from + kColumns + 4));
        }
        continue;
      }
      const Vec<float, 4> x0 = load_vec<float, 4>(from), x1 = load_vec<float, 4>(from + 4);
      if constexpr (kHalves) {
        const Vec<float, 4> u0 = load_vec<float, 4>(from + kColumns), u1 = load_vec<float, 4>(from + kColumns + 4);
        if (m >= a.m.extent || n >= a.n_half) continue;
        put_gated<T, 8>(a, m, n, {x0.at[0], x0.at[1], x0.at[2], x0.at[3], x1.at[0], x1.at[1], x1.at[2], x1.at[3]},
                     {u0.at[0], u0.at[1], u0.at[2], u0.at[3], u1.at[0], u1.at[1], u1.at[2], u1.at[3]});
      } else {
        if (m >= a.m.extent || n >= a.n.extent) continue;
        put_columns<T, EPILOGUE, O>(a, m, n, {x0.at[0], x0.at[1], x0.at[2], x0.at[3], x1.at[0], x1.at[1], x1.at[2], x1.at[3]}, before[p]);
        if (i + 1 < MF) read_ahead(i + 1, p);
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// ---- few tokens --------------------------------------------------------------------------------------------------------
//
// At most 16 rows: the weights are read once, and that is what it takes.  A workgroup has 16 columns (16 of the gate's and the same of the
// other half's), its wavefronts a share of k each; weights go from memory to the matrix instruction's registers, 128 bytes of
// a row at a time by four lanes, and the rows of x beside them from cache in the same order of k.  (More rows, in sixteens: 17 to 64 of
// 4,096 took 62 to 126 us, and the tiles with k in parts take 56 to 65.)
constexpr int kFewRows = 16;

template <typename T>
struct Frag16;
typedef float f32x4 __attribute__((ext_vector_type(4)));
template <>
struct Frag16<__bf16> {
  static __device__ __forceinline__ f32x4 mul(Frag<__bf16>::type a, Frag<__bf16>::type b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Frag16<_Float16> {
  static __device__ __forceinline__ f32x4 mul(Frag<_Float16>::type a, Frag<_Float16>::type b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

template <typename T, int EPILOGUE, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void few_rows_kernel(Gemm a) {
  constexpr int kSets = EPILOGUE == kGated ? 2 : 1;
  using F = typename Frag<T>::type;
  __shared__ __align__(16) float sums[WAVES][kSets][64][4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int64_t columns = EPILOGUE == kGated ? a.n_half : a.n.extent;
  const int at = lane & 15, group = lane >> 4;
  const T* weights[kSets];
#pragma unroll
  for (int s = 0; s < kSets; ++s) weights[s] = static_cast<const T*>(a.n.data) + (min(n0 + at, columns - 1) + s * a.n_half) * a.n.stride;
  const T* row = static_cast<const T*>(a.m.data) + min((int64_t)at, a.m.extent - 1) * a.m.stride;
  f32x4 acc[kSets] = {};
  constexpr int kPiece = 64, kAhead = 4;   // k that the four groups of lanes have together; pieces on their way
  const int64_t share = (a.depth + kPiece * WAVES - 1) / (kPiece * WAVES) * kPiece;
  const int64_t begin = wave * share, end = min(begin + share, a.depth);
  for (int64_t k0 = begin; k0 < end; k0 += kAhead * kPiece) {
    F w[kAhead][kSets][2], x[kAhead][2];
#pragma unroll
    for (int p = 0; p < kAhead; ++p)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int64_t k = k0 + p * kPiece + group * 16 + j * 8;
        const bool in = k < end;   // (k is a multiple of 8, as is the depth)
        const int64_t from = in ? k : 0;
#pragma unroll
        for (int s = 0; s < kSets; ++s) {
          w[p][s][j] = *reinterpret_cast<const F*>(weights[s] + from);
          if (!in) w[p][s][j] = F{};
        }
        x[p][j] = *reinterpret_cast<const F*>(row + from);
        if (!in) x[p][j] = F{};
      }
#pragma unroll
    for (int p = 0; p < kAhead; ++p)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int s = 0; s < kSets; ++s) acc[s] = Frag16<T>::mul(w[p][s][j], x[p][j], acc[s]);
  }
#pragma unroll
  for (int s = 0; s < kSets; ++s) *reinterpret_cast<f32x4*>(sums[wave][s][lane]) = acc[s];
  __syncthreads();
  // four columns of a row a lane
  const int64_t m = at, n = n0 + group * 4;
  if (wave || m >= a.m.extent || n >= columns) return;
  f32x4 total[kSets] = {};
#pragma unroll
  for (int s = 0; s < kSets; ++s)
#pragma unroll
    for (int w = 0; w < WAVES; ++w) total[s] += *reinterpret_cast<const f32x4*>(sums[w][s][lane]);
  if constexpr (EPILOGUE == kGated) {
    put_gated<T, 4>(a, m, n, {total[0][0], total[0][1], total[0][2], total[0][3]}, {total[1][0], total[1][1], total[1][2], total[1][3]});
  } else {
    store_vec<T, 4>(static_cast<T*>(a.out) + m * a.out_stride + n, {(T)total[0][0], (T)total[0][1], (T)total[0][2], (T)total[0][3]});
  }
}

template <typename T, int EPILOGUE>
int few_rows(const Gemm& a, hipStream_t stream) {
  constexpr int W = EPILOGUE == kGated ? 4 : 8;   // (the second product has fewer columns and a longer k)
  few_rows_kernel<T, EPILOGUE, W><<<dim3((unsigned)ceil_div(EPILOGUE == kGated ? a.n_half : a.n.extent, 16)), dim3(W * 64), 0, stream>>>(a);
  return launched();
}

// A product of nothing: the zeros that it leaves.
template <typename O>
__global__ __launch_bounds__(256) void zero_rows_kernel(O* out, int64_t stride, int64_t rows, int64_t columns) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * columns; i += (int64_t)gridDim.x * 256)
    out[i / columns * stride + i % columns] = (O)0.f;
}

// The sums of the workgroups that share a tile, added up in order, and what becomes of them.
template <typename T, int EPILOGUE, typename O, int SIDE>
__global__ __launch_bounds__(256) void add_shares_kernel(Gemm a) {
  constexpr int kColumns = EPILOGUE == kGated ? SIDE / 2 : SIDE, kPieces = kColumns / 8, kGroups = SIDE * kPieces / 256;
  const int tile = blockIdx.x / kGroups, at = blockIdx.x % kGroups * 256 + threadIdx.x, r = at / kPieces, c = at % kPieces * 8;
  int tm, tn;
  tile_of(a.whole + tile, a.tiles_m, a.tiles_n, &tm, &tn);
  const int64_t m = (int64_t)tm * SIDE + r, n = (int64_t)tn * kColumns + c;
  if (m >= a.m.extent || n >= (EPILOGUE == kGated ? a.n_half : a.n.extent)) return;
  auto total = [&](int column) {
    Vec<float, 8> sum = {};
    const float* x = a.sums + ((int64_t)tile * a.parts * SIDE + r) * SIDE + column;
    for (int p = 0; p < a.parts; ++p, x += SIDE * SIDE) {
      const Vec<float, 4> low = load_vec<float, 4>(x), high = load_vec<float, 4>(x + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum.at[e] += low.at[e], sum.at[e + 4] += high.at[e];
    }
    return sum;
  };
  if constexpr (EPILOGUE == kGated) put_gated<T, 8>(a, m, n, total(c), total(SIDE / 2 + c));
  else {
    Before<EPILOGUE, O> before;
    before.load(a, m, n);
    put_columns<T, EPILOGUE, O>(a, m, n, total(c), before);
  }
}

// How a product is cut: into tiles of 256 x 256, one workgroup to a compute unit, or of 128 x 128, two of them; and the tiles
// of the last round, where they leave compute units idle, into shares of k, whose sums another kernel adds up.  What decides is an estimate:
// a step of 64 k takes 1.63 us and what becomes of a tile 5 (of the gate's gradient 30: it reads and writes 0.8 MB a tile); of the small tiles 1.1 us, 0.65 with one workgroup to a compute
// unit (a fifth less with four places; counted so, cuts were no better), and 3; sums are written and read at 8 TB/s, in a launch more.  (Measured, whole and so: W of
// 8,192 x 4,096 x 10,752, whose 1,344 tiles are five rounds and a quarter, 1.80 and 1.69 ms; d_x of 509 x 2,560 x 6,912, 80 small tiles of 216 steps, 134
// and 45 us.)
struct Split {
  bool large;
  // Small tiles, one to a compute unit, of eight steps or more: four places in LDS instead of two, so that three tiles of loads are on their way (F of 200 x
  // 2,560 x 6,912 42 us instead of 50, B of 509 73 instead of 79; with one to four steps a kernel takes a microsecond more).
  bool deep;
  int tiles_m, tiles_n, whole, parts;
  int64_t part_depth;
};

Split split(int64_t m, int64_t n, int64_t depth, bool heavy) {
  Split best = {};
  double least = 0;
  const int64_t steps = ceil_div(depth, kDepth);
  for (const bool large : {true, false}) {
    const int64_t side = large ? 256 : 128, slots = large ? 256 : 512, tm = ceil_div(m, side), tn = ceil_div(n, side), tiles = tm * tn;
    if (large && tiles < 64) continue;
    const double step = large ? 1.63 : 1.1, end = (large ? 5 : 3) * (heavy ? 6 : 1);
    const int64_t rounds = tiles / slots, rest = tiles % slots;
    for (int parts = 1; parts <= 16 && (parts == 1 || (rest && steps >= 4 * parts)); ++parts) {
      const int64_t each = ceil_div(steps, parts), used = ceil_div(steps, each);   // (as many shares as there is something for)
      const double alone = !large && rounds == 0 && rest * used <= 256 ? 0.65 : step;
      const double us = rounds * (steps * step + end) + (rest ? ceil_div(rest * used, slots) * (each * alone + (used > 1 ? 3 : end)) : 0) +
                        (used > 1 ? 4 + end + rest * used * (std::min(m, side) * side * 8 / 8e6) : 0);
      if (least == 0 || us < least) {
        least = us;
        best = {large, !large && tiles - rest + rest * used <= 256 && each >= 8, (int)std::min<int64_t>(tm, INT32_MAX), (int)std::min<int64_t>(tn, INT32_MAX), (int)std::min<int64_t>(used > 1 ? tiles - rest : tiles, INT32_MAX), (int)used, each * kDepth};
      }
    }
  }
  return best;
}

size_t split_bytes(int64_t m, int64_t n, int64_t depth, bool heavy) {
  const Split s = split(m, n, depth, heavy);
  const size_t side = s.large ? 256 : 128;
  return s.parts > 1 ? ((size_t)s.tiles_m * s.tiles_n - s.whole) * s.parts * side * side * sizeof(float) : 0;
}

template <typename T, int LM, int LN, int EPILOGUE, typename O>
int gemm(Gemm a, void* workspace, hipStream_t stream) {
  const Split s = split(a.m.extent, a.n.extent, a.depth, EPILOGUE == kGatedGrad);   // (of kGated, n has both halves)
  const int64_t tiles = (int64_t)s.tiles_m * s.tiles_n;
  if (tiles > 0x7fffff) return FPSCHED_EUNSUPPORTED;   // (workgroups and their numbers are 32-bit)
  a.tiles_m = s.tiles_m;
  a.tiles_n = s.tiles_n;
  a.whole = s.whole;
  a.parts = s.parts;
  a.part_depth = s.part_depth;
  a.sums = static_cast<float*>(workspace);
  const int shared = (int)(tiles - s.whole);
  const dim3 grid(s.whole + shared * s.parts);
  constexpr int kHalf = EPILOGUE == kGated ? 2 : 1;
  if (s.large) {
    gemm_kernel<T, LM, LN, EPILOGUE, O, 256, 256, 2, 4, 2><<<grid, dim3(512), 0, stream>>>(a);
    if (shared) add_shares_kernel<T, EPILOGUE, O, 256><<<dim3(shared * 32 / kHalf), dim3(256), 0, stream>>>(a);
  } else {
    if (s.deep) gemm_kernel<T, LM, LN, EPILOGUE, O, 128, 128, 2, 2, 4><<<grid, dim3(256), 0, stream>>>(a);
    else gemm_kernel<T, LM, LN, EPILOGUE, O, 128, 128, 2, 2, 2><<<grid, dim3(256), 0, stream>>>(a);
    if (shared) add_shares_kernel<T, EPILOGUE, O, 128><<<dim3(shared * 8 / kHalf), dim3(256), 0, stream>>>(a);
  }
  return launched();
}

constexpr int64_t kMostStride = 1 << 21;   // (256 rows of a tile are within 2^31 bytes)

bool row_ok(const void* p, int64_t stride) { return p && aligned(p, 16) && stride % 8 == 0 && stride <= kMostStride; }

int check_sizes(int type, int act, int64_t n_tokens, int64_t width, int64_t hidden_width) {
  if (type != FPSCHED_BF16 && type != FPSCHED_F16) return FPSCHED_EINVAL;
  if (act < FPSCHED_SILU || act > FPSCHED_RELU || n_tokens < 0 || n_tokens > 0x7fffffffll) return FPSCHED_EINVAL;
  if (width < 8 || hidden_width < 8 || width % 8 || hidden_width % 8 || width > kMostStride || hidden_width > kMostStride / 2) return FPSCHED_EINVAL;
  return FPSCHED_OK;
}

// Room for the largest of the products' parts.
size_t workspace_for(int64_t t, int64_t k, int64_t f) {
  if (t == 0) return 16;
  const size_t forward = t <= kFewRows ? 0 : std::max(split_bytes(t, 2 * f, k, false), split_bytes(t, k, f, false));
  const size_t backward = std::max(split_bytes(t, f, k, true), split_bytes(t, k, 2 * f, false));
  const size_t weights = std::max(split_bytes(2 * f, k, t, false), split_bytes(k, f, t, false));
  return std::max<size_t>({16, forward, backward, weights});
}

int check_workspace(const void* workspace, size_t bytes, int64_t t, int64_t k, int64_t f) {
  const size_t needed = workspace_for(t, k, f);
  if (needed > 16 && (!workspace || !aligned(workspace, 16))) return FPSCHED_EINVAL;
  return needed > 16 && bytes < needed ? FPSCHED_ENOMEM : FPSCHED_OK;
}

template <typename F>
int with_half_type(int type, F f) {
  return type == FPSCHED_BF16 ? f(__bf16()) : f(_Float16());
}

}  // namespace
}  // namespace fpsched

using namespace fpsched;

extern "C" {

size_t fpsched_op_ffn_workspace_bytes(int64_t n_tokens, int64_t width, int64_t hidden_width) {
  if (check_sizes(FPSCHED_BF16, 0, n_tokens, width, hidden_width) != FPSCHED_OK) return 0;
  return workspace_for(n_tokens, width, hidden_width);
}

int fpsched_op_ffn(int device_id, int type, int act, int64_t n_tokens, int64_t width, int64_t hidden_width, const void* x,
                   int64_t x_stride, const void* w_in, const void* w_out, void* kept, void* hidden, void* out, int64_t out_stride,
                   void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  if (check_sizes(type, act, n_tokens, width, hidden_width) != FPSCHED_OK || x_stride < width || out_stride < width) return FPSCHED_EINVAL;
  if (device_id < 0) return FPSCHED_ENODEV;
  if (n_tokens == 0) return FPSCHED_OK;
  if (!row_ok(x, x_stride) || !row_ok(out, out_stride) || !row_ok(w_in, 0) || !row_ok(w_out, 0) || !row_ok(hidden, 0) || (kept && !aligned(kept, 16)))
    return FPSCHED_EINVAL;
  const int room = check_workspace(d_workspace, workspace_bytes, n_tokens, width, hidden_width);
  if (room != FPSCHED_OK) return room;
  OpsDevice g(device_id);
  if (!g.ok) return FPSCHED_EHIP;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  return with_half_type(type, [&](auto zero) {
    using T = decltype(zero);
    Gemm a = {};
    a.m = {x, x_stride, n_tokens}; a.n = {w_in, width, 2 * hidden_width}; a.depth = width; a.n_half = hidden_width;
    a.out = hidden; a.out_stride = hidden_width; a.act = act; a.kept = kept;
    const int first = n_tokens <= kFewRows ? few_rows<T, kGated>(a, stream) : gemm<T, kAlong, kAlong, kGated, T>(a, d_workspace, stream);
    if (first != FPSCHED_OK) return first;
    Gemm b = {};
    b.m = {hidden, hidden_width, n_tokens}; b.n = {w_out, hidden_width, width}; b.depth = hidden_width;
    b.out = out; b.out_stride = out_stride;
    return n_tokens <= kFewRows ? few_rows<T, kStore>(b, stream) : gemm<T, kAlong, kAlong, kStore, T>(b, d_workspace, stream);
  });
}

int fpsched_op_ffn_input_grad(int device_id, int type, int act, int64_t n_tokens, int64_t width, int64_t hidden_width,
                              const void* grad, int64_t grad_stride, const void* w_in, const void* w_out, void* kept,
                              void* d_x, int64_t d_x_stride, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  if (check_sizes(type, act, n_tokens, width, hidden_width) != FPSCHED_OK || grad_stride < width || d_x_stride < width) return FPSCHED_EINVAL;
  if (device_id < 0) return FPSCHED_ENODEV;
  if (n_tokens == 0) return FPSCHED_OK;
  if (!row_ok(grad, grad_stride) || !row_ok(d_x, d_x_stride) || !row_ok(w_in, 0) || !row_ok(w_out, 0) || !row_ok(kept, 0))
    return FPSCHED_EINVAL;
  const int room = check_workspace(d_workspace, workspace_bytes, n_tokens, width, hidden_width);
  if (room != FPSCHED_OK) return room;
  OpsDevice g(device_id);
  if (!g.ok) return FPSCHED_EHIP;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  return with_half_type(type, [&](auto zero) {
    using T = decltype(zero);
    Gemm a = {};
    a.m = {grad, grad_stride, n_tokens}; a.n = {w_out, hidden_width, hidden_width}; a.depth = width; a.n_half = hidden_width;
    a.act = act; a.kept = kept;
    const int first = gemm<T, kAlong, kDown, kGatedGrad, T>(a, d_workspace, stream);
    if (first != FPSCHED_OK) return first;
    Gemm b = {};
    b.m = {kept, 2 * hidden_width, n_tokens}; b.n = {w_in, width, width}; b.depth = 2 * hidden_width;
    b.out = d_x; b.out_stride = d_x_stride;
    return gemm<T, kAlong, kDown, kStore, T>(b, d_workspace, stream);
  });
}

int fpsched_op_ffn_weight_grad(int device_id, int type, int64_t n_tokens, int64_t width, int64_t hidden_width, const void* x,
                               int64_t x_stride, const void* grad, int64_t grad_stride, const void* kept, int out_type, void* d_w_in, void* d_w_out, int accumulate, void* d_workspace,
                               size_t workspace_bytes, void* hip_stream) {
  if (check_sizes(type, 0, n_tokens, width, hidden_width) != FPSCHED_OK || x_stride < width || grad_stride < width) return FPSCHED_EINVAL;
  if ((out_type != type && out_type != FPSCHED_F32) || (accumulate && out_type != FPSCHED_F32)) return FPSCHED_EINVAL;
  if (device_id < 0) return FPSCHED_ENODEV;
  if (!row_ok(d_w_in, 0) || !row_ok(d_w_out, 0)) return FPSCHED_EINVAL;
  if (n_tokens > 0 && (!row_ok(x, x_stride) || !row_ok(grad, grad_stride) || !row_ok(kept, 0))) return FPSCHED_EINVAL;
  if (n_tokens == 0 && accumulate) return FPSCHED_OK;
  const int room = check_workspace(d_workspace, workspace_bytes, n_tokens, width, hidden_width);
  if (room != FPSCHED_OK) return room;
  OpsDevice g(device_id);
  if (!g.ok) return FPSCHED_EHIP;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  return with_half_type(type, [&](auto zero) {
    using T = decltype(zero);
    auto go = [&](auto zero_out) {
      using O = decltype(zero_out);
      if (n_tokens == 0) {
        zero_rows_kernel<O><<<dim3(1024), dim3(256), 0, stream>>>(static_cast<O*>(d_w_in), width, 2 * hidden_width, width);
        zero_rows_kernel<O><<<dim3(1024), dim3(256), 0, stream>>>(static_cast<O*>(d_w_out), hidden_width, width, hidden_width);
        return launched();
      }
      Gemm a = {};
      a.m = {kept, 2 * hidden_width, 2 * hidden_width}; a.n = {x, x_stride, width}; a.depth = n_tokens;
      a.out = d_w_in; a.out_stride = width; a.accumulate = accumulate;
      const int first = gemm<T, kDown, kDown, kStore, O>(a, d_workspace, stream);
      if (first != FPSCHED_OK) return first;
      Gemm b = {};
      b.m = {grad, grad_stride, width}; b.n = {static_cast<const T*>(kept) + n_tokens * 2 * hidden_width, hidden_width, hidden_width}; b.depth = n_tokens;
      b.out = d_w_out; b.out_stride = hidden_width; b.accumulate = accumulate;
      return gemm<T, kDown, kDown, kStore, O>(b, d_workspace, stream);
    };
    if (out_type == FPSCHED_F32) return go(float());
    return go(T());
  });
}

}  // extern "C"
