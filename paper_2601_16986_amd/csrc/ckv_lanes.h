// What the kernels of this library share: vector types, moves and sums across the lanes of a wavefront, stores and loads that are
// coherent across the chip one by one, and the selection of the smallest keys that a workgroup holds in registers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ckv {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef unsigned long long u64;
constexpr int kThreads = 256;
constexpr int kWideThreads = 1024;        // kernels with one workgroup per unit and few units

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Cross-lane moves inside a row of 16 lanes without going through LDS.
template <int kCtrl>
__device__ __forceinline__ int dpp_i32(int v) {
  return __builtin_amdgcn_update_dpp(0, v, kCtrl, 0xF, 0xF, true);
}
constexpr int kDppQuadSwap1 = 0xB1;      // quad_perm [1,0,3,2]
constexpr int kDppQuadSwap2 = 0x4E;      // quad_perm [2,3,0,1]
constexpr int kDppRowHalfMirror = 0x141;
constexpr int kDppRowMirror = 0x140;
constexpr int kDppRowShl = 0x100, kDppRowShr = 0x110;      // + 1 .. 15: from so many lanes up / down, 0 from beyond the row

// Lanes j, j + 16, j + 32 and j + 48 into one value, the same in all four: op(op(v0, v1), op(v2, v3)).  By swaps of rows, without a trip through LDS.
template <class Op>
__device__ __forceinline__ float rows_combine(float v, Op op) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return op(__uint_as_float(h[0]), __uint_as_float(h[1]));
}

// Maxima and minima that are NaN if an operand is.
__device__ __forceinline__ float min2(float a, float b) { return __builtin_elementwise_minimum(a, b); }
__device__ __forceinline__ float max2(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float max3(float a, float b, float c) { return max2(max2(a, b), c); }

// Sum over the 64 lanes, same fixed order in every lane: butterfly inside each
// row of 16 lanes, then the four row sums are read out and added.
__device__ __forceinline__ float wave_sum_f32(float v) {
  v += __int_as_float(dpp_i32<kDppQuadSwap1>(__float_as_int(v)));
  v += __int_as_float(dpp_i32<kDppQuadSwap2>(__float_as_int(v)));
  v += __int_as_float(dpp_i32<kDppRowHalfMirror>(__float_as_int(v)));
  v += __int_as_float(dpp_i32<kDppRowMirror>(__float_as_int(v)));
  const float r0 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 0));
  const float r1 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 16));
  const float r2 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 32));
  const float r3 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 48));
  return (r0 + r1) + (r2 + r3);
}

__device__ __forceinline__ int wave_sum_i32(int v) {
  v += dpp_i32<kDppQuadSwap1>(v);
  v += dpp_i32<kDppQuadSwap2>(v);
  v += dpp_i32<kDppRowHalfMirror>(v);
  v += dpp_i32<kDppRowMirror>(v);
  return __builtin_amdgcn_readlane(v, 0) + __builtin_amdgcn_readlane(v, 16) + __builtin_amdgcn_readlane(v, 32) +
         __builtin_amdgcn_readlane(v, 48);
}

template <int kCtrl>
__device__ __forceinline__ u64 dpp_u64(u64 v) {
  const uint32_t lo = (uint32_t)dpp_i32<kCtrl>((int)(uint32_t)v);
  const uint32_t hi = (uint32_t)dpp_i32<kCtrl>((int)(uint32_t)(v >> 32));
  return ((u64)hi << 32) | lo;
}

__device__ __forceinline__ u64 readlane_u64(u64 v, int lane) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane);
  return ((u64)hi << 32) | lo;
}

template <int kCtrl>
__device__ __forceinline__ double dpp_f64(double v) {
  return __longlong_as_double((long long)dpp_u64<kCtrl>((u64)__double_as_longlong(v)));
}
__device__ __forceinline__ double readlane_f64(double v, int lane) { return __longlong_as_double((long long)readlane_u64((u64)__double_as_longlong(v), lane)); }

__device__ __forceinline__ u64 wave_sum_u64(u64 v) {
  v += dpp_u64<kDppQuadSwap1>(v);
  v += dpp_u64<kDppQuadSwap2>(v);
  v += dpp_u64<kDppRowHalfMirror>(v);
  v += dpp_u64<kDppRowMirror>(v);
  return (readlane_u64(v, 0) + readlane_u64(v, 16)) + (readlane_u64(v, 32) + readlane_u64(v, 48));
}

// Sum over the lanes up to each: inside its row of 16, then the rows before.  (Six shuffles through LDS take 0.3 us, one after another.)
__device__ __forceinline__ int wave_scan_i32(int v, int lane) {
  v += dpp_i32<kDppRowShr + 1>(v);
  v += dpp_i32<kDppRowShr + 2>(v);
  v += dpp_i32<kDppRowShr + 4>(v);
  v += dpp_i32<kDppRowShr + 8>(v);
  const int row0 = __builtin_amdgcn_readlane(v, 15), row1 = row0 + __builtin_amdgcn_readlane(v, 31), row2 = row1 + __builtin_amdgcn_readlane(v, 47);
  return v + (lane < 16 ? 0 : lane < 32 ? row0 : lane < 48 ? row1 : row2);
}

__device__ __forceinline__ u64 min_u64(u64 a, u64 b) { return a < b ? a : b; }

__device__ __forceinline__ u64 wave_min_u64(u64 v) {
  v = min_u64(v, dpp_u64<kDppQuadSwap1>(v));
  v = min_u64(v, dpp_u64<kDppQuadSwap2>(v));
  v = min_u64(v, dpp_u64<kDppRowHalfMirror>(v));
  v = min_u64(v, dpp_u64<kDppRowMirror>(v));
  return min_u64(min_u64(readlane_u64(v, 0), readlane_u64(v, 16)), min_u64(readlane_u64(v, 32), readlane_u64(v, 48)));
}

// a value that is the same in all lanes, into scalar registers
__device__ __forceinline__ int uniform_i32(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float uniform_f32(float v) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v))); }

template <int kCtrl>
__device__ __forceinline__ float dpp_f32(float v) {
  return __int_as_float(dpp_i32<kCtrl>(__float_as_int(v)));
}

// Stores and loads that are coherent across the chip's L2 caches one by one (no cache-wide write-back or
// invalidation, which a fence at that scope would cost every workgroup): how a scan hands its partials from the
// workgroups that wrote them to the one that combines them.
template <class T>
__device__ __forceinline__ void put_coherent(T* p, T v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <class T>
__device__ __forceinline__ T get_coherent(const T* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// ------------------------------------------------------------------ selection, keys in registers
// Thread tid of NT holds R keys (which ones does not matter): b[i] = the leading word (0xFFFFFFFF: no key), np[i] = the word that orders equal
// ones. In an eviction b is the score's pattern and np = ~position.
struct alignas(16) CutBuf {
  uint32_t hist[3][256];  // digit counts of a round; three in turn, so that one barrier per round is enough
  uint32_t lo[16], hi[16];
  int a[16], b[16];
};

template <int kCtrl>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t v) {
  return (uint32_t)dpp_i32<kCtrl>((int)v);
}
__device__ __forceinline__ uint32_t wave_min_u32(uint32_t v) {
  v = min(v, dpp_u32<kDppQuadSwap1>(v));
  v = min(v, dpp_u32<kDppQuadSwap2>(v));
  v = min(v, dpp_u32<kDppRowHalfMirror>(v));
  v = min(v, dpp_u32<kDppRowMirror>(v));
  const uint32_t x = (uint32_t)__builtin_amdgcn_readlane((int)v, 0), y = (uint32_t)__builtin_amdgcn_readlane((int)v, 16);
  const uint32_t z = (uint32_t)__builtin_amdgcn_readlane((int)v, 32), w = (uint32_t)__builtin_amdgcn_readlane((int)v, 48);
  return min(min(x, y), min(z, w));
}

// The k-th smallest key is (S, P): an entry is among the k smallest (score, then higher position first) if its
// pattern is below S, or equal to S with ~position <= P.
struct KeyCut {
  uint32_t S, P;
  __device__ __forceinline__ bool operator()(uint32_t b, uint32_t np) const { return (b < S) | ((b == S) & (np <= P)); }
};

// Eight bits per round from the highest bit in which the values differ (positions share most of theirs: 14 bits are
// left of 32 for a unit that spans 16384 tokens): a histogram of the digit in LDS over the entries that still
// match the prefix, then every wavefront finds the digit at which the count passes `want` by itself.  Scores that have decayed to
// zero (most of a prompt's) are counted first: their common digit would serialise the LDS atomics of every round.
// 64 units of 9350 entries, 7300 of them evicted, the whole kernel: 21.7 us; with two-bit rounds that count with ballots
// 70 us (16 entries per thread and three compares each make such a round 2.5 us of issue); with two-bit rounds over
// scores in LDS and positions in memory by 256 threads, moves included, 632 us.
template <int R, int NT>
__device__ __forceinline__ KeyCut select_low_keys(const uint32_t (&b)[R], const uint32_t (&np)[R], int k, CutBuf& cb, int tid) {
  const int lane = tid & 63, wave = tid >> 6;
  constexpr int W = NT / 64;
  int turn = 0;
  int zeros = 0;
#pragma unroll
  for (int i = 0; i < R; ++i) zeros += __popcll(__ballot(b[i] == 0u));
  if (lane == 0) cb.a[wave] = zeros;
  for (int i = tid; i < 256; i += NT) cb.hist[0][i] = 0u;
  __syncthreads();
  zeros = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) zeros += cb.a[w];
  // The `want`-th smallest of the values for which `value(i, v)` is true; all of them equal to the result are
  // wanted if all_equal comes back true (the result may then lie above the value itself, below the next larger one).
  auto radix = [&](auto value, int want, bool& all_equal) -> uint32_t {
    uint32_t lo = 0xFFFFFFFFu, nhi = 0xFFFFFFFFu;              // minimum, and ~maximum
#pragma unroll
    for (int i = 0; i < R; ++i) {
      uint32_t v;
      if (value(i, v)) {
        lo = min(lo, v);
        nhi = min(nhi, ~v);
      }
    }
    lo = wave_min_u32(lo);
    nhi = wave_min_u32(nhi);
    if (lane == 0) {
      cb.lo[wave] = lo;
      cb.hi[wave] = nhi;
    }
    __syncthreads();
    lo = cb.lo[0];
    nhi = cb.hi[0];
#pragma unroll
    for (int w = 1; w < W; ++w) {
      lo = min(lo, cb.lo[w]);
      nhi = min(nhi, cb.hi[w]);
    }
    const uint32_t diff = lo ^ ~nhi;
    int top = diff ? 32 - __builtin_clz(diff) : 0;             // the values agree in all bits from `top` on
    uint32_t X = top < 32 ? lo >> top << top : 0u;
    all_equal = false;
    while (top > 0) {
      const int s = max(top - 8, 0);
      const uint32_t digits = 1u << (top - s);
      uint32_t* h = cb.hist[turn];
#pragma unroll
      for (int i = 0; i < R; ++i) {
        uint32_t v;
        if (value(i, v) && (v >> s) - (X >> s) < digits) atomicAdd(&h[(v >> s) - (X >> s)], 1u);      // (X ends in zeros from the digit on)
      }
      turn = turn == 2 ? 0 : turn + 1;
      for (int i = tid; i < 256; i += NT) cb.hist[turn][i] = 0u;       // read last two rounds ago
      __syncthreads();
      const u32x4 q = *reinterpret_cast<const u32x4*>(h + 4 * lane);
      const int mine = (int)(q[0] + q[1] + q[2] + q[3]);
      const int incl = wave_scan_i32(mine, lane);
      const int at = __ffsll((long long)__ballot(incl >= want)) - 1;   // the lane whose four digits hold the wanted one
      int below = __builtin_amdgcn_readlane(incl - mine, at);
      uint32_t digit = 4u * (uint32_t)at;
      int count = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        count = __builtin_amdgcn_readlane((int)q[e], at);
        if (below + count >= want) {
          digit += e;
          break;
        }
        below += count;
      }
      want -= below;
      X |= digit << s;
      top = s;
      if (count == want) {                                     // the whole digit is wanted: no need to look inside
        X |= (1u << s) - 1u;
        all_equal = true;
        break;
      }
    }
    return X;
  };
  KeyCut cut;
  cut.P = 0xFFFFFFFFu;
  bool all_equal = false;
  int want = k;
  if (zeros >= k) {
    cut.S = 0u;
    if (zeros == k) return cut;
  } else {
    want = k - zeros;
    cut.S = radix([&](int i, uint32_t& v) { v = b[i]; return b[i] - 1u < 0xFFFFFFFEu; }, want, all_equal);      // neither zero nor beyond the unit
    if (all_equal) return cut;
    int below = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) below += __popcll(__ballot(b[i] < cut.S));
    if (lane == 0) cb.b[wave] = below;
    __syncthreads();
    want = k;
#pragma unroll
    for (int w = 0; w < W; ++w) want -= cb.b[w];
  }
  // of the entries equal to S the `want` highest positions go (radix() returns at once if that is all of them)
  cut.P = radix([&](int i, uint32_t& v) { v = np[i]; return b[i] == cut.S; }, want, all_equal);
  return cut;
}

}  // namespace ckv
