// Device code that all kernels of the cache in pages share: pools and table, a call's rows, rows in 8 bits.
//
// A row is the 128 values of one key or value.  Pools hold rows one after another in pages, k, v [page][KV head][slot][128] with strides of
// the caller's, as bf16 or as e4m3 codes with one power of two per row, scales [page][KV head][slot][2] (key, value), exponent + 127.  With
// powers of two a code's value is a bf16 number, so that reading back, the products' operands and a page's extremes are all exact;
// and e4m3 loses nothing by them, since its steps are relative.
#pragma once
#include "ckv_lanes.h"
#include "ckv_layout.h"
#include "ckv_paged.h"

namespace ckv {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Pools, table and lengths.  Strides in bytes.
struct Paged {
  uint8_t* k;
  uint8_t* v;
  uint8_t* scales;
  uint8_t* bounds;
  int32_t* status;
  const int32_t* table;
  const int32_t* lengths;
  int64_t page_stride, head_stride, scale_page_stride, scale_head_stride, bounds_page_stride, bounds_head_stride;
  int64_t table_stride;    // in elements
  int32_t slot_stride;
  int32_t n_pages, shift, hkv, batch, columns, max_length;

  __device__ __forceinline__ int page_size() const { return 1 << shift; }
  // a sequence's length, 0 .. max_length whatever the caller's array holds
  __device__ __forceinline__ int length(int b, int& bad) const {
    const int n = lengths[b];
    if (n < 0 || n > max_length) bad |= PAGED_BAD_LENGTH;
    return min(max(n, 0), max_length);
  }
  // page of the pool behind column `c` < columns of a sequence's row, -1 if there is none
  __device__ __forceinline__ int page(int b, int c, int& bad) const {
    const int x = table[(int64_t)b * table_stride + c];
    if (page_there(x, n_pages)) return x;
    bad |= PAGED_BAD_PAGE;
    return -1;
  }
  __device__ __forceinline__ void report(int bad) const {
    if (bad && status) atomicOr(status, bad);
  }
};

__device__ __forceinline__ u32x4 load16(const uint8_t* p) { return *reinterpret_cast<const u32x4*>(p); }
__device__ __forceinline__ u32x2 load8(const uint8_t* p) { return *reinterpret_cast<const u32x2*>(p); }
__device__ __forceinline__ u32x4 stream16(const uint8_t* p) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)); }
__device__ __forceinline__ u32x2 stream8(const uint8_t* p) { return __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p)); }

__device__ __forceinline__ float bf16_low(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float bf16_high(uint32_t x) { return __uint_as_float(x & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t bf16_pack(float a, float b) { return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b}); }
// two codes (the low or the high half of a word) as bf16, times a power of two
template <bool HIGH>
__device__ __forceinline__ uint32_t codes_bf16(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HIGH));
}

// ------------------------------------------------------------------ rows
// Where the call's own rows lie: row i of sequence b, KV head h at base + b * seq_stride (or starts[b] * row_stride) + i * row_stride + h * head_stride.
struct Rows {
  uint8_t* k;
  uint8_t* v;
  const int32_t* first;
  const int32_t* starts;
  int64_t seq_stride, row_stride, head_stride;     // bytes
  int32_t rows, total;

  // rows of sequence b whose length the caller gives as `told`
  __device__ __forceinline__ RowSpan span(int b, int told, int max_length, int64_t& base) const {
    const int start = starts ? starts[b] : 0, stop = starts ? starts[b + 1] : 0;
    base = starts ? start * row_stride : b * seq_stride;
    return span(told, first ? first[b] : 0, start, stop, max_length);
  }
  __device__ __forceinline__ RowSpan span(int told, int first_b, int start, int stop, int max_length) const {
    return rows_below(row_span(told, rows, first != nullptr, first_b, starts != nullptr, start, stop, total), max_length);
  }
};

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pk_max_u16(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
// Largest of the lane's row of 16 lanes.
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
  v = max(v, (uint32_t)dpp_i32<kDppQuadSwap1>((int)v));
  v = max(v, (uint32_t)dpp_i32<kDppQuadSwap2>((int)v));
  v = max(v, (uint32_t)dpp_i32<kDppRowHalfMirror>((int)v));
  return max(v, (uint32_t)dpp_i32<kDppRowMirror>((int)v));
}

__device__ __forceinline__ void unpack8(u32x4 x, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = bf16_low(x[i]);
    f[2 * i + 1] = bf16_high(x[i]);
  }
}

constexpr uint32_t kInfinite = 0x7F80u;       // a bf16's magnitude from which it is not finite
// Largest magnitude (its bits) of a row that 16 lanes hold, 8 values each; with infinities and NaN if there are any.
__device__ __forceinline__ uint32_t magnitude(u32x4 x) {
  constexpr uint32_t kBits = 0x7FFF7FFFu;
  const uint32_t m = pk_max_u16(pk_max_u16(x[0] & kBits, x[1] & kBits), pk_max_u16(x[2] & kBits, x[3] & kBits));
  return row_max(max(m & 0xFFFFu, m >> 16));
}
// The row without what is not finite, as NaN for the codes.
__device__ __forceinline__ u32x4 finite8(u32x4 x, uint32_t instead) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((x[i] & 0x7F80u) == 0x7F80u) x[i] = (x[i] & 0xFFFF0000u) | instead;
    if ((x[i] & 0x7F800000u) == 0x7F800000u) x[i] = (x[i] & 0xFFFFu) | instead << 16;
  }
  return x;
}
// Eight values of a row that 16 lanes hold, to codes and the scale's byte E + 127: E = the smallest integer for which the row's largest finite magnitude is at most
// 448 * 2^E, from -100 to 120 (so that codes times 2^E stay normal bf16 numbers).  448 = 1.75 * 2^8, so E follows from the magnitude's bits: its exponent less 8, one more
// if its mantissa is above 0x60.  x / 2^E is exact, the conversion rounds to nearest, ties to even; what is no number or infinite becomes the format's NaN.
__device__ __forceinline__ u32x2 quantise8(u32x4 x, uint32_t& e) {
  uint32_t m = magnitude(x);
  if (__any(m >= kInfinite)) {
    m = magnitude(finite8(x, 0u));
    x = finite8(x, 0x7FC0u);
  }
  e = (uint32_t)min(max((int)((m + 0x1Fu) >> 7) - 8, 127 - 100), 127 + 120);
  const float scale = __uint_as_float(e << 23);
  u32x2 codes;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const uint32_t a = x[2 * w], z = x[2 * w + 1];       // (a bit cast of a vector's element itself takes the first)
    i16x2 c = {0, 0};
    c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, a), scale, false);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, z), scale, true);
    codes[w] = __builtin_bit_cast(uint32_t, c);
  }
  return codes;
}

__device__ __forceinline__ u32x4 values8(u32x2 codes, float scale) {
  return u32x4{codes_bf16<false>(codes[0], scale), codes_bf16<true>(codes[0], scale), codes_bf16<false>(codes[1], scale), codes_bf16<true>(codes[1], scale)};
}

// Least and largest key of each dimension over rows of one page that a workgroup of NT threads writes, sixteen lanes a row.
template <bool E4M3, int NT>
struct Extremes {
  float lo[8], hi[8];
  __device__ __forceinline__ Extremes() {
#pragma unroll
    for (int i = 0; i < 8; ++i) lo[i] = INFINITY, hi[i] = -INFINITY;
  }
  __device__ __forceinline__ void widen(u32x4 k) {
    float x[8];
    unpack8(k, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) lo[i] = fminf(lo[i], x[i]), hi[i] = fmaxf(hi[i], x[i]);
  }
  // Into the page's bounds, that of rows begin .. end - 1 of column `col` of a sequence of `length`.
  __device__ __forceinline__ void write(const Paged& p, int page, int h, int col, int begin, int end, int length, float (&s_lo)[NT / 64][kDim], float (&s_hi)[NT / 64][kDim],
                                        int tid) {
    const int lane = tid & 63, wave = tid >> 6, piece = lane & 15, group = tid >> 4;
    const bool anew = (begin & (p.page_size() - 1)) == 0;
    if (anew) {                                              // the page's rows behind those written, if the sequence has any
      const int stop = min(length, (col + 1) << p.shift);
      for (int row = end + group; row < stop; row += NT / 16) {
        const int slot = row & (p.page_size() - 1);
        const uint8_t* from = p.k + page * p.page_stride + h * p.head_stride + (int64_t)slot * p.slot_stride;
        if constexpr (E4M3) {
          const uint32_t e = p.scales[page * p.scale_page_stride + h * p.scale_head_stride + 2 * slot];
          widen(values8(load8(from + 8 * piece), __uint_as_float(e << 23)));
        } else {
          widen(load16(from + 16 * piece));
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      lo[i] = rows_combine(lo[i], [](float x, float y) { return fminf(x, y); });
      hi[i] = rows_combine(hi[i], [](float x, float y) { return fmaxf(x, y); });
    }
    if (lane < 16) {
#pragma unroll
      for (int i = 0; i < 8; ++i) s_lo[wave][8 * piece + i] = lo[i], s_hi[wave][8 * piece + i] = hi[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = tid; i < 2 * kDim; i += NT) {             // 0 .. 127 the least values, 128 .. 255 the largest
      const int d = i & (kDim - 1), side = i >> 7;
      const float(*s)[kDim] = side ? s_hi : s_lo;
      uint16_t* to = reinterpret_cast<uint16_t*>(p.bounds + page * p.bounds_page_stride + h * p.bounds_head_stride) + i;
      float x = s[0][d];
#pragma unroll
      for (int w = 1; w < NT / 64; ++w) x = side ? fmaxf(x, s[w][d]) : fminf(x, s[w][d]);
      if (!anew) {                                           // rows that were there before
        const float old = __uint_as_float((uint32_t)*to << 16);
        x = side ? fmaxf(x, old) : fminf(x, old);
      }
      *to = (uint16_t)(__float_as_uint(x) >> 16);            // a bf16 value as it is
    }
  }
};

constexpr float kNoLogit = -3.0e38f;     // where the running maximum starts: a logit of -inf, masked or not, weighs nothing

__device__ __forceinline__ float natural(float m, float l) { return l > 0.f ? (m + __log2f(l)) * 0.69314718055994530942f : l == 0.f ? -INFINITY : NAN; }

}  // namespace ckv
