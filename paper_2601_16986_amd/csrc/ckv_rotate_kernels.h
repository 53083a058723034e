// Device code of rows that enter the cache in pages with their positions' rotation.
#pragma once
#include "ckv_paged_device.h"

namespace ckv {

// Queries of the call's rows, and where they go turned.  Strides in bytes; with Rows::starts rows lie packed.
struct Turned {
  const uint8_t* q;
  uint8_t* out;
  const double* frequencies;     // [pairs]
  const int32_t* positions;      // [batch][rows], or [total] where rows are packed; NULL: positions in the sequence
  int64_t q_seq, q_row, q_head, out_seq, out_row, out_head;
  float magnitude;
  int32_t G, pairs, interleaved;
};

// Sine and cosine of the angle p * f, rounded to float.  A position times a frequency has more digits than a float keeps of a far angle (131072 rad to 2^-7), so it
// is 64 bits that count turns; what is left of them, an eighth at most to either side of the nearest quarter, goes into the Taylor series of both, in 64 bits
// too (as fast as 32 here), up to terms of 2^-33.
__device__ __forceinline__ void sine_cosine(int p, double f, float magnitude, float& sine, float& cosine) {
  const double turns = (double)p * f * 0.15915494309189533577, quarters = rint(turns * 4.0);
  const double x = fma(quarters, -0.25, turns) * 6.28318530717958647693, y = x * x;
  double s = fma(y, fma(y, -1.0 / 39916800, 1.0 / 362880), -1.0 / 5040), c = fma(y, -1.0 / 3628800, 1.0 / 40320);
  s = fma(y, fma(y, fma(y, s, 1.0 / 120), -1.0 / 6), 1.0) * x;
  c = fma(y, fma(y, fma(y, fma(y, c, -1.0 / 720), 1.0 / 24), -0.5), 1.0);
  const int quarter = (int)(quarters - 4.0 * floor(quarters * 0.25));         // 0 .. 3
  const double a = quarter & 1 ? c : s, b = quarter & 1 ? s : c;
  sine = (float)((quarter & 2 ? -a : a) * magnitude);
  cosine = (float)((quarter == 1 || quarter == 2 ? -b : b) * magnitude);
}

// Largest finite magnitude (its bits) of a row that 16 lanes hold, 8 floats each.
__device__ __forceinline__ uint32_t magnitude_finite(const float (&x)[8]) {
  uint32_t m = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = __float_as_uint(x[i]) & 0x7FFFFFFFu;
    m = max(m, b >= 0x7F800000u ? 0u : b);
  }
  return row_max(m);
}
// quantise8 of values in 32 bits: the exponent one more if the mantissa is above 0x600000, one rounding to the code.
__device__ __forceinline__ u32x2 quantise8(const float (&x)[8], uint32_t& e) {
  e = (uint32_t)min(max((int)((magnitude_finite(x) + 0x1FFFFFu) >> 23) - 8, 127 - 100), 127 + 120);
  const float scale = __uint_as_float(e << 23);
  u32x2 codes;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = (__float_as_uint(x[4 * w + i]) & 0x7F800000u) == 0x7F800000u ? NAN : x[4 * w + i];
    i16x2 c = {0, 0};
    c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, y[0], y[1], scale, false);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, y[2], y[3], scale, true);
    codes[w] = __builtin_bit_cast(uint32_t, c);
  }
  return codes;
}

// Eight values of a row that sixteen lanes hold, turned: s and c for each of them, s negative where the value is a pair's first; `turn`: whether the lane's values are in
// pairs at all, with whom it exchanges them at `partner` (none where pairs lie side by side).
struct Turn {
  float s[8], c[8];
  int partner;
  bool turn, exchange;
  __device__ __forceinline__ void operator()(u32x4 x, float (&y)[8]) const {
    float a[8], z[8];
    unpack8(x, a);
    if (exchange) {
      u32x4 other;
#pragma unroll
      for (int i = 0; i < 4; ++i) other[i] = (uint32_t)__builtin_amdgcn_ds_bpermute(partner << 2, (int)x[i]);
      unpack8(other, z);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] = a[i ^ 1];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = turn ? fmaf(a[i], c[i], z[i] * s[i]) : a[i];
  }
};

// One workgroup per (sequence, KV head with its queries) and page that new rows reach, as in paged_append_kernel.  Sixteen lanes take a row: each works out the sines and
// cosines of four pairs and gives them to those who need them, then the row's heads go by, key and value first, kAhead of them on their way at once; where the page gets
// fewer than sixteen rows, sixteen lanes take some of a row's heads.
constexpr int kTurnAhead = 4;
template <bool E4M3>
__global__ __launch_bounds__(kThreads) void paged_append_rotated_kernel(Paged p, Rows r, Turned c) {
  constexpr int kGroups = kThreads / 16;
  __shared__ float s_lo[kThreads / 64][kDim], s_hi[kThreads / 64][kDim];
  const int u = blockIdx.x, b = u / p.hkv, h = u - b * p.hkv;
  const int tid = threadIdx.x, lane = tid & 63, piece = lane & 15, group = tid >> 4;
  int bad = 0;
  const int length = p.length(b, bad);
  int64_t base;
  const RowSpan span = r.span(b, p.lengths[b], p.max_length, base);
  if (span.bad) bad |= PAGED_BAD_LENGTH;
  const int col = (span.first >> p.shift) + blockIdx.y;
  const int begin = max(span.first, col << p.shift), end = (int)min((int64_t)span.first + span.count, ((int64_t)col + 1) << p.shift);
  if (begin >= end || col >= p.columns) {
    if (blockIdx.y == 0 && tid == 0) p.report(bad);
    return;
  }
  const int page = p.page(b, col, bad);
  if (tid == 0) p.report(bad);
  const int64_t at = (int64_t)page * p.page_stride + h * p.head_stride;
  const int64_t start = r.starts ? r.starts[b] : 0;
  const uint8_t* q0 = c.q + (r.starts ? start * c.q_row : b * c.q_seq) + (int64_t)h * c.G * c.q_head + 16 * piece;
  uint8_t* out0 = c.out + (r.starts ? start * c.out_row : b * c.out_seq) + (int64_t)h * c.G * c.out_head + 16 * piece;
  const int32_t* positions = c.positions ? c.positions + (r.starts ? start : (int64_t)b * r.rows) : nullptr;

  double f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = 4 * piece + i < c.pairs ? c.frequencies[4 * piece + i] : 0.0;
  Turn t;
  const int half = c.pairs >> 3;                       // pieces that hold the pairs' first values
  t.exchange = !c.interleaved;
  t.turn = piece < 2 * half;
  t.partner = (lane & 48) + (piece < half ? piece + half : t.turn ? piece - half : piece);
  const int mine = (lane & 48) + (c.interleaved ? piece : 2 * (piece < half ? piece : t.turn ? piece - half : 0));      // the lane with the first four pairs of this one's

  int parts = 1;                                       // of a row's heads
  while (parts < kGroups && 2 * parts * (end - begin) <= kGroups) parts *= 2;
  const int part = group & (parts - 1), heads = c.G + 1;        // the key and value, then the queries
  Extremes<E4M3, kThreads> extremes;
  const int rows_each = kGroups / parts;
  for (int row0 = begin; row0 < end; row0 += rows_each) {
    const int row = min(row0 + group / parts, end - 1);
    const bool there = row0 + group / parts < end;
    const int i = row - span.first, slot = row & (p.page_size() - 1), position = positions ? positions[i] : row;
    float sine[4], cosine[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) sine_cosine(position, f[k], c.magnitude, sine[k], cosine[k]);
    if (c.interleaved) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        t.c[k] = cosine[k >> 1];
        t.s[k] = k & 1 ? sine[k >> 1] : -sine[k >> 1];
      }
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        t.c[k] = __int_as_float(__builtin_amdgcn_ds_bpermute((mine + (k >> 2)) << 2, __float_as_int(cosine[k & 3])));
        const float s = __int_as_float(__builtin_amdgcn_ds_bpermute((mine + (k >> 2)) << 2, __float_as_int(sine[k & 3])));
        t.s[k] = piece < half ? -s : s;
      }
    }
    for (int first = part; first < heads; first += parts * kTurnAhead) {
      u32x4 x[kTurnAhead], v = {0u, 0u, 0u, 0u};
#pragma unroll
      for (int n = 0; n < kTurnAhead; ++n) {
        const int head = first + n * parts;
        if (head == 0) {
          const int64_t from = base + (int64_t)i * r.row_stride + h * r.head_stride + 16 * piece;
          x[n] = load16(r.k + from);
          v = load16(r.v + from);
        } else if (head < heads) {
          x[n] = load16(q0 + i * c.q_row + (head - 1) * c.q_head);
        } else {
          x[n] = u32x4{0u, 0u, 0u, 0u};
        }
      }
#pragma unroll
      for (int n = 0; n < kTurnAhead; ++n) {
        const int head = first + n * parts;
        float y[8];
        t(x[n], y);
        const u32x4 packed = {bf16_pack(y[0], y[1]), bf16_pack(y[2], y[3]), bf16_pack(y[4], y[5]), bf16_pack(y[6], y[7])};
        if (head > 0) {
          if (head < heads && there) *reinterpret_cast<u32x4*>(out0 + i * c.out_row + (head - 1) * c.out_head) = packed;
        } else if (n == 0 && page >= 0 && there) {
          u32x4 k = packed;
          if constexpr (E4M3) {
            uint32_t ek, ev;
            const u32x2 ck = quantise8(y, ek), cv = quantise8(v, ev);
            const int64_t to = at + (int64_t)slot * p.slot_stride + 8 * piece;
            *reinterpret_cast<u32x2*>(p.k + to) = ck;
            *reinterpret_cast<u32x2*>(p.v + to) = cv;
            if (piece == 0)
              *reinterpret_cast<uint16_t*>(p.scales + page * p.scale_page_stride + h * p.scale_head_stride + 2 * slot) = (uint16_t)(ek | ev << 8);
            k = values8(ck, __uint_as_float(ek << 23));
          } else {
            const int64_t to = at + (int64_t)slot * p.slot_stride + 16 * piece;
            *reinterpret_cast<u32x4*>(p.k + to) = k;
            *reinterpret_cast<u32x4*>(p.v + to) = v;
          }
          if (p.bounds) extremes.widen(k);
        }
      }
    }
  }
  if (p.bounds && page >= 0) extremes.write(p, page, h, col, begin, end, length, s_lo, s_hi, tid);
}

}  // namespace ckv
