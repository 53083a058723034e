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

// Sine and cosine of the angle p * f, times the magnitude.  A position times a frequency has more digits than a float keeps of a far angle (131072 rad to 2^-7), so it
// is 64 bits that count turns; what is left of them, an eighth at most to either side of the nearest quarter, goes into the Taylor series of both, in 64 bits
// too (as fast as 32 here), up to terms of 2^-33.
__device__ __forceinline__ void sine_cosine(int p, double f, float magnitude, double& sine, double& cosine) {
  const double turns = (double)p * f * 0.15915494309189533577, quarters = rint(turns * 4.0);
  const double x = fma(quarters, -0.25, turns) * 6.28318530717958647693, y = x * x;
  double s = fma(y, fma(y, -1.0 / 39916800, 1.0 / 362880), -1.0 / 5040), c = fma(y, -1.0 / 3628800, 1.0 / 40320);
  s = fma(y, fma(y, fma(y, s, 1.0 / 120), -1.0 / 6), 1.0) * x;
  c = fma(y, fma(y, fma(y, fma(y, c, -1.0 / 720), 1.0 / 24), -0.5), 1.0);
  const int quarter = (int)(quarters - 4.0 * floor(quarters * 0.25));         // 0 .. 3
  const double a = quarter & 1 ? c : s, b = quarter & 1 ? s : c;
  sine = (quarter & 2 ? -a : a) * magnitude;
  cosine = (quarter == 1 || quarter == 2 ? -b : b) * magnitude;
}

// A value in 64 bits to 32 with the rest remembered in the lowest bit (towards zero, and odd where that is not exact), so that rounding it to fewer bits is one rounding.
__device__ __forceinline__ float to_odd(double y) {
  const float f = (float)y;
  uint32_t b = __float_as_uint(f);
  if (fabs((double)f) > fabs(y)) --b;
  return fabsf(f) < INFINITY ? __uint_as_float((double)f != y ? b | 1u : b) : f;
}

__device__ __forceinline__ float of_lane(float v, int lane) { return __int_as_float(__builtin_amdgcn_ds_bpermute(lane << 2, __float_as_int(v))); }
__device__ __forceinline__ double of_lane(double v, int lane) {
  const long long x = __double_as_longlong(v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_ds_bpermute(lane << 2, (int)(uint32_t)x), hi = (uint32_t)__builtin_amdgcn_ds_bpermute(lane << 2, (int)(uint32_t)(x >> 32));
  return __longlong_as_double((long long)((u64)hi << 32 | lo));
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

// How sixteen lanes turn a row, eight values each: with whom a lane exchanges them (nobody where pairs lie side by side), which lane worked out the first four pairs of its
// eight (or four), whether its values are a pair's first ones, and whether they are in pairs at all.
struct Pairing {
  int partner, from;
  bool exchange, first, turn;
  __device__ __forceinline__ Pairing(int lane, int pairs, bool interleaved) {
    const int piece = lane & 15, row = lane & 48, half = pairs >> 3;
    exchange = !interleaved;
    first = piece < half;
    turn = piece < 2 * half;
    const int other = first ? piece + half : turn ? piece - half : piece;
    partner = row + other;
    from = row + (interleaved ? piece : turn ? 2 * min(piece, other) : 0);
  }
  // of four pairs per lane the sine and cosine of its value k, a pair's first value with the sine's other sign
  template <class T>
  __device__ __forceinline__ void spread(const double (&sine)[4], const double (&cosine)[4], int k, T& s, T& c) const {
    if (exchange) {
      s = of_lane((T)sine[k & 3], from + (k >> 2));
      c = of_lane((T)cosine[k & 3], from + (k >> 2));
      if (first) s = -s;
    } else {
      s = (T)(k & 1 ? sine[k >> 1] : -sine[k >> 1]);
      c = (T)cosine[k >> 1];
    }
  }
  __device__ __forceinline__ void values(u32x4 x, float (&a)[8], float (&z)[8]) const {
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
  }
  __device__ __forceinline__ u32x4 bf16(u32x4 x, const float (&s)[8], const float (&c)[8]) const {
    float a[8], z[8], y[8];
    values(x, a, z);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = turn ? fmaf(a[i], c[i], z[i] * s[i]) : a[i];
    return u32x4{bf16_pack(y[0], y[1]), bf16_pack(y[2], y[3]), bf16_pack(y[4], y[5]), bf16_pack(y[6], y[7])};
  }
  // Keys in 8 bits stay in 64 until they are rounded: a bf16 number is half way between two codes often enough (one in thirty-two), and slow pairs turn it by less than a
  // float's last bit.
  __device__ __forceinline__ u32x2 codes(u32x4 x, const double (&sine)[4], const double (&cosine)[4], uint32_t& e) const {
    float a[8], z[8], y[8];
    values(x, a, z);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      double s, c;
      spread(sine, cosine, i, s, c);
      y[i] = turn ? to_odd(fma((double)a[i], c, (double)z[i] * s)) : a[i];
    }
    return quantise8(y, e);
  }
};

// One workgroup per (sequence, KV head with its queries) and page that new rows reach, as in paged_append_kernel.  Sixteen lanes take a row: each works out the sines and
// cosines of four pairs and gives them to those who need them, then the row's heads go by, key and value first, kTurnAhead of them on their way at once; where the page gets
// fewer than sixteen rows, sixteen lanes take some of a row's heads.  Where pages are few, more workgroups (blockIdx.z) share a page's heads, the first of them keys and values too
// (SHARED, turned_by; 64 rows of 4 sequences with 8 heads for each of 4 KV heads: 13.3 us by one, 9.4 by eight).
// What bounds it: prompts of 8 sequences of up to 9350, 40 heads of queries, memory (1074 MB in 260 us, 4.1 TB/s; a plain copy 4.7), as long as four wavefronts per SIMD fit: with 1, 2, 3, 4 or 8 heads on their
// way (108, 115, 125, 134, 170 registers) 299, 260, 259, 277 and 328 us.  A row of each of 32 sequences, 7.2 us, by what comes one after another: lengths, table, rows, sines and cosines, codes, bounds.
constexpr int kTurnAhead = 2;
template <bool E4M3, bool SHARED>
__global__ __launch_bounds__(kThreads) void paged_append_rotated_kernel(Paged p, Rows r, Turned c) {
  const int z = SHARED ? blockIdx.z : 0;
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
    if (blockIdx.y == 0 && z == 0 && tid == 0) p.report(bad);
    return;
  }
  const int page = p.page(b, col, bad);
  if (z == 0 && tid == 0) p.report(bad);
  const int64_t at = (int64_t)page * p.page_stride + h * p.head_stride;
  const int64_t start = r.starts ? r.starts[b] : 0;
  const uint8_t* q0 = c.q + (r.starts ? start * c.q_row : b * c.q_seq) + (int64_t)h * c.G * c.q_head + 16 * piece;
  uint8_t* out0 = c.out + (r.starts ? start * c.out_row : b * c.out_seq) + (int64_t)h * c.G * c.out_head + 16 * piece;
  const int32_t* positions = c.positions ? c.positions + (r.starts ? start : (int64_t)b * r.rows) : nullptr;

  double f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = 4 * piece + i < c.pairs ? c.frequencies[4 * piece + i] : 0.0;
  const Pairing t(lane, c.pairs, c.interleaved);

  int parts = 1;                                       // of a row's heads
  while (parts < kGroups && 2 * parts * (end - begin) <= kGroups) parts *= 2;
  const int part = group & (parts - 1), heads = c.G + 1, rows_each = kGroups / parts;       // the key and value, then the queries
  const int first_head = part + parts * z, every = SHARED ? parts * gridDim.z : parts;
  Extremes<E4M3, kThreads> extremes;
  for (int row = begin + group / parts; row < end; row += rows_each) {
    const int i = row - span.first, slot = row & (p.page_size() - 1), position = positions ? positions[i] : row;
    u32x4 x[kTurnAhead], v = {0u, 0u, 0u, 0u};
    auto ask = [&](int first) {
#pragma unroll
      for (int n = 0; n < kTurnAhead; ++n) {
        const int head = first + n * every;
        if (head > 0 && head < heads) x[n] = load16(q0 + i * c.q_row + (head - 1) * c.q_head);
      }
    };
    if (first_head == 0) {
      const int64_t from = base + (int64_t)i * r.row_stride + h * r.head_stride + 16 * piece;
      x[0] = load16(r.k + from);
      v = load16(r.v + from);
    }
    ask(first_head);
    double sine[4], cosine[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) sine_cosine(position, f[k], c.magnitude, sine[k], cosine[k]);
    float fs[8], fc[8];
    auto floats = [&]() {
#pragma unroll
      for (int k = 0; k < 8; ++k) t.spread(sine, cosine, k, fs[k], fc[k]);
    };
    if constexpr (!E4M3) floats();
    if (first_head == 0 && page >= 0) {
      u32x4 k;
      if constexpr (E4M3) {
        uint32_t ek, ev;
        const u32x2 ck = t.codes(x[0], sine, cosine, ek), cv = quantise8(v, ev);
        const int64_t to = at + (int64_t)slot * p.slot_stride + 8 * piece;
        *reinterpret_cast<u32x2*>(p.k + to) = ck;
        *reinterpret_cast<u32x2*>(p.v + to) = cv;
        if (piece == 0)
          *reinterpret_cast<uint16_t*>(p.scales + page * p.scale_page_stride + h * p.scale_head_stride + 2 * slot) = (uint16_t)(ek | ev << 8);
        k = values8(ck, __uint_as_float(ek << 23));
      } else {
        k = t.bf16(x[0], fs, fc);
        const int64_t to = at + (int64_t)slot * p.slot_stride + 16 * piece;
        *reinterpret_cast<u32x4*>(p.k + to) = k;
        *reinterpret_cast<u32x4*>(p.v + to) = v;
      }
      if (p.bounds) extremes.widen(k);
    }
    if constexpr (E4M3) floats();
    for (int first = first_head; first < heads; first += every * kTurnAhead) {
      if (first != first_head) ask(first);
#pragma unroll
      for (int n = 0; n < kTurnAhead; ++n) {
        const int head = first + n * every;
        if (head == 0 || head >= heads) continue;
        *reinterpret_cast<u32x4*>(out0 + i * c.out_row + (head - 1) * c.out_head) = t.bf16(x[n], fs, fc);
      }
    }
  }
  if (p.bounds && page >= 0 && z == 0) extremes.write(p, page, h, col, begin, end, length, s_lo, s_hi, tid);
}

}  // namespace ckv
