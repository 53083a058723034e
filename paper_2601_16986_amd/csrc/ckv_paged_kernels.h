// Device code of the cache in pages: rows in (quantised as they are written) and out, attention of one new token per sequence
// over its pages or over pages picked for it, and the picking.
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

  __device__ __forceinline__ RowSpan span(int b, int length, int64_t& base) const {
    const int start = starts ? starts[b] : 0, stop = starts ? starts[b + 1] : 0;
    base = starts ? start * row_stride : b * seq_stride;
    return row_span(length, rows, first != nullptr, first ? first[b] : 0, starts != nullptr, start, stop, total);
  }
};

// Largest of the lane's row of 16 lanes.
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, __int_as_float(dpp_i32<kDppQuadSwap1>(__float_as_int(v))));
  v = fmaxf(v, __int_as_float(dpp_i32<kDppQuadSwap2>(__float_as_int(v))));
  v = fmaxf(v, __int_as_float(dpp_i32<kDppRowHalfMirror>(__float_as_int(v))));
  return fmaxf(v, __int_as_float(dpp_i32<kDppRowMirror>(__float_as_int(v))));
}

// Eight values of a row that 16 lanes hold, to codes: E = the smallest integer for which the row's largest finite magnitude is at most
// 448 * 2^E, from -100 to 120 (so that codes times 2^E stay normal bf16 numbers).  448 = 1.75 * 2^8, so E follows from the magnitude's exponent and its first two bits of
// mantissa.  x * 2^-E is exact, the conversion rounds to nearest, ties to even; what is no number or infinite becomes the format's NaN.
__device__ __forceinline__ u32x2 quantise8(const float (&x)[8], int& e) {
  float big = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = fabsf(x[i]);
    big = fmaxf(big, a < INFINITY ? a : 0.f);
  }
  const uint32_t bits = __float_as_uint(row_max(big));
  e = min(max((int)(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u), -100), 120);
  const float inverse = __uint_as_float((uint32_t)(127 - e) << 23);
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = fabsf(x[i]) < INFINITY ? x[i] * inverse : NAN;
  u32x2 codes;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w], y[4 * w + 1], 0, false);
    codes[w] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w + 2], y[4 * w + 3], c, true);
  }
  return codes;
}

__device__ __forceinline__ void unpack8(u32x4 x, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = bf16_low(x[i]);
    f[2 * i + 1] = bf16_high(x[i]);
  }
}
__device__ __forceinline__ u32x4 values8(u32x2 codes, float scale) {
  return u32x4{codes_bf16<false>(codes[0], scale), codes_bf16<true>(codes[0], scale), codes_bf16<false>(codes[1], scale), codes_bf16<true>(codes[1], scale)};
}

// One workgroup per (sequence, KV head) and page that new rows reach: it alone touches the page's rows and extremes, so that these need no atomics.  Sixteen
// lanes take a row, 16 bytes of bf16 each, for key and value.
template <bool E4M3>
__global__ __launch_bounds__(kThreads) void paged_append_kernel(Paged p, Rows r) {
  __shared__ float s_lo[kThreads / 64][kDim], s_hi[kThreads / 64][kDim];
  const int u = blockIdx.x, b = u / p.hkv, h = u - b * p.hkv;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, piece = lane & 15, group = tid >> 4;
  int bad = 0;
  const int length = p.length(b, bad);
  int64_t base;
  const RowSpan span = r.span(b, length, base);
  if (span.bad) bad |= PAGED_BAD_LENGTH;
  const int col = (span.first >> p.shift) + blockIdx.y;
  const int begin = max(span.first, col << p.shift), end = (int)min((int64_t)span.first + span.count, ((int64_t)col + 1) << p.shift);
  if (begin >= end || col >= p.columns) {
    if (blockIdx.y == 0 && tid == 0) p.report(bad);
    return;
  }
  const int page = p.page(b, col, bad);
  if (tid == 0) p.report(bad);
  if (page < 0) return;
  const int64_t at = page * p.page_stride + h * p.head_stride;
  float lo[8], hi[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) lo[i] = INFINITY, hi[i] = -INFINITY;
  for (int row = begin + group; row < end; row += kThreads / 16) {
    const int64_t from = base + (int64_t)(row - span.first) * r.row_stride + h * r.head_stride + 16 * piece;
    const int slot = row & (p.page_size() - 1);
    u32x4 k = load16(r.k + from), v = load16(r.v + from);
    if constexpr (E4M3) {
      float x[8];
      int ek, ev;
      unpack8(k, x);
      const u32x2 ck = quantise8(x, ek);
      unpack8(v, x);
      const u32x2 cv = quantise8(x, ev);
      const int64_t to = at + (int64_t)slot * p.slot_stride + 8 * piece;
      *reinterpret_cast<u32x2*>(p.k + to) = ck;
      *reinterpret_cast<u32x2*>(p.v + to) = cv;
      if (piece == 0)
        *reinterpret_cast<uint16_t*>(p.scales + page * p.scale_page_stride + h * p.scale_head_stride + 2 * slot) = (uint16_t)((ek + 127) | (ev + 127) << 8);
      k = values8(ck, __uint_as_float((uint32_t)(ek + 127) << 23));
    } else {
      const int64_t to = at + (int64_t)slot * p.slot_stride + 16 * piece;
      *reinterpret_cast<u32x4*>(p.k + to) = k;
      *reinterpret_cast<u32x4*>(p.v + to) = v;
    }
    float x[8];
    unpack8(k, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) lo[i] = fminf(lo[i], x[i]), hi[i] = fmaxf(hi[i], x[i]);
  }
  if (!p.bounds) return;
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
  if (tid >= 2 * kDim) return;
  const int d = tid & (kDim - 1), side = tid >> 7;       // threads 0 .. 127 the least values, 128 .. 255 the largest
  const float(*s)[kDim] = side ? s_hi : s_lo;
  uint16_t* to = reinterpret_cast<uint16_t*>(p.bounds + page * p.bounds_page_stride + h * p.bounds_head_stride) + tid;
  float x = s[0][d];
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) x = side ? fmaxf(x, s[w][d]) : fminf(x, s[w][d]);
  if (begin & (p.page_size() - 1)) {                       // rows that were there before
    const float old = __uint_as_float((uint32_t)*to << 16);
    x = side ? fmaxf(x, old) : fminf(x, old);
  }
  *to = (uint16_t)(__float_as_uint(x) >> 16);              // a bf16 value as it is
}

// Sixteen lanes take a row, 64 rows per workgroup.
constexpr int kReadRows = 64;
template <bool E4M3>
__global__ __launch_bounds__(kThreads) void paged_read_kernel(Paged p, Rows r) {
  const int u = blockIdx.x, b = u / p.hkv, h = u - b * p.hkv, piece = threadIdx.x & 15, group = threadIdx.x >> 4;
  int bad = 0;
  const int length = p.length(b, bad);
  int64_t base;
  const RowSpan span = r.span(b, length, base);
  if (span.bad) bad |= PAGED_BAD_LENGTH;
#pragma unroll
  for (int n = 0; n < kReadRows / 16; ++n) {
    const int i = blockIdx.y * kReadRows + 16 * n + group;
    if (i >= span.count) break;
    const int row = span.first + i, slot = row & (p.page_size() - 1);
    const int page = p.page(b, row >> p.shift, bad);
    if (page < 0) continue;
    const int64_t from = page * p.page_stride + h * p.head_stride + (int64_t)slot * p.slot_stride;
    const int64_t to = base + (int64_t)i * r.row_stride + h * r.head_stride + 16 * piece;
    if constexpr (E4M3) {
      const uint32_t s = *reinterpret_cast<const uint16_t*>(p.scales + page * p.scale_page_stride + h * p.scale_head_stride + 2 * slot);
      const u32x2 k = load8(p.k + from + 8 * piece), v = load8(p.v + from + 8 * piece);
      *reinterpret_cast<u32x4*>(r.k + to) = values8(k, __uint_as_float((s & 0xFF) << 23));
      *reinterpret_cast<u32x4*>(r.v + to) = values8(v, __uint_as_float((s >> 8) << 23));
    } else {
      *reinterpret_cast<u32x4*>(r.k + to) = load16(p.k + from + 16 * piece);
      *reinterpret_cast<u32x4*>(r.v + to) = load16(p.v + from + 16 * piece);
    }
  }
  if (piece == 0) p.report(bad);
}

// ------------------------------------------------------------------ attention of one token
struct Attend {
  const uint8_t* q;          // bf16
  const int32_t* picked;     // [batch][hkv][n_picked] pages of the sequence (-1: none), or NULL
  uint8_t* out;
  float* lse;
  float* partial;            // [unit][pieces][G][128]
  float* ml;                 // [unit][pieces][G][2]
  int64_t q_seq_stride, q_head_stride;     // bytes
  float scale_log2e;
  int32_t G, n_picked, piece, pieces, out_bf16;
};

constexpr float kNoLogit = -3.0e38f;     // where the running maximum starts: a logit of -inf, masked or not, weighs nothing

// Two rows of a pair of entries into pairs of one dimension: word w of the result holds dimension w of both.
__device__ __forceinline__ void interleave_bytes(uint32_t a, uint32_t b, uint32_t (&x)[2]) {
  x[0] = __builtin_amdgcn_perm(b, a, 0x05010400u);
  x[1] = __builtin_amdgcn_perm(b, a, 0x07030602u);
}

__device__ __forceinline__ void put_out(const Attend& c, int64_t row, int d4, f32x4 y) {
  if (c.out_bf16) *reinterpret_cast<u32x2*>(c.out + (row * kDim + d4) * 2) = u32x2{bf16_pack(y[0], y[1]), bf16_pack(y[2], y[3])};
  else *reinterpret_cast<f32x4*>(c.out + (row * kDim + d4) * 4) = y;
}
__device__ __forceinline__ float natural(float m, float l) { return l > 0.f ? (m + __log2f(l)) * 0.69314718055994530942f : l == 0.f ? -INFINITY : NAN; }

// One workgroup of four wavefronts per (sequence, KV head) and `piece` entries; wavefronts take blocks of 32 entries in turn.  With the rows as
// they lie a lane (j = lane % 16, kg = lane / 16) reads of a block, per tile of 16 entries,
//   keys    entry j, 16 bytes at 16 kg of each 64: operands of K Q^T (rows = entries) whose order of dimensions the queries share;
//   values  entries 4 kg .. 4 kg + 3, the eighth of the row at j: byte (or word) moves between pairs of entries make them operands of P V (columns =
//           dimensions 8 j + dt), in the entry order in which K Q^T leaves the logits.
// The weights are split into bf16 terms: high ones in rows 0 .. 7 and low ones in rows 8 .. 15 of one operand for up to eight heads (the queries are
// there twice), as operands of their own for more (WIDE).  Two terms hold 16 bits of a weight; a float output gets a third.
template <bool E4M3, int TERMS, bool WIDE>
__global__ __launch_bounds__(kThreads) void paged_attend_kernel(Paged p, Attend c) {
  constexpr int kHeads = WIDE ? 16 : 8, kWaves = kThreads / 64, kRow = kDim + 4;
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  __shared__ __align__(16) float s_acc[kWaves][kHeads * kRow];
  const int u = blockIdx.x, part = blockIdx.y, b = u / p.hkv, h = u - b * p.hkv;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform_i32(tid >> 6), j = lane & 15, kg = lane >> 4;
  int bad = 0;
  const int length = p.length(b, bad), shift = p.shift;
  const int total = c.picked ? c.n_picked << shift : length, e0 = part * c.piece;
  if (e0 >= total && part > 0) return;
  const int blocks = (min(total - e0, c.piece) + 31) >> 5;

  // ---- where the piece's pages lie and how far they are filled, a lane each
  const int slot0 = e0 >> shift;
  int page = 0, fill = 0;
  {
    int logical = slot0 + lane;
    if (c.picked) logical = logical < c.n_picked ? c.picked[(int64_t)u * c.n_picked + logical] : -1;
    if (logical < -1 || (logical >= 0 && (logical >= p.columns || page_fill(length, logical, shift) == 0))) {
      if (c.picked) bad |= PAGED_BAD_PICK;
      logical = -1;
    }
    if (logical >= 0) {
      fill = page_fill(length, logical, shift);
      page = p.page(b, logical, bad);
      if (page < 0) page = fill = 0;
    }
    if (__any(bad)) p.report(bad);
  }

  bf16x8 q[4];
  {
    const int head = WIDE ? j : j & 7;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int d = E4M3 ? 64 * (s >> 1) + 16 * kg + 8 * (s & 1) : 32 * s + 8 * kg;
      u32x4 x = {0u, 0u, 0u, 0u};
      if (head < c.G) x = load16(c.q + b * c.q_seq_stride + (h * c.G + head) * c.q_head_stride + 2 * d);
      q[s] = __builtin_bit_cast(bf16x8, x);
    }
  }
  f32x4 acc[8];
#pragma unroll
  for (int dt = 0; dt < 8; ++dt) acc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = kNoLogit, l_run = 0.f;

  for (int blk = wave; blk < blocks; blk += kWaves) {
    int valid[2];
    float sv[8], vs[8];
    u32x4 kf[2][E4M3 ? 2 : 4], vf[2][4];
    u32x2 sc[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int e = e0 + 32 * blk + 16 * t, off = e & ((1 << shift) - 1), at = (e >> shift) - slot0;
      valid[t] = min(max(__builtin_amdgcn_readlane(fill, at) - off, 0), 16);
      const int64_t pg = __builtin_amdgcn_readlane(page, at);
      const int64_t base = pg * p.page_stride + h * p.head_stride + (int64_t)off * p.slot_stride;
      const uint8_t* kb = p.k + base + j * p.slot_stride + 16 * kg;
#pragma unroll
      for (int s = 0; s < (E4M3 ? 2 : 4); ++s) kf[t][s] = stream16(kb + 64 * s);
      const uint8_t* vb = p.v + base + 4 * kg * p.slot_stride;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (E4M3) {
          const u32x2 x = stream8(vb + i * p.slot_stride + 8 * j);
          vf[t][i] = u32x4{x[0], x[1], 0u, 0u};
        } else {
          vf[t][i] = stream16(vb + i * p.slot_stride + 16 * j);
        }
      }
      if constexpr (E4M3) sc[t] = stream8(p.scales + pg * p.scale_page_stride + h * p.scale_head_stride + 2 * off + 8 * kg);
    }
    // ---- logits of four entries of each tile
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        u32x4 x;
        if constexpr (E4M3) {
          const uint32_t lo = kf[t][n >> 1][2 * (n & 1)], hi = kf[t][n >> 1][2 * (n & 1) + 1];
          x = u32x4{codes_bf16<false>(lo, 1.f), codes_bf16<true>(lo, 1.f), codes_bf16<false>(hi, 1.f), codes_bf16<true>(hi, 1.f)};
        } else {
          x = kf[t][n];
        }
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), q[n], s, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float k_scale = c.scale_log2e;
        vs[4 * t + i] = 1.f;
        if constexpr (E4M3) {
          const uint32_t x = sc[t][i >> 1];
          k_scale *= __uint_as_float(i & 1 ? (x & 0xFF0000u) << 7 : (x & 0xFFu) << 23);
          vs[4 * t + i] = __uint_as_float(i & 1 ? (x & 0xFF000000u) >> 1 : (x & 0xFF00u) << 15);
        }
        sv[4 * t + i] = s[i] * k_scale;
      }
    }
    // ---- entries that are not there: logits of -inf, values and their scales of nothing (the rows may hold anything)
    if (valid[0] + valid[1] < 32) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (4 * kg + i >= valid[t]) {
            sv[4 * t + i] = -INFINITY;
            vs[4 * t + i] = 0.f;
            vf[t][i] = u32x4{0u, 0u, 0u, 0u};
          }
    }
    // ---- softmax with a running maximum
    float bm = fmaxf(fmaxf(fmaxf(sv[0], sv[1]), fmaxf(sv[2], sv[3])), fmaxf(fmaxf(sv[4], sv[5]), fmaxf(sv[6], sv[7])));
    bm = rows_combine(bm, [](float x, float y) { return fmaxf(x, y); });
    if (__any(bm > m_run)) {
      const float m_new = fmaxf(m_run, bm), shrink = fast_exp2(m_run - m_new);
      l_run *= shrink;
      m_run = m_new;
      float f[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = __shfl(shrink, 4 * kg + i);
#pragma unroll
      for (int dt = 0; dt < 8; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[dt][i] *= f[i];
    }
    bf16x8 w[3];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float weight = fast_exp2(sv[i] - m_run);
      l_run += weight;
      float rest = E4M3 ? weight * vs[i] : weight;
#pragma unroll
      for (int n = 0; n < TERMS; ++n) {
        w[n][i] = (__bf16)rest;
        rest -= (float)w[n][i];
      }
    }
    if constexpr (!WIDE) {
      const bool low = j >= 8;
      const u32x4 a = __builtin_bit_cast(u32x4, w[0]), z = __builtin_bit_cast(u32x4, w[1]);
      w[0] = __builtin_bit_cast(bf16x8, u32x4{low ? z[0] : a[0], low ? z[1] : a[1], low ? z[2] : a[2], low ? z[3] : a[3]});
      if constexpr (TERMS == 3) {
        const u32x4 y = __builtin_bit_cast(u32x4, w[2]);
        w[1] = __builtin_bit_cast(bf16x8, u32x4{low ? 0u : y[0], low ? 0u : y[1], low ? 0u : y[2], low ? 0u : y[3]});
      }
    }
    // ---- weights times values: dimension 8 j + dt
#pragma unroll
    for (int d2 = 0; d2 < 4; ++d2) {
      u32x4 x[2];                                      // dimensions 2 d2 and 2 d2 + 1, pairs of entries
#pragma unroll
      for (int pair = 0; pair < 4; ++pair) {
        const u32x4 a = vf[pair >> 1][2 * (pair & 1)], z = vf[pair >> 1][2 * (pair & 1) + 1];
        if constexpr (E4M3) {
          uint32_t y[2];
          interleave_bytes(a[d2 >> 1], z[d2 >> 1], y);
          x[0][pair] = codes_bf16<false>(y[d2 & 1], 1.f);
          x[1][pair] = codes_bf16<true>(y[d2 & 1], 1.f);
        } else {
          x[0][pair] = __builtin_amdgcn_perm(z[d2], a[d2], 0x05040100u);
          x[1][pair] = __builtin_amdgcn_perm(z[d2], a[d2], 0x07060302u);
        }
      }
#pragma unroll
      for (int n = 0; n < (WIDE ? TERMS : TERMS - 1); ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          acc[2 * d2 + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[n], __builtin_bit_cast(bf16x8, x[i]), acc[2 * d2 + i], 0, 0, 0);
    }
  }

  // ---- the wavefronts' states into one
  l_run = rows_combine(l_run, [](float x, float y) { return x + y; });
  if (lane < 16) {
    s_m[wave][lane] = m_run;
    s_l[wave][lane] = l_run;
  }
  if constexpr (!WIDE) {
#pragma unroll
    for (int dt = 0; dt < 8; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[dt][i] += __shfl_xor(acc[dt][i], 32);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int head = 4 * kg + i;
    if (head < kHeads) {
      *reinterpret_cast<f32x4*>(&s_acc[wave][head * kRow + 8 * j]) = f32x4{acc[0][i], acc[1][i], acc[2][i], acc[3][i]};
      *reinterpret_cast<f32x4*>(&s_acc[wave][head * kRow + 8 * j + 4]) = f32x4{acc[4][i], acc[5][i], acc[6][i], acc[7][i]};
    }
  }
  __syncthreads();
  for (int x = tid; x < c.G * (kDim / 4); x += kThreads) {
    const int head = x >> 5, d4 = 4 * (x & 31);
    float M = s_m[0][head], L = 0.f;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) M = fmaxf(M, s_m[w][head]);
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = fast_exp2(s_m[w][head] - M);
      L += s_l[w][head] * f;
      y += *reinterpret_cast<const f32x4*>(&s_acc[w][head * kRow + d4]) * f;
    }
    if (c.pieces > 1) {
      const int64_t at = ((int64_t)u * c.pieces + part) * c.G + head;
      *reinterpret_cast<f32x4*>(c.partial + at * kDim + d4) = y;
      if (d4 == 0) {
        c.ml[2 * at] = M;
        c.ml[2 * at + 1] = L;
      }
    } else {
      const int64_t row = (int64_t)u * c.G + head;
      put_out(c, row, d4, L != 0.f ? y * (1.f / L) : f32x4{0.f, 0.f, 0.f, 0.f});
      if (d4 == 0 && c.lse) c.lse[row] = natural(M, L);
    }
  }
}

// Joins the pieces of one (sequence, query head): eight rows of 32 threads take pieces in turn, a thread four dimensions.
__global__ __launch_bounds__(kThreads) void paged_join_kernel(Paged p, Attend c) {
  __shared__ float s_m[8], s_l[8];
  __shared__ __align__(16) float s_y[8][kDim];
  const int u = blockIdx.x, head = blockIdx.y, b = u / p.hkv, group = threadIdx.x >> 5, d4 = 4 * (threadIdx.x & 31);
  int bad = 0;
  const int length = p.length(b, bad), total = c.picked ? c.n_picked << p.shift : length;
  const int pieces = min(c.pieces, (total + c.piece - 1) / c.piece);
  float m = kNoLogit, l = 0.f;
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
  for (int i = group; i < pieces; i += 8) {
    const int64_t at = ((int64_t)u * c.pieces + i) * c.G + head;
    const f32x4 x = *reinterpret_cast<const f32x4*>(c.partial + at * kDim + d4);
    const float mi = c.ml[2 * at], li = c.ml[2 * at + 1], M = fmaxf(m, mi), f = fast_exp2(m - M), g = fast_exp2(mi - M);
    y = y * f + x * g;
    l = l * f + li * g;
    m = M;
  }
  *reinterpret_cast<f32x4*>(&s_y[group][d4]) = y;
  if (d4 == 0) s_m[group] = m, s_l[group] = l;
  __syncthreads();
  if (group) return;
  float M = s_m[0], L = 0.f;
#pragma unroll
  for (int w = 1; w < 8; ++w) M = fmaxf(M, s_m[w]);
  y = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    const float f = fast_exp2(s_m[w] - M);
    L += s_l[w] * f;
    y += *reinterpret_cast<const f32x4*>(&s_y[w][d4]) * f;
  }
  const int64_t row = (int64_t)u * c.G + head;
  put_out(c, row, d4, L != 0.f ? y * (1.f / L) : f32x4{0.f, 0.f, 0.f, 0.f});
  if (d4 == 0 && c.lse) c.lse[row] = natural(M, L);
}

// ------------------------------------------------------------------ pages picked for a token
struct Select {
  const uint8_t* q;
  float* scores;             // [unit][columns_up]
  int32_t* picked;           // [unit][keep]
  int64_t q_seq_stride, q_head_stride;
  int32_t G, keep, keep_first, keep_last, pages, score_stride;
};

// A page's score is the sum over the group's heads of the largest logit that its extremes allow, sum_d max(q_d min_d, q_d max_d): with the heads'
// positive and negative parts summed beforehand one product of 256 terms.  In 64 bits, because scores decide: whoever adds up in another order gets the same
// pages.  Sixteen lanes take a page, 8 dimensions of both extremes each.
constexpr int kScorePages = 64;        // per workgroup

// Sum over the lane's row of 16 lanes.
__device__ __forceinline__ double row_sum(double s) {
  s += dpp_f64<kDppQuadSwap1>(s);
  s += dpp_f64<kDppQuadSwap2>(s);
  s += dpp_f64<kDppRowHalfMirror>(s);
  return s + dpp_f64<kDppRowMirror>(s);
}

__global__ __launch_bounds__(kThreads) void paged_score_kernel(Paged p, Select c) {
  const int u = blockIdx.x, b = u / p.hkv, h = u - b * p.hkv, piece = threadIdx.x & 15, group = threadIdx.x >> 4;
  int bad = 0;
  const int length = p.length(b, bad), held = (int)(((int64_t)length + p.page_size() - 1) >> p.shift), first = blockIdx.y * kScorePages;
  if (first >= held || held <= c.keep) return;
  double up[8], down[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) up[i] = down[i] = 0.0;
  for (int g = 0; g < c.G; ++g) {
    float x[8];
    unpack8(load16(c.q + b * c.q_seq_stride + (h * c.G + g) * c.q_head_stride + 16 * piece), x);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      up[i] += x[i] < 0.f ? 0.f : x[i];
      down[i] += x[i] < 0.f ? x[i] : 0.f;
    }
  }
#pragma unroll
  for (int n = 0; n < kScorePages / 16; ++n) {
    const int at = first + 16 * n + group;
    const int page = at < held ? p.page(b, at, bad) : -1;
    const uint8_t* from = p.bounds + max(page, 0) * p.bounds_page_stride + h * p.bounds_head_stride + 16 * piece;
    float lo[8], hi[8];
    unpack8(load16(from), lo);
    unpack8(load16(from + 2 * kDim), hi);
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fma((double)hi[i], up[i], fma((double)lo[i], down[i], s));
    s = row_sum(s);
    if (__any(s != s)) {                  // infinite extremes: where no query has a part of that sign the product is nothing
      s = 0.0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (up[i] != 0.0) s += hi[i] * up[i];
        if (down[i] != 0.0) s += lo[i] * down[i];
      }
      s = row_sum(s);
    }
    if (piece == 0 && at < held) c.scores[(int64_t)u * c.score_stride + at] = page < 0 ? -INFINITY : (float)s;
  }
  if (piece == 0) p.report(bad);
}

// A score's place in the order, best first: 0 for what is no number, then from +inf down (0xFFFFFFFF, "no key", is that of no score).
__device__ __forceinline__ uint32_t score_key(float s) {
  if (s != s) return 0u;
  const uint32_t x = __float_as_uint(s == 0.f ? 0.f : s);
  return ~(x & 0x80000000u ? ~x : x | 0x80000000u);
}

// One workgroup per (sequence, KV head), R consecutive pages per thread: the first and last ones, and of the others those with the best scores (ties: lowest
// page), in ascending order.
template <int R, int NT>
__global__ __launch_bounds__(NT) void paged_pick_kernel(Paged p, Select c) {
  __shared__ CutBuf cb;
  __shared__ int s_count[NT / 64];
  const int u = blockIdx.x, b = u / p.hkv, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int bad = 0;
  const int length = p.length(b, bad), held = (int)(((int64_t)length + p.page_size() - 1) >> p.shift);
  if (tid == 0) p.report(bad);
  int32_t* to = c.picked + (int64_t)u * c.keep;
  if (held <= c.keep) {
    for (int i = tid; i < c.keep; i += NT) to[i] = i < held ? i : -1;
    return;
  }
  uint32_t key[R], index[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int at = tid * R + i;
    const bool open = at >= c.keep_first && at < held - c.keep_last;
    index[i] = (uint32_t)at;
    key[i] = open ? score_key(c.scores[(int64_t)u * c.score_stride + at]) : 0xFFFFFFFFu;
  }
  const int want = c.keep - c.keep_first - c.keep_last;
  KeyCut cut{0u, 0u};
  if (want > 0) cut = select_low_keys<R, NT>(key, index, want, cb, tid);
  int mine = 0;
  uint32_t taken = 0u;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int at = tid * R + i;
    const bool open = at >= c.keep_first && at < held - c.keep_last;
    const bool take = at < held && (!open || (want > 0 && cut(key[i], index[i])));
    taken |= (take ? 1u : 0u) << i;
    mine += take;
  }
  const int upto = wave_scan_i32(mine, lane);
  if (lane == 63) s_count[wave] = upto;
  __syncthreads();
  int at = upto - mine;
  for (int w = 0; w < wave; ++w) at += s_count[w];
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (taken >> i & 1u) {
      if (at < c.keep) to[at] = tid * R + i;
      ++at;
    }
}

}  // namespace ckv
