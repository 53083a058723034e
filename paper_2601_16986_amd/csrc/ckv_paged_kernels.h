// Device code of the cache in pages: rows in (quantised as they are written) and out, attention of one new token per sequence
// over its pages or over pages picked for it, and the picking.
#pragma once
#include <type_traits>

#include "ckv_paged_device.h"
#include "ckv_rows.h"

namespace ckv {

// ------------------------------------------------------------------ rows
// One workgroup per (sequence, KV head) and page that new rows reach: it alone touches the page's rows and extremes, so that these need no atomics.  Sixteen
// lanes take a row, 16 bytes of bf16 each, for key and value.  Where rows are many it is bound by memory: 322208 rows (165 MB in, 83 MB out) 57 us, 4.3 TB/s, where a plain copy
// reaches 4.7, as bf16 (165 MB out) 77 us, 4.3 TB/s; magnitudes and codes from packed bf16 instead of floats were worth a fifth where the rows were in the caches (72192 rows 19.3 -> 16.1 us).  A single
// row of each of 32 sequences, 8 heads, takes 4 us: four dependent trips to memory.  (Spans of 64 rows of smaller pages, all rows asked for at once, took
// longer: 69 us, and 6 instead of 4 for a prompt of 777.)
template <bool E4M3, int NT>
__global__ __launch_bounds__(NT) void paged_append_kernel(Paged p, Rows r) {
  __shared__ float s_lo[NT / 64][kDim], s_hi[NT / 64][kDim];
  const int u = blockIdx.x, b = u / p.hkv, h = u - b * p.hkv;
  const int tid = threadIdx.x, piece = tid & 15, group = tid >> 4;
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
  if (page < 0) return;
  const int64_t at = page * p.page_stride + h * p.head_stride;
  Extremes<E4M3, NT> extremes;
  for (int row = begin + group; row < end; row += NT / 16) {
    const int64_t from = base + (int64_t)(row - span.first) * r.row_stride + h * r.head_stride + 16 * piece;
    const int slot = row & (p.page_size() - 1);
    u32x4 k = load16(r.k + from), v = load16(r.v + from);
    if constexpr (E4M3) {
      uint32_t ek, ev;
      const u32x2 ck = quantise8(k, ek), cv = quantise8(v, ev);
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
  if (p.bounds) extremes.write(p, page, h, col, begin, end, length, s_lo, s_hi, tid);
}

// Sixteen lanes take a row, 32 rows per workgroup, two of them asked for at once (64 rows, four at once: 60.4 us for 322208 rows that now take 49.9).  PAST: rows are
// stored past the caches (reads_past_caches).
constexpr int kReadRows = 32;
template <bool E4M3, bool PAST>
__global__ __launch_bounds__(kThreads) void paged_read_kernel(Paged p, Rows r) {
  const int u = blockIdx.x, b = u / p.hkv, h = u - b * p.hkv, piece = threadIdx.x & 15, group = threadIdx.x >> 4;
  int bad = 0;
  p.length(b, bad);
  int64_t base;
  const RowSpan rows = r.span(b, uniform_i32(p.lengths[b]), p.max_length, base);
  if (rows.bad) bad |= PAGED_BAD_LENGTH;
  const int first = blockIdx.y * kReadRows;
  if (first >= rows.count) {
    if (blockIdx.y == 0 && threadIdx.x == 0) p.report(bad);
    return;
  }
  constexpr int N = kReadRows / 16;
  int page[N];
  u32x4 k[N], v[N];
  uint32_t s[N];
#pragma unroll
  for (int n = 0; n < N; ++n) page[n] = p.page(b, (rows.first + min(first + 16 * n + group, rows.count - 1)) >> p.shift, bad);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int slot = (rows.first + min(first + 16 * n + group, rows.count - 1)) & (p.page_size() - 1);
    const int64_t pg = max(page[n], 0), from = pg * p.page_stride + h * p.head_stride + (int64_t)slot * p.slot_stride;
    if constexpr (E4M3) {
      const u32x2 a = load8(p.k + from + 8 * piece), z = load8(p.v + from + 8 * piece);
      k[n] = u32x4{a[0], a[1], 0u, 0u};
      v[n] = u32x4{z[0], z[1], 0u, 0u};
      s[n] = *reinterpret_cast<const uint16_t*>(p.scales + pg * p.scale_page_stride + h * p.scale_head_stride + 2 * slot);
    } else {
      k[n] = load16(p.k + from + 16 * piece);
      v[n] = load16(p.v + from + 16 * piece);
    }
  }
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int i = first + 16 * n + group;
    if (i >= rows.count || page[n] < 0) continue;
    const int64_t to = base + (int64_t)i * r.row_stride + h * r.head_stride + 16 * piece;
    if constexpr (E4M3) {
      k[n] = values8(u32x2{k[n][0], k[n][1]}, __uint_as_float((s[n] & 0xFF) << 23));
      v[n] = values8(u32x2{v[n][0], v[n][1]}, __uint_as_float((s[n] >> 8) << 23));
    }
    if constexpr (PAST) {
      __builtin_nontemporal_store(k[n], reinterpret_cast<u32x4*>(r.k + to));
      __builtin_nontemporal_store(v[n], reinterpret_cast<u32x4*>(r.v + to));
    } else {
      *reinterpret_cast<u32x4*>(r.k + to) = k[n];
      *reinterpret_cast<u32x4*>(r.v + to) = v[n];
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
  float* partial;            // [piece][G][128]
  float* ml;                 // [piece][G][2]
  int32_t* parts;            // [unit][2]: its first piece, and how many it has
  int64_t q_seq_stride, q_head_stride;     // bytes
  float scale_log2e;
  int32_t G, n_picked, out_bf16;
  int32_t share, places, workers;          // AttendPlan
  const int32_t* first;      // WINDOW: the tokens' positions, or NULL: the sequences' last
  int32_t window, sinks;     // WINDOW: entries that a token looks back to, itself included, and first ones
  float lower;               // WINDOW: lowered_by(), what weights are multiplied by where sums would be infinite
};

// What one token looks at: all entries of its sequence or, WINDOW, those up to its own position, of which only the last `window` and the first `sinks` count.
struct Sight {
  int end, oldest;           // entries oldest .. end - 1, and the first sinks
  RowTiles blocks;           // in blocks of 32
};
template <bool WINDOW>
__device__ __forceinline__ int sight_end(const Paged& p, const Attend& c, int b, int& bad) {
  if constexpr (!WINDOW) return p.length(b, bad);
  p.length(b, bad);
  const RowSpan s = rows_below(row_span(p.lengths[b], 1, c.first != nullptr, c.first ? c.first[b] : 0, false, 0, 0, 0), p.max_length);
  if (s.bad) bad |= PAGED_BAD_LENGTH;
  return s.count ? s.first + 1 : 0;
}
template <bool WINDOW>
__device__ __forceinline__ Sight sight_of(const Attend& c, int end) {
  if constexpr (!WINDOW) return {end, 0, {0, 0, unit_blocks(end)}};
  Sight s = {end, c.window && end > c.window ? end - c.window : 0, {}};
  s.blocks = row_tiles(s.oldest, end, c.sinks, 32);
  if (s.blocks.count == 0) s.blocks.count = 1;
  return s;
}

// Two rows of a pair of entries into pairs of one dimension: word w of the result holds dimension w of both.
__device__ __forceinline__ void interleave_bytes(uint32_t a, uint32_t b, uint32_t (&x)[2]) {
  x[0] = __builtin_amdgcn_perm(b, a, 0x05010400u);
  x[1] = __builtin_amdgcn_perm(b, a, 0x07030602u);
}

__device__ __forceinline__ void put_out(const Attend& c, int64_t row, int d4, f32x4 y) {
  if (c.out_bf16) *reinterpret_cast<u32x2*>(c.out + (row * kDim + d4) * 2) = u32x2{bf16_pack(y[0], y[1]), bf16_pack(y[2], y[3])};
  else *reinterpret_cast<f32x4*>(c.out + (row * kDim + d4) * 4) = y;
}

// Sums of weights of which some, those with a sign, belong to outputs of lowered weights: all outputs are then taken as lowered.
template <bool WINDOW>
struct Lowered {
  float by = 1.f;
  template <class... T>
  __device__ __forceinline__ Lowered(const Attend& c, T... l) {
    if constexpr (WINDOW)
      if (((0u | ... | __float_as_uint(l)) >> 31) != 0u) by = c.lower;
  }
  __device__ __forceinline__ bool any() const { return WINDOW && by < 1.f; }
  __device__ __forceinline__ float size(float l) const { return WINDOW ? fabsf(l) : l; }
  __device__ __forceinline__ float factor(float l, float f) const { return WINDOW && !(__float_as_uint(l) >> 31) ? f * by : f; }
  __device__ __forceinline__ f32x4 raise(f32x4 y) const { return WINDOW ? y * (1.f / by) : y; }
};
// All ones in each half (a bf16 number) that is not finite.
__device__ __forceinline__ u32x4 not_finite(u32x4 x) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = ((x[i] & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((x[i] & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u);
  return r;
}

// The piece that a workgroup takes.  Where lengths decide how the work is cut they are only known here, so every workgroup looks for its own; a lane adds up its
// share of the sequences.  Large pieces come first: the chip's last ones to end are then small.
struct Piece {
  int b, h, length, index, first, last, parts, part;      // length: the end of what the token sees; blocks first .. last - 1 of the unit; piece `index` of all, `part` of the unit's `parts`
};
__device__ __forceinline__ int lane_at(int v, int lane) { return __builtin_amdgcn_ds_bpermute(lane << 2, v); }
template <bool WINDOW>
__device__ __forceinline__ bool find_piece(const Paged& p, const Attend& c, int index, int lane, int& bad, Piece& r) {
  const int fixed = !WINDOW && c.picked ? unit_blocks(c.n_picked << p.shift) : 0;
  auto length_of = [&](int b) { return sight_end<WINDOW>(p, c, b, bad); };
  auto blocks_of = [&](int length) { return sight_of<WINDOW>(c, length).blocks.count; };
  int n;
  if (c.share) {
    const int u = index / c.places;
    r.part = index - u * c.places;
    r.b = u / p.hkv;
    r.h = u - r.b * p.hkv;
    r.length = uniform_i32(length_of(r.b));
    n = fixed ? fixed : blocks_of(r.length);
    r.parts = unit_parts(n, c.share);
    if (r.part >= r.parts) return false;
  } else {
    const int per_lane = (p.batch + 63) >> 6, b0 = lane * per_lane;
    int length = 0, blocks = 0, pieces = 0, who = lane;
    for (int i = 0; i < per_lane && b0 + i < p.batch; ++i) {
      const int m = length_of(b0 + i);
      if (i == 0) length = m;
      blocks += blocks_of(m);
    }
    int share = attend_share(wave_sum_i32(blocks) * p.hkv, c.workers);
    if (per_lane == 1) {
      for (int i = 0; i < 2 && enlarges_share(p.batch, p.hkv, c.workers); ++i) {
        const int all = wave_sum_i32(unit_parts(blocks, share)) * p.hkv;
        if (all <= c.workers) break;
        share = larger_share(share, all, c.workers);
      }
      pieces = unit_parts(blocks, share);
      const int size = pieces ? unit_parts(blocks, pieces) : 0;
      int rank = 0;
      for (int i = 0; i < p.batch; ++i) {
        const int other = __builtin_amdgcn_readlane(size, i);
        rank += other > size || (other == size && i < lane);
      }
      who = __builtin_amdgcn_ds_permute((lane < p.batch ? rank : lane) << 2, lane);
      pieces = lane_at(pieces, who);
      length = lane_at(length, who);
    } else {
      for (int i = 0; i < per_lane && b0 + i < p.batch; ++i) pieces += unit_parts(blocks_of(length_of(b0 + i)), share);
    }
    pieces *= p.hkv;
    const int upto = wave_scan_i32(pieces, lane);
    const u64 beyond = __ballot(upto > index);
    if (beyond == 0) return false;
    const int ln = __ffsll((long long)beyond) - 1;
    int before = __builtin_amdgcn_readlane(upto - pieces, ln);
    r.b = __builtin_amdgcn_readlane(who, ln) * per_lane;
    r.length = __builtin_amdgcn_readlane(length, ln);
    for (;;) {
      n = blocks_of(r.length);
      r.parts = unit_parts(n, share);
      if (index < before + r.parts * p.hkv) break;
      before += r.parts * p.hkv;
      r.length = uniform_i32(length_of(++r.b));
    }
    r.h = (index - before) / r.parts;
    r.part = index - before - r.h * r.parts;
  }
  r.index = index;
  r.first = part_begin(n, r.parts, r.part);
  r.last = part_begin(n, r.parts, r.part + 1);
  return true;
}

// One workgroup of four wavefronts per piece; wavefronts take blocks of 32 entries in turn.  With the rows as
// they lie a lane (j = lane % 16, kg = lane / 16) reads of a block, per tile of 16 entries,
//   keys    of entries 4 (j / 4) + (j / 2) % 2 and that + 2, 16 bytes at 16 (2 kg + j % 2) of each 128: every load takes whole lines (with 16 bytes of all sixteen
//           rows it took halves: 64 sequences of 9350 entries 198 us, 269 where a slot's heads lie side by side). As operands of K Q^T (rows = entries) even rows hold
//           other dimensions than odd ones, so that each goes with both halves of the queries and half of the results are used;
//   values  entries 4 kg .. 4 kg + 3, the eighth of the row at j: byte (or word) moves between pairs of entries make them operands of P V (columns =
//           dimensions 8 j + dt), in the entry order in which K Q^T leaves the logits.
// The weights are split into three bf16 terms, which hold the 24 bits of a float: the high ones in rows 0 .. 7 and the second ones in rows 8 .. 15 of one operand for up to
// eight heads (the queries are there twice), the third in another; operands of their own for more heads (WIDE).  (Two terms, 16
// bits: 1 us less of 190, and outputs that nearly cancel off by 2^-18 of their terms.)
//
// It is bound by memory: 64 sequences x 8 KV heads of 9350 entries in 8 bits, 1236 MB (1240 by the counters), 190 us, 6.5 TB/s of the 7.1 of a plain read, and the same
// without any of the arithmetic, which keeps the vector units busy for a quarter of the time; 16 heads per KV head instead of 4 take 3 % longer, float outputs no longer.  Eight wavefronts per compute unit are enough, and more, or blocks asked
// for one ahead, only make the streams more: 12 .. 16 of them 202 .. 217 us, 8 KB instead of 4 KB in flight each 191.  A piece costs some 3 us beside its
// entries (length, page, rows: three trips; joining four wavefronts), so pieces are as few as fill the chip: twice, four, eight times as many 202, 205, 208 us.
template <bool E4M3, bool WIDE, bool WINDOW = false>
__global__ __launch_bounds__(kThreads) void paged_attend_kernel(Paged p, Attend c) {
  constexpr int kHeads = WIDE ? 16 : 8, kTerms = 3, kWaves = kAttendWaves, kRow = kDim + 4, kParts = E4M3 ? 1 : 2;
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  __shared__ __align__(16) float s_acc[kWaves][kHeads * kRow];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform_i32(tid >> 6), j = lane & 15, kg = lane >> 4, shift = p.shift;
  int bad = 0;
  Piece pc;
  if (!find_piece<WINDOW>(p, c, blockIdx.x, lane, bad, pc)) return;
  const int b = pc.b, h = pc.h, u = b * p.hkv + h;

  // ---- where the unit's pages lie and how far they are filled, kPageSlots of them at a time, a lane each
  const Sight sight = sight_of<WINDOW>(c, pc.length);
  const int oldest = sight.oldest, end = sight.end;
  auto block = [&](int n) { return WINDOW ? sight.blocks.tile(n) : n; };
  int page, fill, window = block(pc.first) >> (shift + 1);
  auto look_up = [&]() {
    int logical = window * kPageSlots + lane;
    if (!WINDOW && c.picked) logical = logical < c.n_picked ? c.picked[(int64_t)u * c.n_picked + logical] : -1;
    page = logical >= 0 && logical < p.columns ? p.table[(int64_t)b * p.table_stride + logical] : 0;      // before the length is there
    fill = logical < 0 || logical >= p.columns ? 0 : page_fill(pc.length, logical, shift);
    if (WINDOW && fill > 0 && (logical + 1) << shift <= oldest && logical << shift >= c.sinks) fill = 0;         // a page that the token does not look at
    if (!WINDOW && c.picked && (logical < -1 || (logical >= 0 && fill == 0))) bad |= PAGED_BAD_PICK;
    if (fill > 0 && !page_there(page, p.n_pages)) {
      bad |= PAGED_BAD_PAGE;
      fill = 0;
    }
    if (fill == 0) page = 0;
  };
  look_up();

  bf16x8 q[4];
  {
    const int head = WIDE ? j : j & 7;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int d = E4M3 ? 32 * kg + 16 * (s >> 1) + 8 * (s & 1) : 64 * (s & 1) + 16 * kg + 8 * (s >> 1);
      u32x4 x = {0u, 0u, 0u, 0u};
      if (head < c.G) x = load16(c.q + b * c.q_seq_stride + (h * c.G + head) * c.q_head_stride + 2 * d);
      q[s] = __builtin_bit_cast(bf16x8, x);
    }
  }
  f32x4 acc[8];
#pragma unroll
  for (int dt = 0; dt < 8; ++dt) acc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = kNoLogit, l_run = 0.f;

  float lowered = 1.f;
  auto blocks = [&](auto careful) __attribute__((always_inline)) {
    constexpr bool CAREFUL = decltype(careful)::value;
    for (int in = pc.first + wave; in < pc.last; in += kWaves) {
      const int blk = block(in);
      if (blk >> (shift + 1) != window) {
        window = blk >> (shift + 1);
        look_up();
      }
      int valid[2];
      float sv[8], vs[8];
      u32x4 kf[2][2][kParts], vf[2][4];
      u32x2 sc[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int e = (blk << 5) + 16 * t, off = e & ((1 << shift) - 1), at = (e >> shift) & (kPageSlots - 1);
        valid[t] = min(max(__builtin_amdgcn_readlane(fill, at) - off, 0), 16);
        const int64_t pg = __builtin_amdgcn_readlane(page, at);
        const int64_t base = pg * p.page_stride + h * p.head_stride + (int64_t)off * p.slot_stride;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const uint8_t* kb = p.k + base + (4 * (j >> 2) + ((j >> 1) & 1) + 2 * n) * p.slot_stride + 16 * (2 * kg + (j & 1));
#pragma unroll
          for (int s = 0; s < kParts; ++s) kf[t][n][s] = stream16(kb + 128 * s);
        }
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
        if constexpr (E4M3) sc[t] = load8(p.scales + pg * p.scale_page_stride + h * p.scale_head_stride + 2 * off + 8 * kg);      // (through the caches: a line serves several blocks)
      }
      // ---- logits of four entries of each tile
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        float dot[4];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            u32x4 x;
            if constexpr (E4M3) {
              const uint32_t lo = kf[t][n][0][2 * s], hi = kf[t][n][0][2 * s + 1];
              x = u32x4{codes_bf16<false>(lo, 1.f), codes_bf16<true>(lo, 1.f), codes_bf16<false>(hi, 1.f), codes_bf16<true>(hi, 1.f)};
            } else {
              x = kf[t][n][s];
            }
            s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), q[s], s0, 0, 0, 0);
            s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), q[2 + s], s1, 0, 0, 0);
          }
          dot[2 * n] = s0[0] + s1[1];
          dot[2 * n + 1] = s0[2] + s1[3];
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
          sv[4 * t + i] = dot[i] * k_scale;
        }
      }
      // ---- entries that are not there, or not looked at: logits of -inf, values and their scales of nothing (the rows may hold anything)
      if (valid[0] + valid[1] < 32 || (WINDOW && blk << 5 < oldest && (blk + 1) << 5 > c.sinks)) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (const int e = (blk << 5) + 16 * t + 4 * kg + i; 4 * kg + i >= valid[t] || (WINDOW && e < oldest && e >= c.sinks)) {
              sv[4 * t + i] = -INFINITY;
              vs[4 * t + i] = 0.f;
              vf[t][i] = u32x4{0u, 0u, 0u, 0u};
            }
      }
      if constexpr (CAREFUL && E4M3) {                   // codes times 2^120 that are infinite as bf16
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (vs[i] == 0x1p120f) {
#pragma unroll
            for (int n = 0; n < 2; ++n) vf[i >> 2][i & 3][n] |= ((((vf[i >> 2][i & 3][n] & 0x7F7F7F7Fu) + 0x08080808u) & 0x80808080u) >> 7) * 0x7Fu;
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
      bf16x8 w[kTerms], some;                            // some: careful, 1 where there is a weight
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float weight = fast_exp2(sv[i] - m_run);
        l_run += weight;
        float rest = E4M3 ? weight * vs[i] : weight;
        if constexpr (CAREFUL) some[i] = (__bf16)(weight != 0.f ? 1.f : 0.f), rest *= lowered;
#pragma unroll
        for (int n = 0; n < kTerms; ++n) {
          w[n][i] = (__bf16)rest;
          rest -= (float)w[n][i];
        }
      }
      if constexpr (!WIDE) {
        const bool low = j >= 8;
        const u32x4 a = __builtin_bit_cast(u32x4, w[0]), z = __builtin_bit_cast(u32x4, w[1]), y = __builtin_bit_cast(u32x4, w[2]);
        w[0] = __builtin_bit_cast(bf16x8, u32x4{low ? z[0] : a[0], low ? z[1] : a[1], low ? z[2] : a[2], low ? z[3] : a[3]});
        w[1] = __builtin_bit_cast(bf16x8, u32x4{low ? 0u : y[0], low ? 0u : y[1], low ? 0u : y[2], low ? 0u : y[3]});
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
        f32x4 wrong[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        if constexpr (CAREFUL) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const u32x4 ones = not_finite(x[i]);
            wrong[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(some, __builtin_bit_cast(bf16x8, ones & 0x3F803F80u), wrong[i], 0, 0, 0);
            x[i] &= ~ones;
          }
        }
#pragma unroll
        for (int n = 0; n < (WIDE ? kTerms : kTerms - 1); ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i)
            acc[2 * d2 + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[n], __builtin_bit_cast(bf16x8, x[i]), acc[2 * d2 + i], 0, 0, 0);
        if constexpr (CAREFUL) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (wrong[i][e] != 0.f) acc[2 * d2 + i][e] = NAN;
        }
      }
    }
  };
  blocks(std::false_type());
  if constexpr (WINDOW) {
    // With care where something that is no number came out, so that values reach those heads only that give them weight; then with lowered weights too where that
    // leaves anything so large that pieces' sums might be infinite, or no number.
    auto sound = [&]() __attribute__((always_inline)) {        // below 2^115, and numbers
      float nothing = 0.f;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) nothing = fmaf(acc[dt][i], kLargeSums, nothing);
      return fabsf(nothing) < INFINITY;
    };
    if (__any(!sound())) {
      asm volatile("");                                    // keeps this in the branch
#pragma unroll 1
      for (int turn = 0; turn < 2; ++turn) {
        if (turn == 1) {
          if (!__any(!sound())) break;                     // (what is no number may be infinity less infinity)
          lowered = c.lower;
        }
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) acc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        m_run = kNoLogit, l_run = 0.f;
        blocks(std::true_type());
      }
    }
  }

  // ---- the wavefronts' states into one
  l_run = rows_combine(l_run, [](float x, float y) { return x + y; });
  if (lane < 16) {
    s_m[wave][lane] = m_run;
    s_l[wave][lane] = WINDOW && lowered < 1.f ? -l_run : l_run;          // of lowered weights the sum, which is not lowered, has a sign
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
    const Lowered<WINDOW> all(c, s_l[0][head], s_l[1][head], s_l[2][head], s_l[3][head]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = fast_exp2(s_m[w][head] - M);
      L += all.size(s_l[w][head]) * f;
      y += *reinterpret_cast<const f32x4*>(&s_acc[w][head * kRow + d4]) * all.factor(s_l[w][head], f);
    }
    if (pc.parts > 1) {
      const int64_t at = (int64_t)pc.index * c.G + head;
      *reinterpret_cast<f32x4*>(c.partial + at * kDim + d4) = y;
      if (d4 == 0) {
        c.ml[2 * at] = M;
        c.ml[2 * at + 1] = all.any() ? -L : L;
      }
    } else if (!WINDOW || end > 0) {
      const int64_t row = (int64_t)u * c.G + head;
      put_out(c, row, d4, L != 0.f ? all.raise(y * (1.f / L)) : f32x4{0.f, 0.f, 0.f, 0.f});
      if (d4 == 0 && c.lse) c.lse[row] = natural(M, L);
    }
  }
  if (c.parts && pc.part == 0 && tid == 0) {
    c.parts[2 * u] = pc.index;
    c.parts[2 * u + 1] = pc.parts;
  }
  p.report(bad);
}

// Joins the pieces of units that have several: a workgroup takes `heads` query heads of a unit, eight / heads rows of 32 threads (four dimensions each) a head, a row eight
// parts at a time.  2.6 .. 4.7 us, of which a launch and three trips to memory are most.  (The last workgroup to arrive at a counter joining instead, with accesses past the
// caches: the same times or 2 us more, and the counters would have to be zero before.)
constexpr int kJoinRows = 8;
template <bool WINDOW>
__global__ __launch_bounds__(32 * kJoinRows) void paged_join_kernel(Attend c, int heads) {
  __shared__ float s_m[kJoinRows], s_l[kJoinRows];
  __shared__ __align__(16) float s_y[kJoinRows][kDim];
  const int u = blockIdx.x, sides = kJoinRows / heads, row = threadIdx.x >> 5, side = row / heads, lane = threadIdx.x & 31, d4 = 4 * lane;
  const int first = c.parts[2 * u], parts = c.parts[2 * u + 1], head = min((int)blockIdx.y * heads + row - side * heads, c.G - 1);
  if (parts == 1) return;
  float M = kNoLogit, L = 0.f;
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
  Lowered<WINDOW> mine(c);
  auto take = [&](auto n, int i0) {                         // parts i0, i0 + sides, ..., n of them
    constexpr int N = decltype(n)::value;
    f32x4 x[N];
    f32x2 st[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int64_t at = (int64_t)(first + min(i0 + k * sides, parts - 1)) * c.G + head;
      st[k] = *reinterpret_cast<const f32x2*>(c.ml + 2 * at);
      x[k] = *reinterpret_cast<const f32x4*>(c.partial + at * kDim + d4);
    }
    float m = M;
#pragma unroll
    for (int k = 0; k < N; ++k) m = fmaxf(m, st[k][0]);
    if constexpr (WINDOW) {
      uint32_t signs = 0u;
#pragma unroll
      for (int k = 0; k < N; ++k) signs |= __float_as_uint(st[k][1]);
      if (signs >> 31 && !mine.any()) mine.by = c.lower, y = y * mine.by;
    }
    const float shrink = fast_exp2(M - m);
    M = m;
    L *= shrink;
    y = y * shrink;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float f = i0 + k * sides < parts ? fast_exp2(st[k][0] - m) : 0.f;
      L += mine.size(st[k][1]) * f;
      y += x[k] * mine.factor(st[k][1], f);
    }
  };
  if (side < sides) {
    int i = side;
    for (; i - side + 2 * sides < parts; i += 8 * sides) take(std::integral_constant<int, 8>(), i);
    if (i - side < parts) take(std::integral_constant<int, 2>(), i);
  }
  if (lane == 0) s_m[row] = M, s_l[row] = mine.any() ? -L : L;
  *reinterpret_cast<f32x4*>(&s_y[row][d4]) = y;
  __syncthreads();
  if (row >= heads || (int)blockIdx.y * heads + row >= c.G) return;
  for (int s = 1; s < sides; ++s) M = fmaxf(M, s_m[s * heads + row]);
  L = 0.f;
  y = f32x4{0.f, 0.f, 0.f, 0.f};
  Lowered<WINDOW> all(c);
  if constexpr (WINDOW)
    for (int s = 0; s < sides; ++s)
      if (__float_as_uint(s_l[s * heads + row]) >> 31) all.by = c.lower;
  for (int s = 0; s < sides; ++s) {
    const float l = s_l[s * heads + row], f = fast_exp2(s_m[s * heads + row] - M);
    L += all.size(l) * f;
    y += *reinterpret_cast<const f32x4*>(&s_y[s * heads + row][d4]) * all.factor(l, f);
  }
  const int64_t to = (int64_t)u * c.G + head;
  put_out(c, to, d4, L != 0.f ? all.raise(y * (1.f / L)) : f32x4{0.f, 0.f, 0.f, 0.f});
  if (d4 == 0 && c.lse) c.lse[to] = natural(M, L);
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
// pages.  Sixteen lanes take a page, 8 dimensions of both extremes each; the arithmetic (16 products in 64 bits and a sum over the lanes) is a third of what the
// memory allows.  512 units of 1000 pages (262 MB) 54 us with the picking; 8 of 2048 5.6 and 4.9, where the picking's rounds over the workgroup decide (512 threads; 256 or 1024 0.6 longer).
struct Parts {
  double up[8], down[8];
};
__device__ __forceinline__ Parts query_parts(const Paged& p, const Select& c, int b, int h, int piece) {
  Parts r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r.up[i] = r.down[i] = 0.0;
  const uint8_t* q = c.q + b * c.q_seq_stride + h * c.G * c.q_head_stride + 16 * piece;
  for (int g0 = 0; g0 < c.G; g0 += 8) {
    u32x4 x[8];
#pragma unroll
    for (int g = 0; g < 8; ++g) x[g] = load16(q + min(g0 + g, c.G - 1) * c.q_head_stride);      // all on their way before the first is looked at
#pragma unroll
    for (int g = 0; g < 8; ++g) {
      if (g0 + g >= c.G) break;
      float y[8];
      unpack8(x[g], y);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        r.up[i] += y[i] < 0.f ? 0.f : y[i];
        r.down[i] += y[i] < 0.f ? y[i] : 0.f;
      }
    }
  }
  return r;
}

// Sum over the lane's row of 16 lanes.
__device__ __forceinline__ double row_sum(double s) {
  s += dpp_f64<kDppQuadSwap1>(s);
  s += dpp_f64<kDppQuadSwap2>(s);
  s += dpp_f64<kDppRowHalfMirror>(s);
  return s + dpp_f64<kDppRowMirror>(s);
}

// Scores of the sequence's pages first, first + step, ... (N of them, as far as there are so many) to put(page, score).
template <int N, bool PAST, class Put>
__device__ __forceinline__ void score_pages(const Paged& p, int b, int h, int held, int first, int step, const Parts& q, int piece, int& bad, Put put) {
  int page[N];
#pragma unroll
  for (int n = 0; n < N; ++n) page[n] = p.table[(int64_t)b * p.table_stride + min(first + n * step, held - 1)];
  u32x4 least[N], most[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if (!page_there(page[n], p.n_pages)) {
      if (first + n * step < held) bad |= PAGED_BAD_PAGE;
      page[n] = -1;
    }
    const uint8_t* from = p.bounds + max(page[n], 0) * p.bounds_page_stride + h * p.bounds_head_stride + 16 * piece;
    least[n] = PAST ? stream16(from) : load16(from);
    most[n] = PAST ? stream16(from + 2 * kDim) : load16(from + 2 * kDim);
  }
#pragma unroll
  for (int n = 0; n < N; ++n) {
    float lo[8], hi[8];
    unpack8(least[n], lo);
    unpack8(most[n], hi);
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fma((double)hi[i], q.up[i], fma((double)lo[i], q.down[i], s));
    s = row_sum(s);
    // Extremes that are infinite, or no numbers: where no query has a part of that sign the product is nothing, and a dimension without any number in the page has the larger
    // one, +inf, as least.  (Least and largest put in order for all pages alike: 512 units of 293 pages 14.5 -> 15.5 us.)
    if (__any(!(fabs(s) < INFINITY))) {
      double t = 0.0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (q.up[i] != 0.0) t += max2(lo[i], hi[i]) * q.up[i];
        if (q.down[i] != 0.0) t += min2(lo[i], hi[i]) * q.down[i];
      }
      t = row_sum(t);
      if (!(fabs(s) < INFINITY)) s = t;                  // (the wavefront's other pages keep theirs)
    }
    if (piece == 0 && first + n * step < held) put(first + n * step, page[n] < 0 ? -INFINITY : (float)s);
  }
}
__device__ __forceinline__ int pages_held(const Paged& p, int length) { return (int)(((int64_t)length + p.page_size() - 1) >> p.shift); }

// A workgroup takes `each` pages of a unit, 64 at a time.  PAST: extremes are read past the caches (bounds_past_caches).
template <bool PAST>
__global__ __launch_bounds__(kThreads) void paged_score_kernel(Paged p, Select c, int each) {
  const int u = blockIdx.x, b = u / p.hkv, h = u - b * p.hkv, piece = threadIdx.x & 15, group = threadIdx.x >> 4;
  int bad = 0;
  const int held = pages_held(p, p.length(b, bad)), first = blockIdx.y * each;
  if (first >= held || held <= c.keep) return;
  const Parts q = query_parts(p, c, b, h, piece);
  float* to = c.scores + (int64_t)u * c.score_stride;
  const int last = min(first + each, held);
  for (int at = first; at < last; at += 64)
    score_pages<4, PAST>(p, b, h, last, at + group, 16, q, piece, bad, [&](int page, float s) { to[page] = s; });
  if (piece == 0) p.report(bad);
}

// A score's place in the order, best first: 0 for what is no number, then from +inf down (0xFFFFFFFF, "no key", is that of no score).
__device__ __forceinline__ uint32_t score_key(float s) {
  if (s != s) return 0u;
  const uint32_t x = __float_as_uint(s == 0.f ? 0.f : s);
  return ~(x & 0x80000000u ? ~x : x | 0x80000000u);
}

// The first and last pages of a unit, and of the others those with the best scores (ties: lowest page), in ascending order, by a workgroup of NT threads with R
// consecutive pages each.
template <int NT>
struct PickBuf {
  CutBuf cut;
  int count[NT / 64];
};
template <int R, int NT>
__device__ __forceinline__ void pick_pages(const Select& c, int u, int held, const float* scores, PickBuf<NT>& pb, int tid) {
  const int lane = tid & 63, wave = tid >> 6;
  int32_t* to = c.picked + (int64_t)u * c.keep;
  if (held <= c.keep) {
    for (int i = tid; i < c.keep; i += NT) to[i] = i < held ? i : -1;
    return;
  }
  auto open = [&](int at) { return at >= c.keep_first && at < held - c.keep_last; };
  uint32_t key[R], index[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int at = tid * R + i;
    index[i] = (uint32_t)at;
    key[i] = open(at) ? score_key(scores[at]) : 0xFFFFFFFFu;
  }
  const int want = c.keep - c.keep_first - c.keep_last;
  KeyCut cut{0u, 0u};
  if (want > 0) cut = select_low_keys<R, NT>(key, index, want, pb.cut, tid);
  int mine = 0;
  uint32_t taken = 0u;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int at = tid * R + i;
    const bool take = at < held && (!open(at) || (want > 0 && cut(key[i], index[i])));
    taken |= (take ? 1u : 0u) << i;
    mine += take;
  }
  const int upto = wave_scan_i32(mine, lane);
  if (lane == 63) pb.count[wave] = upto;
  __syncthreads();
  int at = upto - mine;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) at += w < wave ? pb.count[w] : 0;
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (taken >> i & 1u) {
      if (at < c.keep) to[at] = tid * R + i;
      ++at;
    }
}

template <int R, int NT>
__global__ __launch_bounds__(NT) void paged_pick_kernel(Paged p, Select c) {
  __shared__ PickBuf<NT> pb;
  const int u = blockIdx.x, b = u / p.hkv, tid = threadIdx.x;
  int bad = 0;
  const int held = pages_held(p, p.length(b, bad));
  if (tid == 0) p.report(bad);
  pick_pages<R, NT>(c, u, held, c.scores + (int64_t)u * c.score_stride, pb, tid);
}

// Scores and picking by one workgroup per unit, where units have few pages.
constexpr int kPickThreads = 512;
template <bool PAST>
__global__ __launch_bounds__(kPickThreads) void paged_select_kernel(Paged p, Select c) {
  __shared__ PickBuf<kPickThreads> pb;
  __shared__ float s_scores[kFewPages];
  const int u = blockIdx.x, b = u / p.hkv, h = u - b * p.hkv, tid = threadIdx.x, piece = tid & 15, group = tid >> 4;
  constexpr int kGroups = kPickThreads / 16;
  int bad = 0;
  const int held = pages_held(p, p.length(b, bad));
  if (held > c.keep) {
    const Parts q = query_parts(p, c, b, h, piece);
    for (int first = group; first < held; first += 4 * kGroups)
      score_pages<4, PAST>(p, b, h, held, first, kGroups, q, piece, bad, [&](int page, float s) { s_scores[page] = s; });
    __syncthreads();
  }
  p.report(bad);
  pick_pages<kFewPages / kPickThreads, kPickThreads>(c, u, held, s_scores, pb, tid);
}

}  // namespace ckv
