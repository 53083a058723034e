// Device code of attention of several rows per sequence over a cache in pages: each row over itself and what comes before it, all of it or a window with a few first entries,
// or, where rows are drafted tokens, over what comes before all of them and those that its mask names.
#pragma once
#include <type_traits>

#include "ckv_paged_device.h"
#include "ckv_rows.h"

#define CKV_INLINE __attribute__((always_inline))

namespace ckv {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

struct RowsAttend {
  Rows rows;                 // k: the queries (bf16)
  const uint8_t* tree;       // [batch][rows][rows], not 0: the row (second) sees the one it names (third); or NULL
  uint8_t* out;              // [row][query head][128]
  float* lse;
  float* partial;            // [piece][rows of a block][128]
  float* ml;                 // [piece][rows of a block][2]
  int32_t* parts;            // [unit][block]: pieces that its blocks fall into
  int64_t tree_seq, tree_row;
  int64_t units;
  float scale_log2e;
  int32_t G, window, sinks, out_bf16;
  int32_t blocks, share, places;           // RowsPlan
};

__device__ __forceinline__ void put_row(const RowsAttend& c, int64_t row, int d4, f32x4 y) {
  if (c.out_bf16) *reinterpret_cast<u32x2*>(c.out + (row * kDim + d4) * 2) = u32x2{bf16_pack(y[0], y[1]), bf16_pack(y[2], y[3])};
  else *reinterpret_cast<f32x4*>(c.out + (row * kDim + d4) * 4) = y;
}

// Lanes l and l + 32 into one value, the same in both.
template <class Op>
__device__ __forceinline__ float halves_combine(float v, Op op) {
  const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return op(__uint_as_float(h[0]), __uint_as_float(h[1]));
}
__device__ __forceinline__ int wave_min_i32(int v) { return (int)(wave_min_u32((uint32_t)v ^ 0x80000000u) ^ 0x80000000u); }
__device__ __forceinline__ int wave_max_i32(int v) { return -wave_min_i32(-v); }

// Where row `row`'s 16 bytes `chunk` lie in a tile of rows of 256 bytes: sixteen rows' same chunk in sixteen places, and of four rows that follow one another
// neighbouring chunks too, so that neither way of reading meets a bank twice.
__device__ __forceinline__ int swizzle(int row) { return (row & 3) << 2 | ((row >> 2) & 3); }

// Keeps what a branch does in the branch (it would be done always, and taken or not, otherwise).
__device__ __forceinline__ void apart() { asm volatile(""); }
// What is worked out here is not put off until it is used.
template <class T>
__device__ __forceinline__ void here(T& x) { asm volatile("" : "+v"(x)); }
// Nothing moves from one side to the other.
__device__ __forceinline__ void fence() { __builtin_amdgcn_sched_barrier(0); }

__device__ const uint8_t kNothing[256] __attribute__((aligned(16))) = {};         // a row of zeros

typedef __attribute__((address_space(3))) uint8_t lds8;
__device__ __forceinline__ uint32_t lds_at(const void* p) { return (uint32_t)(uintptr_t)(const lds8*)p; }

// Sixteen bytes of each lane straight into LDS, side by side from `to` on.  The compiler does not know of these loads: told, it takes every read out of LDS for one that may have to
// wait for them, and waits.  They are waited for by hand (arrived()) before the barrier that lets others read.
__device__ __forceinline__ void load_to_lds(const uint8_t* from, uint32_t to) {
  to = (uint32_t)uniform_i32((int)to);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(to), "v"(from) : "memory");
}
__device__ __forceinline__ void load_to_lds(const uint8_t* base, uint32_t lane_at, uint32_t to) {
  to = (uint32_t)uniform_i32((int)to);
  const u64 at = (u64)base;
  base = (const uint8_t*)((u64)(uint32_t)uniform_i32((int)(at >> 32)) << 32 | (uint32_t)uniform_i32((int)at));
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(to), "v"(lane_at), "s"(base) : "memory");
}
__device__ __forceinline__ void arrived() { __builtin_amdgcn_s_waitcnt(0x0F70); }          // vmcnt(0)

__device__ __forceinline__ u32x4 read_row(uint32_t at, int more) { return *(const __attribute__((address_space(3))) u32x4*)((const lds8*)(uintptr_t)at + more); }
// Four rows of sixteen values, 8 bytes of a row each lane of sixteen, four lanes a row: the lane's column of them.
__device__ __forceinline__ s16x4 read_transposed(uint32_t at, int more) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)((lds8*)(uintptr_t)at + more));
}
__device__ __forceinline__ s16x8 beside(s16x4 a, s16x4 z) { return s16x8{a[0], a[1], a[2], a[3], z[0], z[1], z[2], z[3]}; }

// What a pair of floats leaves once its bf16 halves are taken off, one instruction each: the pair times (-1, 0) or (0, -1), added to the float; exact.  (The factors come out of registers: as constants
// the compiler makes one of both.)
struct Rest {
  uint32_t low, high;
  __device__ __forceinline__ Rest() : low(0xBF80u), high(0xBF800000u) { asm("" : "+s"(low), "+s"(high)); }
  __device__ __forceinline__ void operator()(uint32_t pair, float& a, float& z) const {
    a = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, low), a, false);
    z = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, high), z, false);
  }
};

// One workgroup of four wavefronts per piece: 32 WIDE rows (row = one query head of one of the call's rows of a sequence, heads of a KV head side by side) over some tiles
// of entries.  A tile's keys and values go through LDS, two tiles in turn, asked for one ahead; 8 bits become bf16 on the way, times their powers of two, which is exact.
//   logits   K Q^T by 32 x 32 x 16 products, rows = entries, columns = the wavefront's 32 rows, so that a row's maximum and sum are a lane's own but for one exchange of halves;
//   outputs  V^T P^T with the logits' registers as operand, entries in the order in which K Q^T leaves them, and values read out of LDS transposed (columns = rows again,
//            so that what shrinks them is the lane's own too).
// Weights go in as two bf16 terms (16 bits) for bf16 outputs, three for float outputs.  An entry that only some rows of the block see gives the others
// nothing, whatever its value: where something that is not finite comes out the piece is done again with the finite values alone, and rows that give others weight
// get NaN where those are.
template <bool E4M3, int WIDE, int TERMS>
__global__ __launch_bounds__(kThreads, WIDE == 1 ? 1 : 2) void paged_rows_kernel(Paged p, RowsAttend c) {
  constexpr int kDeep = kAttendWaves / WIDE, kUnit = 32 * kDeep, NU = WIDE == 4 ? 2 : 1, kRows = 32 * WIDE, kBuf = NU * kUnit * 256;
  constexpr int kLoads = kUnit / (E4M3 ? 32 : 16), kWords = kMaxDrafts / 32 + 3;
  __shared__ __align__(16) uint8_t s_tile[2][2][kBuf];          // keys, values; two buffers of NU units each
  __shared__ uint32_t s_see[kRows][kWords];
  __shared__ float s_m[kAttendWaves][32], s_l[kAttendWaves][32];
  __shared__ int s_odd;
  static_assert(sizeof s_tile >= kAttendWaves * 32 * kDim * 4, "the outputs go where the tiles were");

  const int tid = threadIdx.x, lane = tid & 63, wave = uniform_i32(tid >> 6), j = lane & 31, half = lane >> 5, wq = wave % WIDE, wk = wave / WIDE;
  const int64_t each = (int64_t)c.blocks * c.places, piece = rows_piece(blockIdx.x, c.units, each);
  if (piece < 0) return;
  const int u = uniform_i32((int)(piece / each)), k_in = uniform_i32((int)(piece - u * each)), part = uniform_i32(k_in / c.blocks), blk = c.blocks - 1 - (k_in - part * c.blocks);      // the last rows have the most to do
  const int b = uniform_i32(u / p.hkv), h = u - b * p.hkv;
  const int64_t block_index = (int64_t)u * c.blocks + blk;
  int bad = 0;
  p.length(b, bad);
  int64_t q_base;
  const RowSpan span = c.rows.span(b, uniform_i32(p.lengths[b]), p.max_length, q_base);
  if (span.bad) bad |= PAGED_BAD_LENGTH;
  const uint32_t r0 = (uint32_t)blk * kRows, n_rows = (uint32_t)uniform_i32(span.count) * (uint32_t)c.G;
  if (r0 >= n_rows) {
    if (part == 0 && tid == 0) {
      if (c.parts) c.parts[block_index] = 0;
      if (blk == 0) p.report(bad);
    }
    return;
  }
  const int first = uniform_i32(span.first), count = uniform_i32(span.count), t_lo = uniform_i32((int)(r0 / c.G)), t_hi = uniform_i32((int)((min(r0 + kRows, n_rows) - 1) / c.G));
  const uint32_t row = r0 + 32 * wq + j;
  const bool valid = row < n_rows;
  const int token = (int)((valid ? row : r0) / c.G), g = (int)((valid ? row : r0) - (uint32_t)token * c.G);

  // ---- which entries the lane's row sees: lo .. hi - 1, the first `sinks`, and of the call's rows those in s_see
  const int sinks = c.window ? c.sinks : 0;
  int position = first + token, hi = position + 1, oldest, end = first + t_hi + 1;
  if (c.tree) {
    const int words = (count + 63) >> 6;
    for (int t = t_lo + wave; t <= t_hi; t += kAttendWaves)
      for (int w = 0; w < kWords / 2 + 1; ++w) {
        const int at = 64 * w + lane;
        const u64 sees = w < words ? __ballot(at < count && c.tree[b * c.tree_seq + t * c.tree_row + at] != 0) : 0ull;
        if (lane < 2 && 2 * w + lane < kWords) s_see[t - t_lo][2 * w + lane] = (uint32_t)(sees >> 32 * lane);
      }
    __syncthreads();
    auto depth = [&](int t) {
      int n = 0;
      for (int w = 0; w < 2 * words; ++w) n += __popc(s_see[t - t_lo][w]);
      return n;
    };
    position = first + depth(token) - 1;
    hi = first;
    end = first + count;
    int least = INT32_MAX;
    for (int t = t_lo + lane; t <= t_hi; t += 64) least = min(least, first + depth(t) - 1);
    oldest = c.window ? max(wave_min_i32(least) - c.window + 1, 0) : 0;
  } else {
    oldest = c.window ? max(first + t_lo - c.window + 1, 0) : 0;
  }
  const int lo = c.window ? max(position - c.window + 1, 0) : 0;
  const int wave_hi = wave_min_i32(valid ? hi : INT32_MAX), wave_lo = wave_max_i32(valid ? lo : 0);       // what all of the wavefront's rows see
  oldest = uniform_i32(oldest);
  end = uniform_i32(end);

  RowTiles tiles = row_tiles(oldest, end, sinks, kUnit);
  tiles = {uniform_i32(tiles.sinks), uniform_i32(tiles.base), uniform_i32(tiles.count)};
  const int share = rows_share(tiles.count, c.share, c.places), parts = unit_parts(tiles.count, share);
  if (part == 0 && tid == 0 && c.parts) c.parts[block_index] = parts;
  if (part >= parts) return;
  const int n_first = uniform_i32(part_begin(tiles.count, parts, part)), n_last = uniform_i32(part_begin(tiles.count, parts, part + 1));

  bf16x8 q[8];
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    u32x4 x = {0u, 0u, 0u, 0u};
    if (valid) x = load16(c.rows.k + q_base + token * c.rows.row_stride + (h * c.G + g) * c.rows.head_stride + 2 * (16 * s + 8 * half));
    q[s] = __builtin_bit_cast(bf16x8, x);
  }
  f32x16 acc[4];
  float m_run, l_run;

  // ---- units' way into LDS: rows of 256 bytes, bf16 straight there, 8 bits through registers
  const int units = n_last - n_first;
  auto unit_at = [&](int i) CKV_INLINE { return tiles.tile(n_first + i) * kUnit; };
  auto seen = [&](int e) CKV_INLINE { return e < end && (e >= oldest || e < sinks); };
  int missing = 0;                               // a page that some row needs and that is not there
  // Where kPageSlots pages lie, a lane each: of the sequence's pages kPageSlots * window and on (page -1 where there is none, and the place of the pool's first).
  struct Known {
    int window = -1, page = -1;
    u64 at = 0ull;
  } k_known, v_known;
  u32x4 kr[E4M3 ? NU * kLoads : 1], vr[E4M3 ? NU * kLoads : 1];
  uint32_t ks[E4M3 ? NU * kLoads : 1], vs[E4M3 ? NU * kLoads : 1];
  const int r_in = E4M3 ? tid >> 3 : tid >> 4;   // the thread's row of those that a load takes
  const uint32_t lane_at = (uint32_t)((E4M3 ? r_in & 15 : r_in) * p.slot_stride + 16 * (E4M3 ? tid & 7 : (tid & 15) ^ swizzle(r_in)));
  const int shift = p.shift, page_mask = p.page_size() - 1, slot_stride = p.slot_stride;
  auto look_up = [&](int e0, const uint8_t* pool, Known& known) CKV_INLINE {
    const int w = (e0 >> shift) / kPageSlots;
    if (w == known.window) return;
    known.window = w;
    const int64_t logical = (int64_t)w * kPageSlots + lane, from = logical << shift, upto = from + page_mask + 1;
    const bool needed = logical < p.columns && from < end && (upto > oldest || from < sinks);
    const int page = needed ? p.table[(int64_t)b * p.table_stride + logical] : -1;
    const bool there = page_there(page, p.n_pages);
    if (needed && !there) bad |= PAGED_BAD_PAGE;
    missing |= __ballot(needed && !there) != 0ull;
    known.page = there ? page : -1;
    known.at = (u64)(pool + (there ? page : 0) * p.page_stride + h * p.head_stride);
  };
  // The unit's entries from e0 on.  ALL: every one is there and seen; otherwise those that no row of the block sees, or that have no page, come as zeros: whatever lies there times a weight of
  // nothing must be nothing.
  auto ask_side = [&](auto all_, int e0, const Known& known, uint32_t to, u32x4* rr, uint32_t* ss, int side) CKV_INLINE {
    constexpr bool ALL = decltype(all_)::value;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int e = e0 + (E4M3 ? 32 * i + 16 * (wave >> 1) : 16 * i), off = e & page_mask, slot = (e >> shift) & (kPageSlots - 1);
      const uint8_t* from = (const uint8_t*)readlane_u64(known.at, slot) + (uint32_t)(off * slot_stride);
      if constexpr (E4M3) {
        const int page = __builtin_amdgcn_readlane(known.page, slot);
        rr[i] = load16(from + lane_at);
        ss[i] = p.scales[max(page, 0) * p.scale_page_stride + h * p.scale_head_stride + 2 * (off + (r_in & 15)) + side];
        if (!ALL) {
          apart();
          if (page < 0 || !seen(e + (r_in & 15))) rr[i] = u32x4{0u, 0u, 0u, 0u}, ss[i] = 127u;
        }
      } else if (ALL) {
        load_to_lds(from, lane_at, to + (16 * i + 4 * wave) * 256);
      } else {
        const int page = __builtin_amdgcn_readlane(known.page, slot);
        load_to_lds(page >= 0 && seen(e + r_in) ? from + lane_at : kNothing + 16 * (tid & 15), to + (16 * i + 4 * wave) * 256);
      }
    }
  };
  const uint32_t k_lds = lds_at(&s_tile[0][0][0]), v_lds = lds_at(&s_tile[1][0][0]);
  // The n-th buffers: keys of units NU n + 1 and on, values of units NU n - 1 and on.
  auto ask = [&](int n, int buf) CKV_INLINE {
#pragma unroll 1
    for (int s = 0; s < NU; ++s) {
      const int k = NU * n + 1 + s, v = NU * n - 1 + s;
      const uint32_t to = buf * kBuf + s * kUnit * 256;
      auto side = [&](int unit, const uint8_t* pool, Known& known, uint32_t lds, u32x4* rr, uint32_t* ss, int which) CKV_INLINE {
        if (unit < 0 || unit >= units) return;
        const int e0 = unit_at(unit);
        look_up(e0, pool, known);
        ask_side(std::false_type(), e0, known, lds + to, rr, ss, which);
      };
      if constexpr (E4M3 && NU == 2) {            // registers by their names
        if (s == 0) {
          side(k, p.k, k_known, k_lds, kr, ks, 0);
          side(v, p.v, v_known, v_lds, vr, vs, 1);
        } else {
          side(k, p.k, k_known, k_lds, kr + kLoads, ks + kLoads, 0);
          side(v, p.v, v_known, v_lds, vr + kLoads, vs + kLoads, 1);
        }
      } else {
        side(k, p.k, k_known, k_lds, kr, ks, 0);
        side(v, p.v, v_known, v_lds, vr, vs, 1);
      }
    }
  };
  auto ask_steady = [&](int buf, int e0) CKV_INLINE {          // values from e0 on, keys two units behind them
#pragma unroll
    for (int s = 0; s < NU; ++s) {
      const uint32_t to = buf * kBuf + s * kUnit * 256;
      look_up(e0 + (2 + s) * kUnit, p.k, k_known);
      look_up(e0 + s * kUnit, p.v, v_known);
      ask_side(std::true_type(), e0 + (2 + s) * kUnit, k_known, k_lds + to, &kr[E4M3 ? s * kLoads : 0], &ks[E4M3 ? s * kLoads : 0], 0);
      ask_side(std::true_type(), e0 + s * kUnit, v_known, v_lds + to, &vr[E4M3 ? s * kLoads : 0], &vs[E4M3 ? s * kLoads : 0], 1);
    }
  };
  auto ask_next = [&](int n, int buf) CKV_INLINE {             // the one where it can be, or the other
    const int v = NU * n - 1, k = NU * n + NU, e0 = unit_at(v), e1 = e0 + (NU + 2) * kUnit - 1;
    if (k < units && unit_at(k) + kUnit - 1 == e1 && e0 >= oldest && e1 < end && !missing) ask_steady(buf, e0);
    else ask(n, buf);
  };
  auto put = [&](int buf) CKV_INLINE {
    if constexpr (E4M3) {
#pragma unroll
      for (int i = 0; i < NU * kLoads; ++i) {
        const float a = __uint_as_float(ks[i] << 23), z = __uint_as_float(vs[i] << 23);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int at = (32 * i + r_in) * 256 + (((2 * (tid & 7) + x) ^ swizzle(r_in)) << 4);
          *reinterpret_cast<u32x4*>(&s_tile[0][buf][at]) = values8(u32x2{kr[i][2 * x], kr[i][2 * x + 1]}, a);
          *reinterpret_cast<u32x4*>(&s_tile[1][buf][at]) = values8(u32x2{vr[i][2 * x], vr[i][2 * x + 1]}, z);
        }
      }
    } else {
      arrived();
    }
    __syncthreads();
  };

  // ---- one unit after another: the weights of one, the outputs of the one before, the logits of the one behind
  uint32_t ka[8], va[4], vz[4];                  // where a lane reads keys of 16 dimensions, and 4 + 4 values of 32
#pragma unroll
  for (int x = 0; x < 8; ++x) ka[x] = k_lds + (wk * 32 + j) * 256 + (((2 * x + half) ^ swizzle(j)) << 4);
  {
    const int l16 = lane & 15, at = (4 * half + (l16 >> 2)) * 256 + (l16 & 1) * 8 + (((((lane >> 4) & 1) * 2 + ((l16 >> 1) & 1)) ^ half) << 4);
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      va[d] = v_lds + wk * 32 * 256 + (at ^ (((l16 >> 2) ^ d) << 6));
      vz[d] = v_lds + wk * 32 * 256 + (at ^ (((l16 >> 2) ^ d) << 6) ^ 32) + 8 * 256;
    }
  }
  auto product = [](s16x8 a, u32x4 w, f32x16 c) CKV_INLINE { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, w), c, 0, 0, 0); };
  auto logits = [&](u32x4 k, int x, f32x16 c) CKV_INLINE { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k), q[x], c, 0, 0, 0); };
  f32x16 nought;
#pragma unroll
  for (int i = 0; i < 16; ++i) nought[i] = 0.f;
  // The running maximum follows the logits only where they outgrow it by 2^kSlack: any value serves as long as weights stay small numbers.  (A logit that is no number
  // leaves it as it is: its weight is none either.)
  constexpr float kSlack = 8.f;
  auto grown = [&](const f32x16& s) CKV_INLINE {
    float bm = max3(s[0], s[1], s[2]);
#pragma unroll
    for (int i = 3; i < 15; i += 2) bm = max3(bm, s[i], s[i + 1]);
    bm = halves_combine(max2(bm, s[15]), [](float x, float y) { return max2(x, y); }) * c.scale_log2e;
    return bm > m_run + kSlack ? bm : m_run;
  };
  auto shrink_by = [&](float f) CKV_INLINE {
    l_run *= f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[d][i] *= f;
  };
  // A unit in the middle of many, all of it seen by all of the wavefront's rows: products, and what else there is to do, in turn, so that neither waits for the other.
  auto steady = [&](auto at_, f32x16& s, f32x16& t, u32x4 (&w)[TERMS][2], u32x4 (&y)[TERMS][2]) CKV_INLINE {
    constexpr int at = decltype(at_)::value;
    u32x4 ko[2] = {read_row(ka[0], at), read_row(ka[1], at)};
    s16x4 vo[2][2] = {{read_transposed(va[0], at), read_transposed(vz[0], at)}, {read_transposed(va[0], at + 16 * 256), read_transposed(vz[0], at + 16 * 256)}};
    const Rest rest;
    const float m = grown(s), f = fast_exp2(m_run - m);
    float sum = 0.f, a = 0.f, z = 0.f;
    // the last term of a pair is taken a step later: what a sum of products leaves can be read only some instructions on
    auto last = [&](int n, float a, float z) CKV_INLINE {
      uint32_t pair = bf16_pack(a, z);
      here(pair);
      y[TERMS - 1][n >> 2][n & 3] = pair;
    };
    fence();
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      t = logits(ko[n & 1], n, n ? t : nought);
      const float a_last = a, z_last = z;
      a = fmaf(s[2 * n], c.scale_log2e, -m), z = fmaf(s[2 * n + 1], c.scale_log2e, -m);
      here(a);
      here(z);
      a = fast_exp2(a);
      here(a);
      if (n) last(n - 1, a_last, z_last);
      if (n < 6) ko[n & 1] = read_row(ka[n + 2], at);
      fence();
      const s16x8 v = beside(vo[n & 1][0], vo[n & 1][1]);
      acc[n >> 1] = product(v, w[0][n & 1], acc[n >> 1]);
      z = fast_exp2(z);
      here(z);
      sum += a;
      sum += z;
      here(sum);
      fence();
#pragma unroll
      for (int x = 1; x < TERMS; ++x) {
        acc[n >> 1] = product(v, w[x][n & 1], acc[n >> 1]);
        uint32_t pair = bf16_pack(a, z);
        here(pair);
        y[x - 1][n >> 2][n & 3] = pair;
        rest(pair, a, z);
        here(a);
        here(z);
        if (x == 1 && n < 6) {
          vo[n & 1][0] = read_transposed(va[(n + 2) >> 1], at + (n & 1) * 16 * 256);
          vo[n & 1][1] = read_transposed(vz[(n + 2) >> 1], at + (n & 1) * 16 * 256);
        }
        fence();
      }
    }
    last(7, a, z);
    if (__any(m > m_run)) {
      apart();
      shrink_by(f);
    }
    m_run = m;
    l_run += sum;
  };
  f32x16 s, t;
  u32x4 w[TERMS][2], y[TERMS][2];
  // Any unit.
  auto any = [&](int careful, int i, int at) CKV_INLINE {
    if (i >= 1 && i <= units) {
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        f32x16 wrong = nought;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          s16x8 v = beside(read_transposed(va[d] + at, x * 16 * 256), read_transposed(vz[d] + at, x * 16 * 256));
          if (careful) {
            apart();
            s16x8 ones;
            u32x4 weight;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const bool infinite = (v[e] & 0x7F80) == 0x7F80;
              ones[e] = infinite ? 0x3F80 : 0;
              v[e] = infinite ? 0 : v[e];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) weight[e] = (w[0][x][e] & 0x7FFFu ? 0x3F80u : 0u) | (w[0][x][e] & 0x7FFF0000u ? 0x3F800000u : 0u);
            wrong = product(ones, weight, wrong);
          }
#pragma unroll
          for (int n = 0; n < TERMS; ++n) acc[d] = product(v, w[n][x], acc[d]);
        }
        if (careful) {
          apart();
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (wrong[e] != 0.f) acc[d][e] = NAN;
        }
      }
    }
    if (i >= 0 && i < units) {
      const int e_first = unit_at(i) + wk * 32, e_last = e_first + 31;
      if (missing || e_last >= wave_hi || (e_first < wave_lo && e_last >= sinks)) {
        apart();
        uint32_t sees = 0u;
        if (valid) {
          sees = (uint32_t)bits_between(e_first, lo, hi) | (uint32_t)bits_between(e_first, 0, min(sinks, hi));
          if (c.tree && e_last >= first) {
            const uint32_t* bits = s_see[token - t_lo];
            const int from = e_first - first, word = max(from, 0) >> 5, by = max(from, 0) & 31;
            const uint32_t drafts = (uint32_t)(((u64)bits[word + 1] << 32 | bits[word]) >> by);
            sees |= from >= 0 ? drafts : drafts << -from;
          }
        }
        for (int x = 0; missing && x < 2; ++x) {
          const int col = (e_first + 16 * x) >> p.shift;
          if (col >= p.columns || !page_there(p.table[(int64_t)b * p.table_stride + col], p.n_pages)) sees &= ~(0xFFFFu << 16 * x);
        }
        sees >>= 4 * half;
#pragma unroll
        for (int x = 0; x < 16; ++x)
          if (!(sees >> (8 * (x >> 2) + (x & 3)) & 1u)) s[x] = -INFINITY;
      }
      const float m = grown(s);
      if (__any(m > m_run)) {
        apart();
        shrink_by(fast_exp2(m_run - m));
      }
      m_run = m;
      const Rest rest;
      float sum = 0.f;
#pragma unroll
      for (int n = 0; n < 8; ++n) {
        float a = fast_exp2(fmaf(s[2 * n], c.scale_log2e, -m)), z = fast_exp2(fmaf(s[2 * n + 1], c.scale_log2e, -m));
        sum += a;
        sum += z;
#pragma unroll
        for (int x = 0; x < TERMS; ++x) {
          w[x][n >> 2][n & 3] = bf16_pack(a, z);
          if (x + 1 < TERMS) rest(w[x][n >> 2][n & 3], a, z);
        }
      }
      l_run += sum;
    }
    if (i + 1 >= 0 && i + 1 < units) {
#pragma unroll
      for (int x = 0; x < 8; ++x) s = logits(read_row(ka[x] + at, 0), x, x ? s : nought);
    }
  };
  if (tid == 0) s_odd = 0;
  for (int careful = 0;; careful = 1) {
#pragma unroll
    for (int d = 0; d < 4; ++d) acc[d] = nought;
    m_run = kNoLogit, l_run = 0.f;
    const int n_end = units / NU;
    ask(-1, 1);
    put(1);
    for (int n = -1; n <= n_end;) {
      // 2 NU units from the n-th buffers' on, which are those of 0 and 1
      const int i = NU * n;
      if ((n & 1) == 0 && i >= 1 && i + 2 * NU < units && !(missing | careful)) {
        const int e0 = unit_at(i), e1 = e0 + 2 * NU * kUnit - 1;
        if (unit_at(i + 2 * NU - 1) + kUnit - 1 == e1 && e1 < wave_hi && e0 >= wave_lo) {
          ask_next(n + 1, 1);
          steady(std::integral_constant<int, 0>(), s, t, w, y);
          if constexpr (NU == 2) steady(std::integral_constant<int, kUnit * 256>(), t, s, y, w);
          put(1);
          if (missing) {            // a page of those just asked for
            apart();
            if constexpr (NU == 1) {
              s = t;
#pragma unroll
              for (int x = 0; x < TERMS; ++x) w[x][0] = y[x][0], w[x][1] = y[x][1];
            }
            ++n;
            continue;
          }
          ask_next(n + 2, 0);
          if constexpr (NU == 2) {
            steady(std::integral_constant<int, kBuf>(), s, t, w, y);
            steady(std::integral_constant<int, kBuf + kUnit * 256>(), t, s, y, w);
          } else {
            steady(std::integral_constant<int, kBuf>(), t, s, y, w);
          }
          put(0);
          n += 2;
          continue;
        }
      }
      const int buf = n & 1;
      if (n < n_end) ask(n + 1, buf ^ 1);
#pragma unroll 1
      for (int x = 0; x < NU; ++x) any(careful, i + x, buf * kBuf + x * kUnit * 256);
      if (n < n_end) put(buf ^ 1);
      ++n;
    }
    __syncthreads();
    // Once more with care where something that is no number came out: a value that only some rows see must not reach the others.
    if (careful) break;
    float nothing = 0.f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) nothing = fmaf(acc[d][i], 0.f, nothing);
    if (!(nothing == 0.f)) s_odd = 1;
    __syncthreads();
    if (!uniform_i32(s_odd)) break;
    k_known.window = v_known.window = -1;
  }

  // ---- the wavefronts' states into one
  l_run = halves_combine(l_run, [](float x, float y) { return x + y; });
  if (half == 0) s_m[wave][j] = m_run, s_l[wave][j] = l_run;
  float* s_o = reinterpret_cast<float*>(&s_tile[0][0][0]);          // [wave][row][128], chunks of four in another order in each row
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int a = 0; a < 4; ++a)
      *reinterpret_cast<f32x4*>(s_o + (wave * 32 + j) * kDim + 4 * ((8 * d + 2 * a + half) ^ j)) = f32x4{acc[d][4 * a], acc[d][4 * a + 1], acc[d][4 * a + 2], acc[d][4 * a + 3]};
  __syncthreads();
  const int64_t out_row = c.rows.starts ? c.rows.starts[b] : (int64_t)b * c.rows.rows;
  for (int x = tid; x < kRows * (kDim / 4); x += kThreads) {
    const int r = x >> 5, chunk = x & 31, in = r & 31;
    if (r0 + r >= n_rows) break;
    float M = kNoLogit, L = 0.f;
#pragma unroll
    for (int k = 0; k < kDeep; ++k) M = fmaxf(M, s_m[k * WIDE + (r >> 5)][in]);
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kDeep; ++k) {
      const int w = k * WIDE + (r >> 5);
      const float f = fast_exp2(s_m[w][in] - M);
      L += s_l[w][in] * f;
      y += *reinterpret_cast<const f32x4*>(s_o + (w * 32 + in) * kDim + 4 * (chunk ^ in)) * f;
    }
    if (parts > 1) {
      const int64_t at = (block_index * c.places + part) * kRows + r;
      *reinterpret_cast<f32x4*>(c.partial + at * kDim + 4 * chunk) = y;
      if (chunk == 0) c.ml[2 * at] = M, c.ml[2 * at + 1] = L;
    } else {
      const int t = (int)((r0 + r) / c.G);
      const int64_t to = (out_row + t) * (c.G * p.hkv) + h * c.G + (int)(r0 + r - (uint32_t)t * c.G);
      put_row(c, to, 4 * chunk, L != 0.f ? y * (1.f / L) : f32x4{0.f, 0.f, 0.f, 0.f});
      if (chunk == 0 && c.lse) c.lse[to] = natural(M, L);
    }
  }
  p.report(bad);
}

// Joins the pieces of blocks of rows that have several: 32 threads a row, four dimensions each.
constexpr int kRowsJoined = 8;
template <int WIDE>
__global__ __launch_bounds__(32 * kRowsJoined) void paged_rows_join_kernel(Paged p, RowsAttend c) {
  constexpr int kRows = 32 * WIDE;
  const int64_t block_index = blockIdx.x;
  const int parts = c.parts[block_index];
  if (parts <= 1) return;
  const int u = (int)(block_index / c.blocks), blk = (int)(block_index - (int64_t)u * c.blocks), b = u / p.hkv, h = u - b * p.hkv;
  int64_t base;
  const RowSpan span = c.rows.span(b, p.lengths[b], p.max_length, base);
  const int in = blockIdx.y * kRowsJoined + (threadIdx.x >> 5), d4 = 4 * (threadIdx.x & 31);
  const uint32_t row = (uint32_t)blk * kRows + in;
  if (row >= (uint32_t)span.count * (uint32_t)c.G) return;
  float M = kNoLogit, L = 0.f;
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < parts; ++i) {
    const int64_t at = (block_index * c.places + i) * kRows + in;
    const f32x2 st = *reinterpret_cast<const f32x2*>(c.ml + 2 * at);
    const f32x4 x = *reinterpret_cast<const f32x4*>(c.partial + at * kDim + d4);
    const float m = fmaxf(M, st[0]), old = fast_exp2(M - m), now = fast_exp2(st[0] - m);
    M = m;
    L = L * old + st[1] * now;
    y = y * old + x * now;
  }
  const int t = (int)(row / c.G);
  const int64_t to = ((c.rows.starts ? c.rows.starts[b] : (int64_t)b * c.rows.rows) + t) * (c.G * p.hkv) + h * c.G + (int)(row - (uint32_t)t * c.G);
  put_row(c, to, d4, L != 0.f ? y * (1.f / L) : f32x4{0.f, 0.f, 0.f, 0.f});
  if (d4 == 0 && c.lse) c.lse[to] = natural(M, L);
}

}  // namespace ckv
