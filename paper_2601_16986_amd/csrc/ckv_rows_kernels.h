// Device code of attention of several rows per sequence over a cache in pages: each row over itself and what comes before it, all of it or a window with a few first entries,
// or, where rows are drafted tokens, over what comes before all of them and those that its mask names.
#pragma once
#include "ckv_paged_device.h"
#include "ckv_rows.h"

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

// What a block of rows sees of its sequence.
struct Block {
  int b, h, first, count, t_lo, t_hi;      // the call's rows of the sequence; the block's first and last of them
  uint32_t r0, rows;                       // the block's first (row, head); all of the sequence's
  int64_t q_base, out_row;
};

// One workgroup of four wavefronts per piece: 32 WIDE rows (row = one query head of one of the call's rows of a sequence, heads of a KV head side by side) over some tiles
// of entries.  A tile's keys and values go through LDS, two tiles in turn, asked for one ahead; 8 bits become bf16 on the way, times their powers of two, which is exact.
//   logits   K Q^T by 32 x 32 x 16 products, rows = entries, columns = the wavefront's 32 rows, so that a row's maximum and sum are a lane's own but for one exchange of halves;
//   outputs  V^T P^T with the logits' registers as operand, entries in the order in which K Q^T leaves them, and values read out of LDS transposed (columns = rows again,
//            so that what shrinks them is the lane's own too).
// Weights go in as two bf16 terms (16 bits) for bf16 outputs, three for float outputs.  An entry that only some rows of the block see gives the others
// nothing, whatever its value: of values that are not finite the finite rest is used, and rows that give them weight get NaN where they are.
template <bool E4M3, int WIDE, int TERMS>
__global__ __launch_bounds__(kThreads, WIDE == 1 ? 1 : 2) void paged_rows_kernel(Paged p, RowsAttend c) {
  constexpr int kKeys = WIDE == 1 ? 2 * kTile : kTile, kDeep = kAttendWaves / WIDE, NB = kKeys / 32 / kDeep, kRows = 32 * WIDE, kGroups = kKeys / 16;
  constexpr int kLoads = E4M3 ? kKeys / 32 : kKeys / 16, kWords = kMaxDrafts / 32 + 3;
  __shared__ __align__(16) uint8_t s_tile[2][2][kKeys * 256];
  __shared__ uint32_t s_see[kRows][kWords];
  __shared__ float s_m[kAttendWaves][32], s_l[kAttendWaves][32];
  __shared__ int s_odd[2];
  static_assert(sizeof s_tile >= kAttendWaves * 32 * kDim * 4, "the outputs go where the tiles were");

  const int tid = threadIdx.x, lane = tid & 63, wave = uniform_i32(tid >> 6), j = lane & 31, half = lane >> 5, wq = wave % WIDE, wk = wave / WIDE;
  const int64_t each = (int64_t)c.blocks * c.places, piece = rows_piece(blockIdx.x, c.units, each);
  if (piece < 0) return;
  const int u = (int)(piece / each), k_in = (int)(piece - u * each), part = k_in / c.blocks, blk = c.blocks - 1 - (k_in - part * c.blocks);      // the last rows have the most to do
  const int b = u / p.hkv, h = u - b * p.hkv;
  const int64_t block_index = (int64_t)u * c.blocks + blk;
  int bad = 0;
  p.length(b, bad);
  int64_t q_base;
  const RowSpan span = c.rows.span(b, uniform_i32(p.lengths[b]), p.max_length, q_base);
  if (span.bad) bad |= PAGED_BAD_LENGTH;
  const uint32_t r0 = (uint32_t)blk * kRows, n_rows = (uint32_t)span.count * (uint32_t)c.G;
  if (r0 >= n_rows) {
    if (part == 0 && tid == 0) {
      if (c.parts) c.parts[block_index] = 0;
      if (blk == 0) p.report(bad);
    }
    return;
  }
  const int first = uniform_i32(span.first), t_lo = (int)(r0 / c.G), t_hi = (int)((min(r0 + kRows, n_rows) - 1) / c.G);
  const uint32_t row = r0 + 32 * wq + j;
  const bool valid = row < n_rows;
  const int token = (int)((valid ? row : r0) / c.G), g = (int)((valid ? row : r0) - (uint32_t)token * c.G);

  // ---- which entries the lane's row sees: lo .. hi - 1, the first `sinks`, and of the call's rows those in s_see
  const int sinks = c.window ? c.sinks : 0;
  int position = first + token, hi = position + 1, oldest, end = first + t_hi + 1;
  if (c.tree) {
    const int words = (span.count + 63) >> 6;
    for (int t = t_lo + wave; t <= t_hi; t += kAttendWaves)
      for (int w = 0; w < kWords / 2 + 1; ++w) {
        const int at = 64 * w + lane;
        const u64 sees = w < words ? __ballot(at < span.count && c.tree[b * c.tree_seq + t * c.tree_row + at] != 0) : 0ull;
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
    end = first + span.count;
    int least = INT32_MAX;
    for (int t = t_lo + lane; t <= t_hi; t += 64) least = min(least, first + depth(t) - 1);
    oldest = c.window ? max(wave_min_i32(least) - c.window + 1, 0) : 0;
  } else {
    oldest = c.window ? max(first + t_lo - c.window + 1, 0) : 0;
  }
  const int lo = c.window ? max(position - c.window + 1, 0) : 0;
  const int wave_hi = wave_min_i32(valid ? hi : INT32_MAX), wave_lo = wave_max_i32(valid ? lo : 0);       // what all of the wavefront's rows see

  const RowTiles tiles = row_tiles(oldest, end, sinks, kKeys);
  const int share = rows_share(tiles.count, c.share, c.places), parts = unit_parts(tiles.count, share);
  if (part == 0 && tid == 0 && c.parts) c.parts[block_index] = parts;
  if (part >= parts) return;
  const int n_first = part_begin(tiles.count, parts, part), n_last = part_begin(tiles.count, parts, part + 1);

  bf16x8 q[8];
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    u32x4 x = {0u, 0u, 0u, 0u};
    if (valid) x = load16(c.rows.k + q_base + token * c.rows.row_stride + (h * c.G + g) * c.rows.head_stride + 2 * (16 * s + 8 * half));
    q[s] = __builtin_bit_cast(bf16x8, x);
  }
  f32x16 acc[4];
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
  float m_run = kNoLogit, l_run = 0.f;

  // ---- a tile's way into LDS
  int page = 0, there = 0, window = -1;          // whereabouts of kPageSlots pages, a lane each
  u32x4 kr[kLoads], vr[kLoads];
  uint32_t sc[E4M3 ? kLoads : 1];
  auto seen = [&](int e) { return e < end && (e >= oldest || e < sinks); };
  auto look_up = [&]() {
    const int64_t logical = (int64_t)window * kPageSlots + lane, from = logical << p.shift, upto = from + p.page_size();
    const bool needed = logical < p.columns && from < end && (upto > oldest || from < sinks);
    page = needed ? p.table[(int64_t)b * p.table_stride + logical] : 0;
    there = needed && page_there(page, p.n_pages);
    if (needed && !there) bad |= PAGED_BAD_PAGE;
  };
  auto ask = [&](int e0, uint32_t& ok) {
    const int col = e0 >> p.shift;
    if (col / kPageSlots != window) {
      window = col / kPageSlots;
      look_up();
    }
    ok = 0u;
#pragma unroll
    for (int i = 0; i < kGroups; ++i) ok |= (uint32_t)__builtin_amdgcn_readlane(there, ((e0 + 16 * i) >> p.shift) & (kPageSlots - 1)) << i;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int group = E4M3 ? 2 * i + (wave >> 1) : i, e = e0 + 16 * group, off = e & (p.page_size() - 1);
      const int64_t pg = __builtin_amdgcn_readlane(page, (e >> p.shift) & (kPageSlots - 1));
      kr[i] = vr[i] = u32x4{0u, 0u, 0u, 0u};
      if constexpr (E4M3) sc[i] = 0u;
      if (!(ok >> group & 1u)) continue;
      if constexpr (E4M3) {
        const int r = (tid >> 3) & 15;
        const int64_t from = pg * p.page_stride + h * p.head_stride + (int64_t)(off + r) * p.slot_stride + 16 * (tid & 7);
        kr[i] = load16(p.k + from);
        vr[i] = load16(p.v + from);
        sc[i] = *reinterpret_cast<const uint16_t*>(p.scales + pg * p.scale_page_stride + h * p.scale_head_stride + 2 * (off + r));
      } else {
        const int64_t from = pg * p.page_stride + h * p.head_stride + (int64_t)(off + (tid >> 4)) * p.slot_stride + 16 * (tid & 15);
        kr[i] = load16(p.k + from);
        vr[i] = load16(p.v + from);
      }
    }
  };
  auto put = [&](int buf, int e0, int n) {
    const bool all = seen(e0) && seen(e0 + kKeys - 1) && (e0 >= oldest || e0 + kKeys <= sinks);
    uint32_t most = 0u;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = E4M3 ? 32 * i + (tid >> 3) : 16 * i + (tid >> 4);
      if (!all && !seen(e0 + r)) {
        vr[i] = u32x4{0u, 0u, 0u, 0u};
        if constexpr (E4M3) sc[i] &= 0xFFu;
      }
      uint8_t* to_k = &s_tile[buf][0][r * 256];
      uint8_t* to_v = &s_tile[buf][1][r * 256];
      if constexpr (E4M3) {
        const float ks = __uint_as_float((sc[i] & 0xFFu) << 23), vs = __uint_as_float((sc[i] >> 8) << 23);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int at = ((2 * (tid & 7) + x) ^ swizzle(r)) << 4;
          const u32x4 v = values8(u32x2{vr[i][2 * x], vr[i][2 * x + 1]}, vs);
          *reinterpret_cast<u32x4*>(to_k + at) = values8(u32x2{kr[i][2 * x], kr[i][2 * x + 1]}, ks);
          *reinterpret_cast<u32x4*>(to_v + at) = v;
#pragma unroll
          for (int y = 0; y < 4; ++y) most = pk_max_u16(most, v[y] & 0x7FFF7FFFu);
        }
      } else {
        const int at = ((tid & 15) ^ swizzle(r)) << 4;
        *reinterpret_cast<u32x4*>(to_k + at) = kr[i];
        *reinterpret_cast<u32x4*>(to_v + at) = vr[i];
#pragma unroll
        for (int y = 0; y < 4; ++y) most = pk_max_u16(most, vr[i][y] & 0x7FFF7FFFu);
      }
    }
    if ((most & 0xFFFFu) >= kInfinite || most >> 16 >= kInfinite) s_odd[buf] = n + 1;
  };

  if (tid < 2) s_odd[tid] = 0;
  uint32_t ok, ok_next = 0u;
  int e0 = tiles.tile(n_first) * kKeys, e_next = 0;
  ask(e0, ok);
  __syncthreads();
  put(0, e0, n_first);
  __syncthreads();
  int buf = 0;
  const int l16 = lane & 15, sw = swizzle(j);
  const int v_base = (4 * half + (l16 >> 2)) * 256 + (l16 & 1) * 8 + (((((lane >> 4) & 1) * 2 + ((l16 >> 1) & 1)) ^ half) << 4);
  for (int n = n_first; n < n_last; ++n) {
    if (n + 1 < n_last) {
      e_next = tiles.tile(n + 1) * kKeys;
      ask(e_next, ok_next);
    }
    const int e_in = wk * NB * 32, e_first = e0 + e_in, e_last = e_first + 32 * NB - 1;
    const uint32_t mine = ok >> (e_in >> 4) & ((1u << 2 * NB) - 1);
    const bool full = mine == (1u << 2 * NB) - 1 && e_last < wave_hi && (e_first >= wave_lo || e_last < sinks);
    u64 sees = 0ull;
    if (!full) {
      if (valid) {
        sees = bits_between(e_first, lo, hi) | bits_between(e_first, 0, min(sinks, hi));
        if (c.tree && e_last >= first) {
          const uint32_t* s = s_see[token - t_lo];
          const int at = e_first - first, w = max(at, 0) >> 5, by = max(at, 0) & 31;
          const u64 x = (u64)s[w + 1] << 32 | s[w], y = s[w + 2];
          const u64 drafts = by ? x >> by | y << (64 - by) : x;
          sees |= at >= 0 ? drafts : drafts << -at;
        }
      }
#pragma unroll
      for (int i = 0; i < 2 * NB; ++i)
        if (!(mine >> i & 1u)) sees &= ~(0xFFFFull << 16 * i);
      if (NB == 1) sees &= 0xFFFFFFFFull;
    }
    if (full || __any(sees != 0ull)) {
      const uint8_t* tk = &s_tile[buf][0][(e_in + j) * 256];
      f32x16 s[NB];
#pragma unroll
      for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = 0.f;
#pragma unroll
      for (int x = 0; x < 8; ++x)
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) {
          const u32x4 k = *reinterpret_cast<const u32x4*>(tk + kb * 32 * 256 + (((2 * x + half) ^ sw) << 4));
          s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k), q[x], s[kb], 0, 0, 0);
        }
      if (!full) {
        const u64 mask = sees >> 4 * half;
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (!(mask >> (32 * kb + 8 * (i >> 2) + (i & 3)) & 1ull)) s[kb][i] = -INFINITY;
      }
      // ---- softmax with a running maximum
      float bm = s[0][0];
#pragma unroll
      for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) bm = fmaxf(bm, s[kb][i]);
      bm = halves_combine(bm, [](float x, float y) { return fmaxf(x, y); }) * c.scale_log2e;
      if (__any(bm > m_run)) {
        const float m_new = fmaxf(m_run, bm), shrink = fast_exp2(m_run - m_new);
        m_run = m_new;
        l_run *= shrink;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[d][i] *= shrink;
      }
      bf16x8 w[TERMS][2 * NB];
      float sum = 0.f;                 // of the tile first, so that few additions follow one another
#pragma unroll
      for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float rest = fast_exp2(fmaf(s[kb][i], c.scale_log2e, -m_run));
          sum += rest;
#pragma unroll
          for (int t = 0; t < TERMS; ++t) {
            w[t][2 * kb + (i >> 3)][i & 7] = (__bf16)rest;
            rest -= (float)w[t][2 * kb + (i >> 3)][i & 7];
          }
        }
      l_run += sum;
      // ---- weights times values
      const bool odd = s_odd[buf] == n + 1;
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const uint8_t* tv = &s_tile[buf][1][e_in * 256 + (v_base ^ (((l16 >> 2) ^ d) << 6))];
        f32x16 wrong;
#pragma unroll
        for (int x = 0; x < 2 * NB; ++x) {
          typedef __attribute__((address_space(3))) s16x4* lds4;
          const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(tv + x * 16 * 256));
          const s16x4 z = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(uint8_t*)(&s_tile[buf][1][e_in * 256 + ((v_base ^ (((l16 >> 2) ^ d) << 6)) ^ 32)] + (x * 16 + 8) * 256));
          s16x8 v = {a[0], a[1], a[2], a[3], z[0], z[1], z[2], z[3]};
          if (odd) {
            s16x8 ones, weight;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const bool infinite = (v[i] & 0x7F80) == 0x7F80;
              ones[i] = infinite ? 0x3F80 : 0;
              weight[i] = (float)w[0][x][i] != 0.f ? 0x3F80 : 0;
              v[i] = infinite ? 0 : v[i];
            }
            if (x == 0)
#pragma unroll
              for (int i = 0; i < 16; ++i) wrong[i] = 0.f;
            wrong = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, ones), __builtin_bit_cast(bf16x8, weight), wrong, 0, 0, 0);
          }
#pragma unroll
          for (int t = 0; t < TERMS; ++t) acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), w[t][x], acc[d], 0, 0, 0);
        }
        if (odd)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (wrong[i] != 0.f) acc[d][i] = NAN;
      }
    }
    if (n + 1 < n_last) put(buf ^ 1, e_next, n + 1);
    __syncthreads();
    buf ^= 1;
    e0 = e_next;
    ok = ok_next;
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
