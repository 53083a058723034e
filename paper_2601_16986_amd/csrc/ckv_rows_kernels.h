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
  int32_t* parts;            // [unit][block][2]: pieces that its blocks fall into, and how far behind the first piece behind any places those behind its own begin
  int64_t tree_seq, tree_row;
  int64_t units;
  float scale_log2e;
  int32_t G, window, sinks, out_bf16;
  int32_t blocks, least, places, workers, more;      // RowsPlan
  int32_t grid;              // MORE: workgroups before those for pieces behind their block's places
  int32_t* cut;              // MORE: paged_rows_cut_kernel's
  float lower;               // lowered_by(): what weights are multiplied by where sums would be infinite
};

struct RowsCall {
  Paged p;
  RowsAttend c;
};
// The kernel's arguments once more, from memory: what is only used now and then does not stay in scalar registers, of which the inner loop needs all (with the arguments in them it kept others
// in vector registers' lanes, 470 moves a step).
__device__ __forceinline__ const __attribute__((address_space(4))) RowsCall* args() {
  auto a = (const __attribute__((address_space(4))) RowsCall*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(a));
  return a;
}

__device__ __forceinline__ void put_row(uint8_t* out, bool bf16, int64_t row, int d4, f32x4 y) {
  if (bf16) *reinterpret_cast<u32x2*>(out + (row * kDim + d4) * 2) = u32x2{bf16_pack(y[0], y[1]), bf16_pack(y[2], y[3])};
  else *reinterpret_cast<f32x4*>(out + (row * kDim + d4) * 4) = y;
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
__device__ __forceinline__ void here_scalar(int& x) { asm volatile("" : "+s"(x)); }
// Nothing moves from one side to the other.
__device__ __forceinline__ void fence() { __builtin_amdgcn_sched_barrier(0); }

__device__ const uint8_t kNothing[256] __attribute__((aligned(16))) = {};         // a row of zeros

typedef __attribute__((address_space(3))) uint8_t lds8;
__device__ __forceinline__ uint32_t lds_at(const void* p) { return (uint32_t)(uintptr_t)(const lds8*)p; }

__device__ __forceinline__ const uint8_t* uniform_at(const uint8_t* p) {
  const u64 at = (u64)p;
  return (const uint8_t*)((u64)(uint32_t)uniform_i32((int)(at >> 32)) << 32 | (uint32_t)uniform_i32((int)at));
}

// Sixteen bytes of each lane straight into LDS, side by side from `to` on.  The compiler does not know of these loads: told, it takes every read out of LDS for one that may have to
// wait for them, and waits.  They are waited for by hand (arrived()) before the barrier that lets others read.
__device__ __forceinline__ void load_to_lds(const uint8_t* from, uint32_t to) {
  to = (uint32_t)uniform_i32((int)to);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(to), "v"(from) : "memory", "m0");
}
__device__ __forceinline__ void load_to_lds(const uint8_t* base, uint32_t lane_at, uint32_t to) {
  to = (uint32_t)uniform_i32((int)to);
  base = uniform_at(base);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(to), "v"(lane_at), "s"(base) : "memory", "m0");
}
// What lies `more` bytes behind `base`, which is global memory: taken for any memory its load would be waited for as reads of LDS are, by those that follow.
template <class T>
__device__ __forceinline__ T global_at(u64 base, uint32_t more) { return *(const __attribute__((address_space(1))) T*)(base + more); }
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

// What a sequence's rows are worked out from, asked for with no branch between, so that all of it comes at once.
struct Told {
  int length, first, start, stop;
};
__device__ __forceinline__ Told told(const Paged& p, const Rows& r, int b) {
  const int32_t *first = r.first ? r.first : p.lengths, *starts = r.starts ? r.starts : p.lengths;
  return {p.lengths[b], first[b], starts[b], starts[r.starts ? b + 1 : b]};
}

// Blocks of rows that a sequence has for a KV head, and tiles of its longest.
struct Have {
  int blocks, tiles;
};
__device__ __forceinline__ Have have_of(const Paged& p, const RowsAttend& c, int block_rows, int size, const Told& t) {
  const RowSpan s = c.rows.span(t.length, t.first, t.start, t.stop, p.max_length);
  if (s.count == 0) return Have{0, 0};
  const int end = s.first + s.count, oldest = c.window ? max(s.first + (c.tree ? 0 : max(s.count - block_rows / c.G, 0)) - c.window, 0) : 0;
  return Have{(int)(((int64_t)s.count * c.G + block_rows - 1) / block_rows), row_tiles(oldest, end, c.window ? c.sinks : 0, size).count};
}

// rows_cut by the lengths as they are.  Lanes add up their share of the sequences (mine: the first of them).
__device__ __forceinline__ int even_share(const Paged& p, const RowsAttend& c, int block_rows, int size, int lane, const Told& mine) {
  const int per_lane = (p.batch + 63) >> 6, b0 = lane * per_lane;
  Have one = {0, 0};
  if (b0 < p.batch) one = have_of(p, c, block_rows, size, mine);
  auto sum = [&](auto count) {                     // over the sequences' blocks of rows
    float all = (float)one.blocks * count((float)one.tiles);
    for (int b = b0 + 1; b < b0 + per_lane && b < p.batch; ++b) {
      const Have more = have_of(p, c, block_rows, size, told(p, c.rows, b));
      all += (float)more.blocks * count((float)more.tiles);
    }
    return wave_sum_f32(all) * p.hkv;
  };
  float longest = (float)one.tiles;
  for (int b = b0 + 1; b < b0 + per_lane && b < p.batch; ++b) longest = fmaxf(longest, (float)have_of(p, c, block_rows, size, told(p, c.rows, b)).tiles);
  longest = __uint_as_float(~wave_min_u32(~__float_as_uint(longest)));
  const RowsCost cost = {block_rows, c.workers};
  return rows_cut(cost, c.least, c.places, true, 6, longest, sum);
}

// The same, once for a call whose blocks may have more pieces than places: cut[0] = tiles of a piece, cut[1 + b] = pieces behind their blocks' places of the sequences before b, numbered by sequence,
// KV head, block and piece; cut[1 + batch] all of them.  One workgroup, its threads adding up sequences side by side; three trips to memory and a dozen sums over the workgroup, 5 us.  (Every workgroup of the attention for itself, as
// without such pieces: 300 sequences of 8 drafts over 500 entries 242 us where they now take 164.)
constexpr int kCutThreads = 512;
template <int WIDE>
__global__ __launch_bounds__(kCutThreads) void paged_rows_cut_kernel(RowsCall call) {
  const Paged& p = call.p;
  const RowsAttend& c = call.c;
  constexpr int kRows = 32 * WIDE, kUnit = 32 * (kAttendWaves / WIDE), kWaves = kCutThreads / 64;
  __shared__ float s_sum[2][kWaves];
  __shared__ int s_upto[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto have = [&](int b) { return have_of(p, c, kRows, kUnit, told(p, c.rows, b)); };
  constexpr int kHeld = 4;                         // of a thread's sequences in registers
  Have held[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) held[i] = tid + i * kCutThreads < p.batch ? have(tid + i * kCutThreads) : Have{0, 0};
  auto each = [&](auto what) {                     // of the thread's sequences
#pragma unroll
    for (int i = 0; i < kHeld; ++i) what(held[i]);
    for (int b = tid + kHeld * kCutThreads; b < p.batch; b += kCutThreads) what(have(b));
  };
  int turn = 0;
  auto over = [&](float mine, auto of_wave, auto op) {
    mine = of_wave(mine);
    turn ^= 1;                                     // (the sums of the one before may still be read)
    if (lane == 0) s_sum[turn][wave] = mine;
    __syncthreads();
    float all = s_sum[turn][0];
    for (int w = 1; w < kWaves; ++w) all = op(all, s_sum[turn][w]);
    return all;
  };
  auto sum = [&](auto count) {
    float all = 0.f;
    each([&](Have h) { all += (float)h.blocks * count((float)h.tiles); });
    return over(all, [](float x) { return wave_sum_f32(x); }, [](float x, float y) { return x + y; }) * p.hkv;
  };
  float longest = 0.f;
  each([&](Have h) { longest = fmaxf(longest, (float)h.tiles); });
  longest = over(longest, [](float x) { return __uint_as_float(~wave_min_u32(~__float_as_uint(x))); }, [](float x, float y) { return fmaxf(x, y); });
  const RowsCost cost = {kRows, c.workers};
  int share = rows_cut(cost, c.least, c.places, false, kMorePieces, longest, sum);
  // never more than there are workgroups for: by floats so that they can be counted, then as they are
  const float behind = sum([&](float tiles) { return (float)rows_behind((int)tiles, share, c.places); });
  if (!(behind <= 2.f * (float)c.more)) share = INT32_MAX;
  for (;;) {
    int begun = 0;
    for (int b0 = 0; b0 < p.batch; b0 += kCutThreads) {
      const int b = b0 + tid;
      const Have mine = b0 == 0 ? held[0] : b < p.batch ? have(b) : Have{0, 0};
      const int own = p.hkv * mine.blocks * rows_behind(mine.tiles, share, c.places), upto = wave_scan_i32(own, lane);
      if (lane == 63) s_upto[wave] = upto;
      __syncthreads();
      int before = begun;
      for (int w = 0; w < kWaves; ++w) {
        before += w < wave ? s_upto[w] : 0;
        begun += s_upto[w];
      }
      if (b < p.batch) c.cut[1 + b] = before + upto - own;
      __syncthreads();
    }
    if (tid == 0) c.cut[0] = share, c.cut[1 + p.batch] = begun;
    if (begun <= c.more) return;
    share = INT32_MAX;
  }
}

// One workgroup of four wavefronts per piece: 32 WIDE rows (row = one query head of one of the call's rows of a sequence, heads of a KV head side by side) over some tiles
// of entries.  A tile's keys and values go through LDS, two tiles in turn, asked for one ahead; 8 bits become bf16 on the way, times their powers of two, which is exact.
//   logits   K Q^T by 32 x 32 x 16 products, rows = entries, columns = the wavefront's 32 rows, so that a row's maximum and sum are a lane's own but for one exchange of halves;
//   outputs  V^T P^T with the logits' registers as operand, entries in the order in which K Q^T leaves them, and values read out of LDS transposed (columns = rows again,
//            so that what shrinks them is the lane's own too).
// Weights go in as three bf16 terms, which hold the 24 bits of a float: 32 products for 32 entries where one term would need 16.  (Two terms, 16 bits, take a fifth less time, prompts below 1.44 ms and drafts 245 us where
// three take 1.81 and 290, and leave outputs that nearly cancel off by up to 2^-17 of their terms: of 8388608 bf16 outputs over up to 9350 entries 20920 then round the other way than the exact ones, 3102 with three
// terms, 7017 in float arithmetic throughout.)  An entry that only some rows of the block see gives the others
// nothing, whatever its value: where something that is not finite comes out the piece is done again with the finite values alone, and rows that give others weight
// get NaN where those are.  Where finite values add up to 2^115 it is done once more with lowered weights (lowered_by), whose sums stay finite; the sum of weights, which is not lowered, then has a sign
// for the join.  No vector register goes to scratch; 67 to
// 98 scalar ones lie in lanes of vector registers, moved there once (104 to 138, and with 8 bits 16 vector registers in scratch, where the ways that a piece is done again held what they need from the beginning on: 8 drafts of 4
// short sequences 22.4 us, now 21.4).
// What bounds it: long pieces of many rows by what moves, in LDS's time and in power: each wavefront reads all keys and values out of LDS for its 32 rows, 16 KB for the 32 products of 32 entries, beside the
// entries that come in.  A copy that reads nothing out of LDS takes 19 % less, one that loads no entries 16 % less, one without both 25 % (at a higher clock, too), which is what the products take; reads
// asked for a turn earlier change nothing, so it is not their latency; the exponentials and splitting of weights fit between
// products (3 of them 101 cycles, with all that goes with them 122; two exponentials 29, a pair packed 11, a remainder 8).  Prompts of 2 sequences of 8192, 40 heads, window 4096, bf16 1.80 to 1.88 ms from one card to the next, 1032 GFLOP at 570 TFLOP/s
// (1140 counting the three terms; a large product reaches 1250), 59 % of cycles in products, no bank of LDS met twice; the clock falls to 1.9 .. 2.0 GHz under it.  8 bits cost the conversion, which every block of rows does for itself, and a quarter
// of LDS's active cycles are banks met twice as it is written (8.7 M of 35 M): 48 rows of 40 heads over 131072 entries 285 to 310 us, 440 TFLOP/s (890), 48 % of cycles in products; copies without reads, loads and both 13, 16 and 20 % less; parts of
// prompts of many sequences 41 %, and 9, 11 and 16 % less.
// Short pieces are bound by what comes one after another: a piece's beginning and end take 30000 cycles (lengths, mask, table, first entries, outputs), a tile of 128 rows by 32 entries 2400 alone and 3700 beside
// another workgroup.
// Built, measured (with two terms) and not kept: a step's loads between its products (25 drafts in a window of 1024 55 us instead of 52, prompts no faster), a higher priority for wavefronts that load (the same), 32 rows a workgroup with
// 128 entries at once (128 KB of LDS: 8 bits 108 us for 8 rows of 4 heads over 4096 entries of 32 sequences where blocks of 64 rows with idle wavefronts take 83; bf16 113 and 118), 8 bits written to LDS
// in another order of rows, the next logits a turn early with their largest value beside the last outputs (both the same).
template <bool E4M3, int WIDE, bool MORE>
__global__ __launch_bounds__(kThreads, 2) void paged_rows_kernel(RowsCall call) {
  const Paged& p = call.p;
  const RowsAttend& c = call.c;
  constexpr int TERMS = 3, kDeep = kAttendWaves / WIDE, kUnit = 32 * kDeep, NU = WIDE == 4 ? 2 : 1, kRows = 32 * WIDE, kBuf = NU * kUnit * 256;
  constexpr int kLoads = kUnit / (E4M3 ? 32 : 16), kWords = kMaxDrafts / 32 + 3;
  __shared__ __align__(16) uint8_t s_tile[2][2][kBuf];          // keys, values; two buffers of NU units each
  __shared__ uint32_t s_see[kRows][kWords];
  __shared__ float s_m[kAttendWaves][32], s_l[kAttendWaves][32];
  __shared__ int s_odd, s_far;
  static_assert(sizeof s_tile >= kAttendWaves * 32 * kDim * 4, "the outputs go where the tiles were");

  const int tid = threadIdx.x, lane = tid & 63, wave = uniform_i32(tid >> 6), j = lane & 31, half = lane >> 5, wq = wave % WIDE, wk = wave / WIDE;
  if (tid == 0) s_odd = s_far = 0;
  const uint32_t each = (uint32_t)c.blocks;
  int part, b, h, blk, at_behind = 0, share = 0, limit = c.places, begins = 0;      // MORE: tiles of a piece; the most that the block can fall into; where its pieces behind its places begin
  const bool behind = MORE && blockIdx.x >= (uint32_t)c.grid;
  if constexpr (MORE) share = uniform_i32(c.cut[0]);
  if (behind) {
    int index = (int)(blockIdx.x - (uint32_t)c.grid), above = p.batch;
    if (index >= uniform_i32(c.cut[1 + p.batch])) return;
    for (b = 0; above - b > 1;) {                  // the last sequence that begins at it or before it, 64 at a time
      const int step = (above - b + 63) >> 6, at = b + lane * step;
      const u64 upto = __ballot(at < above && c.cut[1 + min(at, above - 1)] <= index);
      b += step * (63 - __clzll((long long)upto));
      above = min(above, b + step);
    }
    index -= uniform_i32(c.cut[1 + b]);
    const Have of = have_of(p, c, kRows, kUnit, told(p, c.rows, b));
    const int blocks = uniform_i32(of.blocks), more = rows_behind(uniform_i32(of.tiles), share, c.places);
    const int piece = rows_behind_piece(index, p.hkv * more, blocks), group = piece / blocks;
    blk = blocks - 1 - (piece - group * blocks);
    part = group / p.hkv;
    h = group - part * p.hkv;
    // where the block's are kept, whatever the order in which they are taken
    at_behind = (h * blocks + blk) * more + part + uniform_i32(c.cut[1 + b]);
    part += c.places;
  } else {
    const uint32_t piece = rows_piece(blockIdx.x, (uint32_t)c.units * (uint32_t)c.places, each);
    if (piece == ~0u) return;
    const uint32_t group = (uint32_t)uniform_i32((int)(piece / each));
    const RowsGroup of = rows_group(group, (uint32_t)c.units);
    part = uniform_i32((int)of.part), blk = uniform_i32((int)(each - 1 - (piece - group * each)));       // the last rows have the most to do
    b = uniform_i32((int)(of.unit / (uint32_t)p.hkv)), h = uniform_i32((int)of.unit) - b * p.hkv;
  }
  part = uniform_i32(part), b = uniform_i32(b), h = uniform_i32(h), blk = uniform_i32(blk);
  if constexpr (MORE) at_behind = uniform_i32(at_behind);
  const int u = b * p.hkv + h;
  const int64_t block_index = (int64_t)u * c.blocks + blk;
  const Told own = told(p, c.rows, b), mine = told(p, c.rows, MORE ? b : min(lane * ((p.batch + 63) >> 6), p.batch - 1));
  if constexpr (MORE) {
    const Have of = have_of(p, c, kRows, kUnit, own);
    const int more = rows_behind(uniform_i32(of.tiles), share, c.places);
    limit += more;
    begins = uniform_i32(c.cut[1 + b]) + (h * uniform_i32(of.blocks) + blk) * more;
  }
  int bad = p.max_length < own.length || own.length < 0 ? PAGED_BAD_LENGTH : 0;
  const RowSpan span = c.rows.span(uniform_i32(own.length), uniform_i32(own.first), uniform_i32(own.start), uniform_i32(own.stop), p.max_length);
  const int64_t q_base = c.rows.starts ? uniform_i32(own.start) * c.rows.row_stride : b * c.rows.seq_stride;
  if (span.bad) bad |= PAGED_BAD_LENGTH;
  const uint32_t r0 = (uint32_t)blk * kRows, n_rows = (uint32_t)uniform_i32(span.count) * (uint32_t)c.G;
  if (r0 >= n_rows) {
    if (part == 0 && tid == 0) {
      if (c.parts) c.parts[2 * block_index] = 0;
      if (blk == 0) p.report(bad);
    }
    return;
  }
  const int first = uniform_i32(span.first), count = uniform_i32(span.count), t_lo = uniform_i32((int)(r0 / c.G)), t_hi = uniform_i32((int)((min(r0 + kRows, n_rows) - 1) / c.G));
  const uint32_t row = r0 + 32 * wq + j;
  const bool valid = row < n_rows, idle = r0 + 32 * wq >= n_rows;        // idle: a wavefront without rows only brings entries into LDS
  const int token = (int)((valid ? row : r0) / c.G), g = (int)((valid ? row : r0) - (uint32_t)token * c.G);

  bf16x8 q[8];                                   // (a block's rows behind the last one: its first once more, and nobody's)
#pragma unroll
  for (int s = 0; s < 8; ++s) q[s] = __builtin_bit_cast(bf16x8, load16(c.rows.k + q_base + token * c.rows.row_stride + (h * c.G + g) * c.rows.head_stride + 2 * (16 * s + 8 * half)));

  // ---- which entries the lane's row sees: lo .. hi - 1, the first `sinks`, and of the call's rows those in s_see
  int sinks = c.window ? c.sinks : 0;
  int position = first + token, hi = position + 1, oldest, end = first + t_hi + 1;
  if (c.tree) {
    const int words = (count + 63) >> 6;
    const uint8_t* tree = c.tree + b * c.tree_seq;
    constexpr int N = 8;                           // rows on their way at once
    for (int w = 0; w < words; ++w) {
      const int at = 64 * w + lane;
      for (int t0 = t_lo + wave; t0 <= t_hi; t0 += N * kAttendWaves) {
        uint8_t x[N];
#pragma unroll
        for (int n = 0; n < N; ++n) x[n] = tree[min(t0 + n * kAttendWaves, t_hi) * c.tree_row + min(at, count - 1)];
#pragma unroll
        for (int n = 0; n < N; ++n) {
          const u64 sees = __ballot(at < count && x[n] != 0);
          if (lane < 2 && t0 + n * kAttendWaves <= t_hi) s_see[t0 + n * kAttendWaves - t_lo][2 * w + lane] = (uint32_t)(sees >> 32 * lane);
        }
      }
    }
    for (int x = tid; x < (t_hi - t_lo + 1) * kWords; x += kThreads)
      if (x % kWords >= 2 * words) s_see[x / kWords][x % kWords] = 0u;
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
  int each_part = tiles.count;
  if constexpr (MORE) each_part = rows_share(tiles.count, share, limit);
  else if (c.places > 1) each_part = rows_share(tiles.count, even_share(p, c, kRows, kUnit, lane, mine), c.places);
  const int parts = uniform_i32(unit_parts(tiles.count, each_part));
  if (part == 0 && tid == 0 && c.parts) {
    c.parts[2 * block_index] = parts;
    if constexpr (MORE) c.parts[2 * block_index + 1] = begins;
  }
  if (part >= parts) return;
  int n_first = uniform_i32(part_begin(tiles.count, parts, part));
  const int n_last = uniform_i32(part_begin(tiles.count, parts, part + 1));

  f32x16 acc[4];
  float m_run, l_run;
  const float scale_log2e = c.scale_log2e;

  // ---- units' way into LDS: rows of 256 bytes, bf16 straight there, 8 bits through registers
  int units = n_last - n_first;
  auto unit_at = [&](int i) CKV_INLINE { return tiles.tile(n_first + i) * kUnit; };
  auto seen = [&](int e) CKV_INLINE { return (bool)((e < end) & ((e >= oldest) | (e < sinks))); };
  // Where kPageSlots pages lie, a lane each, of the sequence's pages kPageSlots * window and on, and the ones before them (the pool's first instead of one that is not there).
  struct Known {
    int window = -1;
    u64 row = 0ull, scale = 0ull;
  } known, before;
  u32x4 kr[E4M3 ? NU * kLoads : 1], vr[E4M3 ? NU * kLoads : 1];
  uint32_t ks[E4M3 ? NU * kLoads : 1], vs[E4M3 ? NU * kLoads : 1];
  constexpr int kOnce = E4M3 ? 32 : 16;          // rows of a load
  constexpr int kMine = kOnce / kAttendWaves;     // of them a wavefront's, always in one page
  const int r_in = tid / (kThreads / kOnce);     // the thread's
  int shift = p.shift, page_mask = p.page_size() - 1, slot_stride = p.slot_stride;
  const uint32_t in_row = 16 * (E4M3 ? tid & 7 : (tid & 15) ^ swizzle(r_in)), lane_at = (uint32_t)(r_in * slot_stride) + in_row, next_at = lane_at + (uint32_t)(kOnce * slot_stride), wave_at = (uint32_t)(kMine * wave * slot_stride);
  uint32_t near_at = lane_at - wave_at;
  uint32_t scale_near = (uint32_t)(2 * (r_in - kMine * wave));
  const u64 k_to_v = (u64)p.v - (u64)p.k;
  auto pages = [&](int w, Known& to) CKV_INLINE {
    const auto a = args();
    int logical = w * kPageSlots + lane;
    here(logical);                               // (as at the careful pieces)
    const int64_t from = (int64_t)logical << shift, upto = from + page_mask + 1;
    const bool needed = logical < a->p.columns && from < end && (upto > oldest || from < sinks);
    const int page = needed ? a->p.table[(int64_t)b * a->p.table_stride + logical] : -1;
    const bool there = page_there(page, a->p.n_pages);
    if (needed && !there) bad |= PAGED_BAD_PAGE;
    if (__ballot(needed && !there) != 0ull) s_odd = 1;           // once more, with care
    to.row = (u64)(a->p.k + (there ? page : 0) * a->p.page_stride + h * a->p.head_stride);
    if constexpr (E4M3) to.scale = (u64)(a->p.scales + (there ? page : 0) * a->p.scale_page_stride + h * a->p.scale_head_stride);
  };
  const uint32_t k_lds = lds_at(&s_tile[0][0][0]), v_lds = k_lds + 2 * kBuf;

  // The n-th buffers take keys of units NU n + 1 and on, values of units NU n - 1 and on.  The easy way, while units' entries follow one another, each unit in one page of those that are known, all of
  // them seen by some row: a page's place out of its lane, and values where the keys of two units before were.  Units below `easy`, from `plain` on (values), may go it.
  int easy = 0, plain = 0;
  struct Rows4 {
    u64 k_row[NU], k_scale[NU];
  } last = {}, last2 = {};         // of the units whose keys were asked for last, and before that
  uint32_t unseen = 0u;
  // 8 bits go into registers, with no branch around their loads: loaded registers would be copied where ways meet, and waited for.  So the ways only work out places (the wavefront's; a lane's is so
  // much further on in all of them).
  u64 at[E4M3 ? 2 : 1][E4M3 ? NU * kLoads : 1], scale_of[E4M3 ? 2 : 1][E4M3 ? NU * kLoads : 1];
  auto ask_easy = [&](int n, int buf) CKV_INLINE {
    Rows4 now;
    const Rows4& v_last = NU == 2 ? last : last2;
    const int e0 = unit_at(NU * n + 1);
#pragma unroll
    for (int s = 0; s < NU; ++s) {
      const int e = e0 + s * kUnit, slot = (e >> shift) & (kPageSlots - 1), off = e & page_mask;
      now.k_row[s] = readlane_u64(known.row, slot) + (uint32_t)(off * slot_stride);
      if constexpr (E4M3) now.k_scale[s] = readlane_u64(known.scale, slot) + (uint32_t)(2 * off);
#pragma unroll
      for (int side = 0; side < 2; ++side) {
        u64 row = side ? v_last.k_row[s] + k_to_v : now.k_row[s];
        const u64 scale = side ? v_last.k_scale[s] + 1 : now.k_scale[s];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          if constexpr (E4M3) {
            at[side][s * kLoads + i] = row + wave_at;
            scale_of[side][s * kLoads + i] = scale + (uint32_t)(2 * (kOnce * i + kMine * wave));
          } else {
            load_to_lds((const uint8_t*)row, i & 1 ? next_at : lane_at, (side ? v_lds : k_lds) + buf * kBuf + s * kUnit * 256 + (16 * i + 4 * wave) * 256);
          }
          if constexpr (E4M3) row += (uint32_t)(kOnce * slot_stride);
          else if (i & 1) row += (uint32_t)(2 * kOnce * slot_stride);
        }
      }
    }
    last2 = last;
    last = now;
  };
  // Any way: every lane by the place of its own row.  Values of entries that no row of the block sees come as zeros: whatever lies there times a weight of nothing must be nothing (of keys it does not
  // matter).
  auto ask_any = [&](int n, int buf) CKV_INLINE {
    apart();
    last2 = last;
#pragma unroll
    for (int s = 0; s < NU; ++s)
#pragma unroll
      for (int side = 0; side < 2; ++side) {
        const int unit = NU * n + (side ? -1 : 1) + s, e0 = unit_at(min(max(unit, 0), units - 1)), w = (e0 >> shift) / kPageSlots;
        const bool all = unit >= 0 && unit < units && e0 >= oldest && e0 + kUnit <= end;
        Known from;
        if (side == 0) {
          if (w != known.window) {
            before = known;
            known.window = w;
            pages(w, known);
          }
          from = known;
          if (!all) plain = uniform_i32(unit + 1);
          const int left = min((w + 1) * kPageSlots << shift, end) - e0, slot = (e0 >> shift) & (kPageSlots - 1), off = e0 & page_mask;
          easy = all && page_mask + 1 >= kUnit && n_first + unit >= tiles.sinks ? uniform_i32(min(units, unit + left / kUnit)) : 0;
          last.k_row[s] = readlane_u64(known.row, slot) + (uint32_t)(off * slot_stride);
          if constexpr (E4M3) last.k_scale[s] = readlane_u64(known.scale, slot) + (uint32_t)(2 * off);
        } else {
          from.row = w == known.window ? known.row : before.row;
          from.scale = w == known.window ? known.scale : before.scale;
          if (w != known.window && w != before.window) pages(w, from);
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int e = e0 + kOnce * i + kMine * wave, slot = (e >> shift) & (kPageSlots - 1), off = e & page_mask;
          const u64 row = readlane_u64(from.row, slot) + (side ? k_to_v : 0ull) + (uint32_t)(off * slot_stride);
          const bool nobody = side && !((bool)((unit >= 0) & (unit < units)) & seen(e + r_in - kMine * wave));
          if constexpr (E4M3) {
            at[side][s * kLoads + i] = row;
            scale_of[side][s * kLoads + i] = readlane_u64(from.scale, slot) + (uint32_t)(2 * off + side);
            if (nobody) unseen |= 1u << (s * kLoads + i);
          } else {
            const uint32_t to = (side ? v_lds : k_lds) + buf * kBuf + s * kUnit * 256 + (16 * i + 4 * wave) * 256;
            if (side) load_to_lds(nobody ? kNothing + 16 * (tid & 15) : (const uint8_t*)row + near_at, to);
            else load_to_lds((const uint8_t*)row, near_at, to);
          }
        }
      }
  };
  auto ask = [&](auto easy_, int n, int buf) CKV_INLINE {
    unseen = 0u;
    if (decltype(easy_)::value && NU * n + NU < easy && NU * n - 1 >= plain) ask_easy(n, buf);
    else ask_any(n, buf);
    if constexpr (E4M3) {
#pragma unroll
      for (int i = 0; i < NU * kLoads; ++i) {
        kr[i] = global_at<u32x4>(at[0][i], near_at);
        ks[i] = global_at<uint8_t>(scale_of[0][i], scale_near);
        vr[i] = global_at<u32x4>(at[1][i], near_at);
        vs[i] = global_at<uint8_t>(scale_of[1][i], scale_near);
      }
    }
  };
  auto put = [&](int buf) CKV_INLINE {
    if constexpr (E4M3) {
      if (__any(unseen != 0u)) {
        apart();
#pragma unroll
        for (int i = 0; i < NU * kLoads; ++i)
          if (unseen >> i & 1u) vr[i] = u32x4{0u, 0u, 0u, 0u}, vs[i] = 127u;
      }
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
  // where a lane reads keys of the first 16 dimensions, and values of the first 32: of others at that ^ 32 x, that ^ 64 d; the other four of its eight entries at that ^ 32, eight rows on
  uint32_t k_at_ = k_lds + (wk * 32 + j) * 256 + ((half ^ swizzle(j)) << 4);
  const int l16 = lane & 15;
  uint32_t v_at_ = v_lds + (wk * 32 + 4 * half + (l16 >> 2)) * 256 + ((l16 >> 2) << 6 | ((((lane >> 4) & 1) * 2 + ((l16 >> 1) & 1)) ^ half) << 4 | (l16 & 1) * 8);
  // (With registers that 8 bits need on their way these places are worked out again and again, not kept, each in one instruction.)
  auto otherwise = [](uint32_t at, int bits) CKV_INLINE {
    if constexpr (!E4M3) return at ^ bits;
    if (bits == 0) return at;
    uint32_t y;
    asm volatile("v_xor_b32 %0, %1, %2" : "=v"(y) : "i"(bits), "v"(at));
    return y;
  };
  auto keys = [&](int x, int at) CKV_INLINE { return read_row(otherwise(k_at_, 32 * x), at); };
  auto values = [&](int n, int at, s16x4 (&v)[2]) CKV_INLINE {                       // n = 2 d + x: dimensions 32 d and on, entries 16 x and on
    v[0] = read_transposed(otherwise(v_at_, 64 * (n >> 1)), at + (n & 1) * 16 * 256);
    v[1] = read_transposed(otherwise(v_at_, 64 * (n >> 1) + 32), at + (n & 1) * 16 * 256 + 8 * 256);
  };
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
    bm = halves_combine(max2(bm, s[15]), [](float x, float y) { return max2(x, y); }) * scale_log2e;
    return bm > m_run + kSlack ? bm : m_run;
  };
  auto shrink_by = [&](float f) CKV_INLINE {
    l_run *= f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[d][i] *= f;
  };
  // Whether `count` units from the i-th on are there, side by side, and seen whole by all of the wavefront's rows.
  auto clear = [&](int i, int count) CKV_INLINE {
    const int e0 = unit_at(i), e1 = unit_at(i + count - 1) + kUnit;
    return (bool)((i + count <= units) & (e1 - e0 == count * kUnit) & (e1 <= wave_hi) & ((e0 >= wave_lo) | (e1 <= sinks)));
  };
  // Logits of entries that a row does not see: -inf.
  auto mask = [&](auto careful_, int i, f32x16& s) CKV_INLINE {
    apart();
    const int e_first = unit_at(min(i, units - 1)) + wk * 32, e_last = e_first + 31;
    uint32_t sees = 0u;
    const auto a = args();
    if (valid && i < units) {
      sees = (uint32_t)bits_between(e_first, lo, hi) | (uint32_t)bits_between(e_first, 0, min(sinks, hi));
      if (a->c.tree && e_last >= first) {
        const uint32_t* bits = s_see[token - t_lo];
        const int from = e_first - first, word = max(from, 0) >> 5, by = max(from, 0) & 31;
        const uint32_t drafts = (uint32_t)(((u64)bits[word + 1] << 32 | bits[word]) >> by);
        sees |= from >= 0 ? drafts : drafts << -from;
      }
    }
    if constexpr (decltype(careful_)::value) {
      for (int x = 0; x < 2; ++x) {
        const int col = (e_first + 16 * x) >> shift;
        if (col >= a->p.columns || !page_there(a->p.table[(int64_t)b * a->p.table_stride + col], a->p.n_pages)) sees &= ~(0xFFFFu << 16 * x);
      }
    }
    sees >>= 4 * half;
#pragma unroll
    for (int x = 0; x < 16; ++x)
      if (!(sees >> (8 * (x >> 2) + (x & 3)) & 1u)) s[x] = -INFINITY;
  };
  // The step of the i-th unit: products, and what else there is to do, in turn, so that neither waits for the other.
  auto steady = [&](auto at_, int i, bool whole, f32x16& s, f32x16& t, u32x4 (&w)[TERMS][2], u32x4 (&y)[TERMS][2]) CKV_INLINE {
    constexpr int at = decltype(at_)::value;
    u32x4 ko[2] = {keys(0, at), keys(1, at)};
    s16x4 vo[2][2];
    values(0, at, vo[0]);
    values(1, at, vo[1]);
    const Rest rest;
    if (!whole) mask(std::false_type(), i, s);
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
      a = fmaf(s[2 * n], scale_log2e, -m), z = fmaf(s[2 * n + 1], scale_log2e, -m);
      here(a);
      here(z);
      a = fast_exp2(a);
      here(a);
      if (n) last(n - 1, a_last, z_last);
      if (n < 6) ko[n & 1] = keys(n + 2, at);
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
        if (x == 1 && n < 6) values(n + 2, at, vo[n & 1]);
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
  // The same with care: a unit's values that are not finite reach those rows only that give them weight, and weights are `lowered`, after they have gone into their sum, so that all
  // else stays bit by bit what it was.
  float lowered = 1.f;
  auto any = [&](int i, int at) CKV_INLINE {
    if (i >= 1 && i <= units) {
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        f32x16 wrong = nought;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          s16x4 vo[2];
          values(2 * d + x, at, vo);
          s16x8 v = beside(vo[0], vo[1]);
          {
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
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (wrong[e] != 0.f) acc[d][e] = NAN;
      }
    }
    if (i >= 0 && i < units) {
      mask(std::true_type(), i, s);
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
        float a = fast_exp2(fmaf(s[2 * n], scale_log2e, -m)), z = fast_exp2(fmaf(s[2 * n + 1], scale_log2e, -m));
        sum += a;
        sum += z;
        a *= lowered;
        z *= lowered;
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
      for (int x = 0; x < 8; ++x) s = logits(keys(x, at), x, x ? s : nought);
    }
  };
  const uint32_t k_at0 = k_at_, v_at0 = v_at_;
  auto begin = [&]() CKV_INLINE {
#pragma unroll
    for (int d = 0; d < 4; ++d) acc[d] = nought;
    m_run = kNoLogit, l_run = 0.f;
    known.window = before.window = -1;
    ask(std::false_type(), -1, 1);
    put(1);
  };
  __syncthreads();                               // s_odd
  begin();
  ask(std::false_type(), 0, 0);
  k_at_ += kBuf, v_at_ += kBuf;
#pragma unroll
  for (int x = 0; x < 8; ++x) s = logits(keys(x, (NU - 1) * kUnit * 256), x, x ? s : nought);
#pragma unroll
  for (int x = 0; x < TERMS; ++x) w[x][0] = w[x][1] = u32x4{0u, 0u, 0u, 0u};
  put(0);
  // The n-th step, of NU units, works on the buffers of n & 1, while the next ones are filled.
  for (int n = 0;; ++n) {
    const int buf = n & 1, i = NU * n;
    if (i + NU <= units) ask(std::true_type(), n + 1, buf ^ 1);
    k_at_ += buf ? kBuf : -kBuf;
    v_at_ += buf ? kBuf : -kBuf;
    if (!idle) {
      const bool whole = clear(i, NU);
      steady(std::integral_constant<int, 0>(), i, whole, s, t, w, y);
      if constexpr (NU == 2) {
        steady(std::integral_constant<int, kUnit * 256>(), i + 1, whole, t, s, y, w);
      } else {
        s = t;
#pragma unroll
        for (int x = 0; x < TERMS; ++x) w[x][0] = y[x][0], w[x][1] = y[x][1];
      }
    }
    if (i + NU > units) break;
    put(buf ^ 1);
  }
  __syncthreads();
  // Once more with care where a page was missing, or something that is no number came out: a value that only some rows see must not reach the others.  And once more with lowered weights where that leaves
  // anything so large that a few thousand pieces' sums might be infinite (finite values are below 2^128), or no number, as infinite sums of both signs do.
  auto sound = [&]() CKV_INLINE {                // below 2^115, and numbers
    float nothing = 0.f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) nothing = fmaf(acc[d][i], kLargeSums, nothing);
    return fabsf(nothing) < INFINITY;
  };
  if (!sound()) s_odd = 1;
  __syncthreads();
  if (uniform_i32(s_odd)) {
    // (what is worked out of these again would otherwise wait from the beginning on, in lanes of vector registers and in scratch)
    here(near_at), here(scale_near);
    for (int* x : {&tiles.sinks, &tiles.base, &end, &oldest, &sinks, &units, &n_first, &shift, &page_mask, &slot_stride}) here_scalar(*x);
#pragma unroll 1
    for (int turn = 0; turn < 2; ++turn) {
      if (turn == 1) {
        if (!sound()) s_far = 1;                 // (what is no number may be infinity less infinity)
        __syncthreads();
        if (!uniform_i32(s_far)) break;
        lowered = args()->c.lower;
      }
      begin();
      k_at_ = k_at0, v_at_ = v_at0;
#pragma unroll 1
      for (int n = -1; NU * n <= units; ++n) {
        const int buf = n & 1;
        ask(std::false_type(), n + 1, buf ^ 1);
#pragma unroll 1
        for (int x = 0; x < NU; ++x) any(NU * n + x, buf * kBuf + x * kUnit * 256);
        put(buf ^ 1);
      }
    }
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
  const auto a = args();
  const int G = a->c.G, hkv = a->p.hkv;
  const int64_t out_row = a->c.rows.starts ? a->c.rows.starts[b] : (int64_t)b * a->c.rows.rows;
  float *lse = a->c.lse, *partial = a->c.partial, *ml = a->c.ml;
  uint8_t* out = a->c.out;
  const bool out_bf16 = a->c.out_bf16;
  const int64_t piece = behind ? a->c.units * a->c.blocks * a->c.places + at_behind : block_index * a->c.places + part;
  const float raised = 1.f / lowered;
  constexpr int kEnd = 4;                          // rows at once
  const int chunk = tid & 31;
  for (int r_first = tid >> 5; r_first < kRows; r_first += kThreads / 32 * kEnd) {
    f32x4 y[kEnd];
    float M[kEnd], L[kEnd];
#pragma unroll
    for (int i = 0; i < kEnd; ++i) {
      const int r = r_first + kThreads / 32 * i, in = r & 31;
      M[i] = kNoLogit, L[i] = 0.f, y[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < kDeep; ++k) M[i] = fmaxf(M[i], s_m[k * WIDE + (r >> 5)][in]);
#pragma unroll
      for (int k = 0; k < kDeep; ++k) {
        const int w = k * WIDE + (r >> 5);
        const float f = fast_exp2(s_m[w][in] - M[i]);
        L[i] += s_l[w][in] * f;
        y[i] += *reinterpret_cast<const f32x4*>(s_o + (w * 32 + in) * kDim + 4 * (chunk ^ in)) * f;
      }
    }
#pragma unroll
    for (int i = 0; i < kEnd; ++i) {
      const int r = r_first + kThreads / 32 * i;
      if (r0 + r >= n_rows) break;
      if (parts > 1) {
        const int64_t at = piece * kRows + r;
        *reinterpret_cast<f32x4*>(partial + at * kDim + 4 * chunk) = y[i];
        if (chunk == 0) *reinterpret_cast<f32x2*>(ml + 2 * at) = f32x2{M[i], lowered < 1.f ? -L[i] : L[i]};
      } else {
        const int t = (int)((r0 + r) / G);
        const int64_t to = (out_row + t) * (G * hkv) + h * G + (int)(r0 + r - (uint32_t)t * G);
        put_row(out, out_bf16, to, 4 * chunk, L[i] != 0.f ? y[i] * (1.f / L[i]) * raised : f32x4{0.f, 0.f, 0.f, 0.f});
        if (chunk == 0 && lse) lse[to] = natural(M[i], L[i]);
      }
    }
  }
  if (bad && a->p.status) atomicOr(a->p.status, bad);
}

// Joins the pieces of blocks of rows that have several: 32 threads a row, four dimensions each, eight rows a workgroup, which takes every `gridDim.y`-th eight of a block (64 drafts of 32
// sequences of many lengths, 512 blocks: 14.6 us with all of a block's eights side by side, 19.4 with four).  Bound by trips: parts, lengths, partial outputs, eight of them at once.
constexpr int kRowsJoined = 8;
template <int WIDE, bool MORE>
__global__ __launch_bounds__(32 * kRowsJoined) void paged_rows_join_kernel(RowsCall call) {
  const Paged& p = call.p;
  const RowsAttend& c = call.c;
  constexpr int kRows = 32 * WIDE;
  const int64_t block_index = blockIdx.x;
  const int parts = c.parts[2 * block_index];
  if (parts <= 1) return;
  const int64_t begins = block_index * c.places, behind = MORE ? c.units * c.blocks * c.places + c.parts[2 * block_index + 1] - c.places : 0;
  const int u = (int)(block_index / c.blocks), blk = (int)(block_index - (int64_t)u * c.blocks), b = u / p.hkv, h = u - b * p.hkv;
  int64_t base;
  const RowSpan span = c.rows.span(b, p.lengths[b], p.max_length, base);
  const int d4 = 4 * (threadIdx.x & 31);
  for (int in = blockIdx.y * kRowsJoined + (threadIdx.x >> 5); in < kRows; in += kRowsJoined * gridDim.y) {
    const uint32_t row = (uint32_t)blk * kRows + in;
    if (row >= (uint32_t)span.count * (uint32_t)c.G) return;
    float M = kNoLogit, L = 0.f, lowered = 1.f;       // what y, of several parts, is multiplied by
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    constexpr int N = 8;                           // parts on their way at once
    for (int i0 = 0; i0 < parts; i0 += N) {
      f32x2 st[N];
      f32x4 x[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int part = min(i0 + i, parts - 1);
        const int64_t at = ((!MORE || part < c.places ? begins : behind) + part) * kRows + in;
        st[i] = *reinterpret_cast<const f32x2*>(c.ml + 2 * at);
        x[i] = *reinterpret_cast<const f32x4*>(c.partial + at * kDim + d4);
      }
      float m = M;
      uint32_t signs = 0u;                         // of a part with lowered weights the sum of weights has a sign
#pragma unroll
      for (int i = 0; i < N; ++i) m = fmaxf(m, st[i][0]), signs |= __float_as_uint(st[i][1]);
      if (signs >> 31 && lowered == 1.f) lowered = c.lower, y = y * lowered;
      const float old = fast_exp2(M - m);
      M = m;
      L *= old;
      y = y * old;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float now = i0 + i < parts ? fast_exp2(st[i][0] - m) : 0.f;
        L += fabsf(st[i][1]) * now;
        y += x[i] * (__float_as_uint(st[i][1]) >> 31 ? now : now * lowered);
      }
    }
    const int t = (int)(row / c.G);
    const int64_t to = ((c.rows.starts ? c.rows.starts[b] : (int64_t)b * c.rows.rows) + t) * (c.G * p.hkv) + h * c.G + (int)(row - (uint32_t)t * c.G);
    put_row(c.out, c.out_bf16, to, d4, L != 0.f ? y * (1.f / L) * (1.f / lowered) : f32x4{0.f, 0.f, 0.f, 0.f});
    if (d4 == 0 && c.lse) c.lse[to] = natural(M, L);
  }
}

}  // namespace ckv
