// Attention of several rows per sequence over a cache in pages: what host and kernels share by way of sizes.  Plain C++, no HIP, so that a host program can include it.
#pragma once
#include "ckv_paged.h"

namespace ckv {

typedef unsigned long long u64_t;

constexpr int kMaxDrafts = 512;        // rows of a sequence in a call with a tree

// Workgroups that share the heads of a page's rows where rows enter with their rotation, of `pages` that rows may reach: as many as find a compute unit of their own, where there are more rows
// than a workgroup turns at once and so many heads (key and value are one).
CKV_PLAN int turned_by(long long pages, int rows, int group, int n_cu) {
  if (rows <= 16 || pages <= 0) return 1;
  const long long many = n_cu / pages;
  return many < 1 ? 1 : many < group + 1 ? (int)many : group + 1;
}

// A workgroup of four wavefronts has 64 or 128 rows (a row is a query head of one of the call's rows), 32 for each of `wide` = 2 or 4 wavefronts side by side; where two do, the others have the other
// half of the entries.  The entries that they take at once, 32 each, are a tile.  128 rows where there are more than 64: what goes through LDS serves twice as many (us in blocks of 64 and of 128, over 4096 entries
// of 32 sequences with 8 KV heads, then 777 of 4 with 4: 8 bits, 128 rows 180 and 174, 24.9 and 23.5; 64 rows 116 and 140, 19.9 and 21.4; 32 rows 90 and 114, 18.4 and 20.4).
CKV_PLAN int rows_tile(int wide) { return 128 / wide; }

// Which entries a block of rows has to look at, in tiles: those of the first `sinks` entries, and those from the oldest that any row's window holds up to the end of the
// last row's.  Tiles 0 .. first - 1 are the former, from then on those from `base` on.
struct RowTiles {
  int sinks, base, count;        // tiles of sinks; the tile that follows them; all
  CKV_PLAN int tile(int n) const { return n < sinks ? n : n - sinks + base; }
};
CKV_PLAN RowTiles row_tiles(int oldest, int end, int sinks, int size) {
  if (end <= 0) return {0, 0, 0};
  if (oldest > end) oldest = end;
  const int few = sinks < oldest ? sinks : oldest;                      // sinks that lie before the window
  int head = few / size + (few % size != 0), base = oldest / size;
  const int last = (int)(((long long)end + size - 1) / size);
  if (base < head) base = head;
  return {head, base, head + (last > base ? last - base : 0)};
}

// 64 entries from `e0` on, a bit each: those in [lo, hi).
CKV_PLAN u64_t bits_between(long long e0, long long lo, long long hi) {
  const long long a = lo - e0 < 0 ? 0 : lo - e0, z = hi - e0 > 64 ? 64 : hi - e0;
  if (a >= z) return 0;
  return (z >= 64 ? ~0ull : (1ull << z) - 1) & ~((1ull << a) - 1);
}

// How a call is cut, by what the host knows: every block of rows has `places` places for pieces, of `least` tiles at least (us with 1, 3, 4 tiles of 64 rows, 13 in all: 18.6, 20.5, 22.2;
// with 2, 3, 6, 8 of 128 rows, 25 in all: 23.5, 22.7, 23.7, 26.3).  Up to four pieces for each compute unit, none where there are as many blocks: a piece beside whole blocks costs its beginning, end and joining for nothing
// (384 blocks of one length 251 us whole, 257 in pieces), but sequences of many lengths leave units idle without (64 drafts of 32 of them 450 whole, 392 in pieces; one sequence of 131072 4940 and 292).
// Where that could leave one sequence much longer than the others pieces of more than kLongPiece tiles, and a sequence's blocks do not fill the chip by themselves, every block has one place instead, and the pieces behind it,
// up to kMorePieces for each compute unit, are dealt out by the lengths on the device (paged_rows_cut_kernel).  us, equal places / dealt out: one sequence of 131072 among others of 200, 8 KV heads with 4 each, 2 x 64 drafts 535 / 345,
// 32 x 64 1780 / 423, 64 x 64 5190 / 412, 64 x 8 1154 / 166, 600 x 8 3350 / 335, parts of 256 rows of 16 5180 / 1087; 32 x 64 of lengths evenly up to 30000 1250 / 1085.  Of one length: 32 x 64 of 8192 585 / 577, 64 x 8 of 2000 92 / 83,
// 300 x 8 of 500 152 / 164.  Where it turns, one of n among others of 200: 64 x 64, n = 1500 (47 tiles) 89 / 121, 2000 (63) 108 / 104, 3000 (94) 148 / 131; 300 x 8, n = 4000 (63) 123 / 149, 6000 (94) 174 / 154.
constexpr int kLongPiece = 80, kMorePieces = 4;
struct RowsPlan {
  int wide, blocks;              // wavefronts side by side over rows; blocks of rows per unit (sequence, KV head)
  int least, places, workers;    // workers: compute units
  long long pieces;              // workgroups
  int more;                      // and those for pieces behind their block's places
};
CKV_PLAN RowsPlan rows_plan(long long units, int rows, int group, int entries, int n_cu, int batch = 1) {
  const long long all = (long long)rows * group;
  RowsPlan p = {all <= 64 ? 2 : 4, 0, 0, 1, 0, 0, 0};
  const int each = 32 * p.wide, size = rows_tile(p.wide);
  p.blocks = (int)((all + each - 1) / each);
  p.least = p.wide == 4 ? 3 : 1;
  p.workers = n_cu;
  const int tiles = (int)(((long long)entries + size - 1) / size) + 2;          // sinks and window begin inside a tile
  const long long blocks = units * p.blocks, many = 4ll * n_cu, most = 1 + (many + blocks - 1) / blocks;
  p.places = unit_parts(tiles, p.least);
  if (p.places > most) p.places = (int)most;
  if (blocks >= many) p.places = 1;
  if (batch > 1 && units / batch * p.blocks < n_cu && unit_parts(tiles, p.places) > kLongPiece) {
    p.places = 1;
    p.more = kMorePieces * n_cu;
  }
  p.pieces = units * p.blocks * p.places;
  return p;
}

// Tiles of a piece, where a block of rows turns out to have `tiles` of them: never more pieces than places.
CKV_PLAN int rows_share(int tiles, int share, int places) {
  const int least = unit_parts(tiles, places);
  return share > least ? share : least;
}
// What a call takes, in the time of a tile that has its compute unit for itself (about 1.1 us): two side by side take half as
// long again.  A piece's beginning and end (its rows, pages and first tiles) take as much as 11, joining 4, and what pieces leave for it 3 for 128 rows each.
struct RowsCost {
  int block_rows, workers;
  CKV_PLAN float turn(int k) const { return k > 1 ? 0.75f * k : 1.f; }
  CKV_PLAN float split(int k, float tiles) const { return turn(k) * (tiles + 11.f) + 4.f + 3.f * k * block_rows / 128; }
  // whole blocks: the longest, or what each unit has to do and half of that
  CKV_PLAN float whole(float blocks, float tiles, float longest) const {
    if (blocks <= workers) return longest + 11.f;
    if (blocks <= 2 * workers) return 1.5f * (longest + 11.f);
    return 0.75f * (tiles + 11.f * blocks) / workers + 0.5f * longest;
  }
};

// Tiles of a piece, by the lengths as they are: of the ways to have one, two, four or six pieces for each compute unit, and of no pieces (INT_MAX), the one that ends first.  sum(f): over all
// blocks of rows, of f(its tiles).  `most` pieces for each compute unit at most; where a block has no more than its places (`only`), the longest has what they leave it.
template <class Sum>
CKV_PLAN int rows_cut(const RowsCost& cost, int least, int places, bool only, int most, float longest, const Sum& sum) {
  const float all = sum([](float tiles) { return tiles; }), blocks = sum([](float) { return 1.f; });
  float best = cost.whole(blocks, all, longest);
  int share = 0x7FFFFFFF;
#if defined(__HIPCC__)
#pragma unroll 1
#endif
  for (int k = 1; k <= most; k += k == 1 ? 1 : 2) {
    const float pieces_at_most = (float)(k * cost.workers);
    float s = __builtin_ceilf(all / pieces_at_most);
    if (s < (float)least) s = (float)least;
    const float pieces = sum([&](float tiles) { return __builtin_ceilf(tiles / s); });
    float took = 0.f;
    if (!only && blocks > pieces_at_most) {          // more blocks than pieces: only the long ones fall into some
      took = cost.whole(pieces, all, s) + 4.f;
    } else {
      if (pieces > pieces_at_most) s = __builtin_ceilf(s * pieces / pieces_at_most);
      const float left = __builtin_ceilf(longest / (float)places);
      took = cost.split(k, only && left > s ? left : s);
    }
    if (took < best) best = took, share = s < 0x1p30f ? (int)s : 1 << 30;
  }
  return share;
}
// A block's pieces behind its places, where a sequence's blocks have so many tiles.
CKV_PLAN int rows_behind(int tiles, int share, int places) {
  const int parts = unit_parts(tiles, share);
  return parts > places ? parts - places : 0;
}
// Which of a sequence's pieces behind places, `groups` of `blocks` that read the same entries, the index-th is: the blocks of a group, eight apart, go to one part of the chip as long as groups make full rounds.
CKV_PLAN int rows_behind_piece(int index, int groups, int blocks) {
  if (index >= groups / 8 * 8 * blocks) return index;
  const int round = index / (8 * blocks), in = index - round * 8 * blocks;
  return (round * 8 + in % 8) * blocks + in / 8;
}

// What a piece's outputs, before they are divided by the sum of weights, may reach without care: kLargeSums times that (more than a block of rows has pieces) is 2^128.
constexpr float kLargeSum = 0x1p115f, kLargeSums = 0x1p13f;
// By what weights of at most 2^8 each are multiplied where they reach it: as many of them as a sequence has entries then add up to less than a half, and their sum times any values is finite.
CKV_PLAN float lowered_by(int max_length) {
  float f = 0x1p-10f;
  for (; max_length > 1; max_length = max_length / 2 + max_length % 2) f *= 0.5f;
  return f;
}

// Which of all groups' `each` blocks of rows the workgroup `index` takes: workgroups go to the eight parts of the chip in turn, each with a cache of its own, so the blocks of a group, which read the
// same entries (a unit's, in one piece of it), go to one of them, groups in turn; those of the last groups that make no full round are dealt out evenly, neighbours together.  T(-1): none.
constexpr int kParts = 8;
template <class T>
CKV_PLAN T rows_grid(T units, T each) {
  const T full = units / kParts * kParts, rest = (units - full) * each;
  return full * each + (rest + kParts - 1) / kParts * kParts;
}
template <class T>
CKV_PLAN T rows_piece(T index, T units, T each) {
  const T full = units / kParts * kParts;
  if (index < full * each) {
    const T round = index / (kParts * each), in = index - round * kParts * each;
    return (round * kParts + in % kParts) * each + in / kParts;
  }
  const T in = index - full * each, rest = (units - full) * each, chunk = (rest + kParts - 1) / kParts, at = in % kParts * chunk + in / kParts;
  return at < rest ? full * each + at : T(-1);
}
// The groups: all units' first pieces, then all second ones and so on, so that the places that turn out to be empty come last (first to last in each unit they took workgroups' room from what there was
// to do: 25 rows for 16 sequences in a window of 1024 69 us, not 52).  Where units are few or make no full rounds, each piece of a unit on another part of the chip than the one before (39 rows of 3 heads for
// 3 sequences of up to 6845 x 4 KV heads 30.6 us, all on one 43.6); else on the same, which has its queries, mask and table then (8 drafts of 4 short sequences x 4 heads 20.3 us, 21.6 on another each).
struct RowsGroup {
  unsigned part, unit;
};
CKV_PLAN RowsGroup rows_group(unsigned group, unsigned units) {
  const unsigned part = group / units, in = group - part * units;
  if (units % 2 || (units % kParts == 0 && units > kParts)) return {part, in};
  return {part, (in + part) % units};
}

}  // namespace ckv
