// Attention of several rows per sequence over a cache in pages: what host and kernels share by way of sizes.  Plain C++, no HIP, so that a host program can include it.
#pragma once
#include "ckv_paged.h"

namespace ckv {

typedef unsigned long long u64_t;

constexpr int kMaxDrafts = 512;        // rows of a sequence in a call with a tree

// A workgroup of four wavefronts has 32, 64 or 128 rows (a row is a query head of one of the call's rows), which its wavefronts share, 32 each; where fewer wavefronts do, each of
// them has its part of the entries.  `wide`: wavefronts side by side over rows, 1, 2 or 4.
// The entries that they take at once, 32 each, are a tile.
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
  int head = (few + size - 1) / size, base = oldest / size;
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

// How a call is cut.  Every block of rows has `places` places for pieces of `share` tiles at least.
struct RowsPlan {
  int wide, blocks;              // wavefronts side by side over rows; blocks of rows per unit (sequence, KV head)
  int share, places;
  long long pieces;              // workgroups
};
CKV_PLAN RowsPlan rows_plan(long long units, int rows, int group, int entries, int n_cu) {
  const long long all = (long long)rows * group;
  RowsPlan p = {all <= 32 ? 1 : all <= 64 ? 2 : 4, 0, 0, 1, 0};
  const int each = 32 * p.wide, size = rows_tile(p.wide);
  p.blocks = (int)((all + each - 1) / each);
  const int tiles = (int)(((long long)entries + size - 1) / size) + 2;          // sinks and window begin inside a tile
  const long long work = units * p.blocks * tiles, workers = (p.wide == 1 ? 1ll : 2ll) * n_cu;
  long long share = (work + 2 * workers - 1) / (2 * workers);
  if (share < 4 * p.wide) share = 4 * p.wide;
  p.share = share < tiles ? (int)share : tiles;
  p.places = unit_parts(tiles, p.share);
  p.pieces = units * p.blocks * p.places;
  return p;
}

// Tiles of a piece, where a block of rows turns out to have `tiles` of them: never more pieces than places.
CKV_PLAN int rows_share(int tiles, int share, int places) {
  const int least = unit_parts(tiles, places);
  return share > least ? share : least;
}

// Which piece the workgroup `index` takes: workgroups go to the eight parts of the chip in turn, each with a cache of its own, so a unit's pieces go to one of them, units in
// turn; those of the last units that make no full round are dealt out evenly, neighbours together.  -1: none.
constexpr int kParts = 8;
CKV_PLAN long long rows_grid(long long units, long long each) {
  const long long full = units / kParts * kParts, rest = (units - full) * each;
  return full * each + (rest + kParts - 1) / kParts * kParts;
}
CKV_PLAN long long rows_piece(long long index, long long units, long long each) {
  const long long full = units / kParts * kParts;
  if (index < full * each) {
    const long long round = index / (kParts * each), in = index - round * kParts * each;
    return (round * kParts + in % kParts) * each + in / kParts;
  }
  const long long in = index - full * each, rest = (units - full) * each, chunk = (rest + kParts - 1) / kParts, at = in % kParts * chunk + in / kParts;
  return at < rest ? full * each + at : -1;
}

}  // namespace ckv
