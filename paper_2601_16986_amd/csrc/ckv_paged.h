// A cache in pages: what host and kernels share by way of sizes.  Plain C++, no HIP, so that a host program can include it.
#pragma once
#include "ckv_plan.h"

namespace ckv {

constexpr int kMinPage = 16, kMaxPage = 256;
constexpr int kPageSlots = 64;         // pages that a wavefront knows the whereabouts of, one per lane
constexpr int kPagedGroup = 16;        // query heads per KV head, at most
constexpr int kMaxPicked = 32768;      // pages that a selection can choose from (32 keys in each of 1024 threads)
enum { PAGED_BAD_PAGE = 1, PAGED_BAD_LENGTH = 2, PAGED_BAD_PICK = 4 };

// Entries of the sequence's page `page` that lie before its end.
CKV_PLAN int page_fill(int length, int page, int shift) {
  const long long left = length - ((long long)page << shift);
  return left <= 0 ? 0 : left < (1 << shift) ? (int)left : 1 << shift;
}

// Whether a table's value names a page of the pool.
CKV_PLAN bool page_there(int page, int n_pages) { return (unsigned)page < (unsigned)n_pages; }

// Rows of one sequence in a call that writes or reads rows: positions first .. first + count - 1 of `length`; the last ones where the caller names no first, as many as
// the sequence has in the call.
struct RowSpan {
  int first, count;
  bool bad;
};
CKV_PLAN RowSpan row_span(int length, int most, bool has_first, int first, bool packed, int start, int stop, int total) {
  if (packed) {
    if (start < 0 || stop < start || stop > total) return {0, 0, true};
    if (stop - start < most) most = stop - start;
  }
  if (!has_first) first = length > most ? length - most : 0;
  if (first < 0 || first > length) return {0, 0, true};
  return {first, length - first < most ? length - first : most, false};
}
// Those below `limit`, the most that a length may be: of a sequence that outgrew it rows behind the limit are left out, none moves.
CKV_PLAN RowSpan rows_below(RowSpan s, int limit) {
  if (s.count > 0 && s.count > limit - s.first) s.count = limit - s.first;
  if (s.count <= 0) s.first = s.count = 0;
  return s;
}

// Whether a page's rows are written by one wavefront instead of four, where pages are enough to fill the chip all the same and have few new rows: the smallest
// pages, or up to four rows a sequence (one pass either way). us, four / one: prompts of 8 x 9350 over 8 heads, pages of 16 80.7 / 63.3, of 32 62.6 / 63.5, of 64
// 60.5 / 68; 32 prompts of up to 1000, pages of 16, 26.9 / 16.3; one of 777 over 4 heads (196 pages) 4.1 / 5.0; single rows of 32 x 8 4.0 / 4.2, 256 x 8 7.3 / 5.1.
CKV_PLAN bool appends_by_wave(int page_size, int rows, long long pages, int n_cu) {
  return page_size == kMinPage ? pages >= 16ll * n_cu : rows <= 4 && pages >= 4ll * n_cu;
}

// Whether rows that are read back (so many keys, and as many values) are stored past the caches: where they would fill a good part of the last one (256 MiB). us,
// through / past: 322208 rows (165 MB) 55.8 / 49.9 out of 8 bits, 71.6 / 68.2 out of bf16; 72192 rows (37 MB) 11.7 / 11.6.
CKV_PLAN bool reads_past_caches(long long rows) { return rows * kDim * 4 >= (64ll << 20); }

// An attention's work in blocks of 32 entries: one for a unit (sequence, KV head) without entries, whose output somebody has to write.
constexpr int kAttendWaves = 4;         // of a workgroup, which take blocks in turn
CKV_PLAN int unit_blocks(int entries) { return entries > 32 ? (int)(((long long)entries + 31) / 32) : 1; }
CKV_PLAN int unit_parts(int blocks, int share) { return blocks / share + (blocks % share != 0); }
// The work is cut into pieces of at most an even share of all blocks, at least a block for each wavefront.
CKV_PLAN int attend_share(int blocks, int workers) {
  const int even = unit_parts(blocks, workers);
  return even > kAttendWaves ? even : kAttendWaves;
}

// Units that end inside a share make more pieces than there are shares. Where units are few, larger pieces make up for it, so that no compute unit has more than
// its two; of many units pieces would become too uneven.  Sequences of 8 heads, lengths spread up to 9350 entries, us, as they are / larger: bf16, 64 units 36.7 / 33.3, 96 45.1 / 41.2,
// 128 46.9 / 43.0, 192 59.9 / 55.3, 256 92.9 / 92.8, 320 108 / 114, 384 112 / 118, 512 139 / 157; 8 bits, 128 28.8 / 27.8, 192 35.8 / 34.9, 256 53.0 / 53.1, 384 61.8 / 68.2.  (Taken up to 128
// units of 256 compute units, clear of where it turns.)
CKV_PLAN bool enlarges_share(int batch, int hkv, int workers) { return batch <= 64 && 4 * batch * hkv <= workers; }
CKV_PLAN int larger_share(int share, int pieces, int workers) { return (int)((float)share * (float)pieces / (float)workers) + 1; }
// First block of one of a unit's parts (that of part `parts` is `blocks`): the first ones have a block more.
CKV_PLAN int part_begin(int blocks, int parts, int part) {
  const int even = blocks / parts, more = blocks - even * parts;
  return part * even + (part < more ? part : more);
}

// How the host has it cut, knowing no length but the most that there can be.  Two shares per compute unit (1, 2, 3, 4 of them, us: 64 x 8 units of 9350 entries in 8 bits 188 /
// 188 / 216 / 216, 8 of 131072 64 / 52 / 55 / 62, 64 x 8 ragged ones 98 / 78 / 87 / 82, 16 x 8 ragged in bf16 45 / 45 / 45 / 44).  Units of up to twelve blocks are not
// cut (2 of 300 entries 6.7 us whole, 7.2 cut; of 600 9.3 and 8.1), nor up to 32 blocks where there is one for each compute unit (512 of up to 500 12 / 17).  Looking
// for the pieces takes a workgroup about 1 us, which small work is spared (32 units of 2049 entries 11.7 / 13.2).
struct AttendPlan {
  int share;            // blocks of a piece, where every unit has the same number of places for pieces; 0: workgroups look for theirs
  int places;           // then so many for each unit
  int workers;          // otherwise the shares of all blocks that pieces are cut by
  long long pieces;     // workgroups
  bool split;           // whether a unit may fall into several pieces
};
CKV_PLAN AttendPlan attend_plan(long long units, int entries, bool same, int n_cu) {
  const int blocks = unit_blocks(entries), workers = 2 * n_cu;
  if (blocks <= 3 * kAttendWaves || (blocks <= 8 * kAttendWaves && units >= n_cu)) return {blocks, 1, 0, units, false};
  if (same || units * unit_parts(blocks, kAttendWaves) <= 4 * n_cu) {
    const long long even = (units * blocks + workers - 1) / workers;
    const int share = even > kAttendWaves ? (int)(even < blocks ? even : blocks) : kAttendWaves, places = unit_parts(blocks, share);
    return {share, places, 0, units * places, places > 1};
  }
  return {0, 0, workers, workers + units, true};
}

// Whether a selection is one kernel, a workgroup per unit, or two: scores by workgroups of so many pages, then the picking.  us, one kernel / two: 8 units of 256 pages 8.6 /
// 8.3, 64 of 293 14.3 / 14.0, 64 of 512 14.7 / 13.1, 8 of 512 11.5 / 8.5, 512 of 293 14.6 / 16.3, 512 of 512 28.6 / 42; a second launch takes the host 3 us more.
constexpr int kFewPages = 512;
CKV_PLAN bool selects_whole(int units, int columns, int n_cu) { return columns <= (units >= n_cu ? kFewPages : kFewPages * 5 / 8); }
// Whether a selection reads bounds past the caches: not where those of several layers stay in the last one (256 MiB).  us, through / past: 64 sequences of 8 heads, 256
// pages each (67 MB) 16.4 / 17.7, 512 (134 MB) 32.8 / 28.6, 1000 (262 MB) 63 / 54.
CKV_PLAN bool bounds_past_caches(long long units, int columns) { return units * columns * 4 * kDim >= (96ll << 20); }
CKV_PLAN int score_pages_each(int units, int columns, int n_cu) {
  int each = 64;
  while (each < 512 && (long long)units * ((columns + each - 1) / each) > 4ll * n_cu) each *= 2;
  return each;
}

}  // namespace ckv
