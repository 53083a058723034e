// A cache in pages: what host and kernels share by way of sizes.  Plain C++, no HIP, so that a host program can include it.
#pragma once
#include "ckv_plan.h"

namespace ckv {

constexpr int kTile = 16;              // entries of one operand of a matrix product, never across a page's end
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

// Rows of one sequence in a call that writes or reads rows: positions first .. first + count - 1 of `length`.
struct RowSpan {
  int first, count;
  bool bad;
};
CKV_PLAN RowSpan row_span(int length, int most, bool has_first, int first, bool packed, int start, int stop, int total) {
  if (!has_first) first = length > most ? length - most : 0;
  if (first < 0 || first > length) return {0, 0, true};
  int count = length - first < most ? length - first : most;
  if (packed) {
    if (start < 0 || stop < start || stop > total) return {0, 0, true};
    if (stop - start < count) count = stop - start;
  }
  return {first, count, false};
}

// Entries per workgroup of an attention over `entries` at most for each of `units`: a power of two from 128 (a block of 32 for each of four
// wavefronts) to what kPageSlots pages hold, the smallest that makes no more than eight workgroups per compute unit.
CKV_PLAN int attend_piece(long long units, long long entries, int shift, int n_cu) {
  const int most = (kPageSlots << shift) < 4096 ? kPageSlots << shift : 4096;
  int piece = 128;
  while (piece < most && units * ((entries + piece - 1) / piece) > 8ll * n_cu) piece *= 2;
  return piece;
}
CKV_PLAN int attend_pieces(long long entries, int piece) { return entries <= piece ? 1 : (int)((entries + piece - 1) / piece); }

}  // namespace ckv
