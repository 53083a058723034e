"""The cache in pages without a GPU: which positions rows of a call go to, how an attention is cut, and what refusals say.  The
index arithmetic is that of the kernels, compiled on its own."""
import ctypes as C

import pytest

from paper_2601_16986_amd import ckv
from tests.test_paged_cpu import _run, good  # noqa: F401


# ------------------------------------------------------------------ rows
def test_rows_go_to_the_positions_that_the_header_names(tmp_path):
    """Without `first` the last ones of the sequence, as many as it has in the call, packed or not."""
    _run(tmp_path, r"""
  const int total = 400;
  for (int length : {0, 1, 5, 100, 300, 1 << 30})
    for (int most : {1, 5, 10, 150, 300})
      for (int has = 0; has < 2; ++has)
        for (int first : {0, 1, 90, 97, 100})
          for (int packed = 0; packed < 2; ++packed)
            for (int start : {0, 7, 100})
              for (int own : {0, 1, 3, 10, 200, 300}) {
                const ckv::RowSpan s = ckv::row_span(length, most, has, first, packed, start, start + own, total);
                const int there = packed && own < most ? own : most;
                if (has && first > length) {
                  if (!s.bad || s.count) return std::printf("rows behind the sequence\n"), 1;
                  continue;
                }
                const int want = has ? first : length > there ? length - there : 0;
                const int count = length - want < there ? length - want : there;
                if (s.bad || s.count != count || (count && s.first != want)) return std::printf("length %d rows %d own %d: first %d count %d, %d %d expected\n", length, most, packed ? own : -1, s.first, s.count, want, count), 1;
              }
  const ckv::RowSpan s = ckv::row_span(100, 10, false, 0, true, 0, 3, 3);
  if (s.first != 97 || s.count != 3 || s.bad) return std::printf("%d %d\n", s.first, s.count), 1;""")


def test_rows_behind_the_largest_length_are_left_out(tmp_path):
    """Of a sequence of any length, whatever the array holds, the rows below the limit keep their positions."""
    _run(tmp_path, r"""
  for (int limit : {0, 1, 48, 1 << 30})
    for (int length : {INT_MIN, -1, 0, 1, 47, 48, 49, 60, 1 << 30, (1 << 30) + 1, INT_MAX})
      for (int most : {1, 5, 64, 1 << 30})
        for (int has = 0; has < 2; ++has)
          for (int first : {INT_MIN, -1, 0, 1, 40, 47, 48, 49, 1 << 30, INT_MAX}) {
            const ckv::RowSpan all = ckv::row_span(length, most, has, first, false, 0, 0, 0), s = ckv::rows_below(all, limit);
            const long long stop = (long long)all.first + all.count, end = stop < limit ? stop : limit;
            const long long want = end > all.first ? end - all.first : 0;
            if (s.bad != all.bad || s.count != want || s.first < 0 || (long long)s.first + s.count > limit || (want && s.first != all.first))
              return std::printf("limit %d length %d rows %d first %d: %d, %d\n", limit, length, most, has ? first : -1, s.first, s.count), 1;
          }""")


# ------------------------------------------------------------------ how an attention is cut
def test_every_piece_has_a_workgroup_and_a_place(tmp_path):
    """Batches of any size and any lengths, each sequence's and head's unit counted: as many workgroups as pieces, parts only where the host expects them, and a unit's parts are its blocks."""
    _run(tmp_path, r"""
  static int length[4096];
  unsigned seed = 1;
  auto random = [&](long long n) { seed = seed * 1664525u + 1013904223u; return (int)((seed >> 8) % (unsigned long long)n); };
  long long enlarged = 0, cut = 0, many = 0;
  for (int batch : {1, 2, 3, 7, 15, 16, 17, 40, 63, 64, 65, 100, 128, 129, 300, 1000, 4096})
    for (int hkv : {1, 2, 3, 8, 16, 64})
      for (int n_cu : {256, 64})
        for (long long most = 0; most <= (1 << 24); most = most * 2 + 1 + random(40)) {
          const long long units = (long long)batch * hkv;
          if (units * ckv::unit_blocks((int)most) > (1 << 30)) break;
          for (bool same : {false, true}) {
            const ckv::AttendPlan p = ckv::attend_plan(units, (int)most, same, n_cu);
            for (int kind = 0; kind < 6; ++kind) {
              long long blocks = 0;
              for (int b = 0; b < batch; ++b) {
                length[b] = kind == 0 || same ? (int)most : kind == 1 ? 0 : kind == 2 ? random(most + 1) : kind == 3 ? (b ? random(most / 50 + 1) : (int)most)
                          : kind == 4 ? (int)(most / (1 + b % 7)) : (b % 3 ? (int)most : 1);
                blocks += ckv::unit_blocks(length[b]);
              }
              auto pieces = [&](int share) {
                long long n = 0;
                for (int b = 0; b < batch; ++b) n += ckv::unit_parts(ckv::unit_blocks(length[b]), share);
                return n * hkv;
              };
              int share = p.share;
              if (!share) {
                share = ckv::attend_share((int)(blocks * hkv), p.workers);
                for (int i = 0; i < 2 && ckv::enlarges_share(batch, hkv, p.workers); ++i) {
                  const long long all = pieces(share);
                  if (all <= p.workers) break;
                  const int before = share;
                  share = ckv::larger_share(share, (int)all, p.workers);
                  if (share < before) return std::printf("smaller share\n"), 1;
                  ++enlarged;
                }
                if (pieces(share) > p.pieces) return std::printf("%lld pieces, %lld workgroups: %d x %d of up to %lld\n", pieces(share), p.pieces, batch, hkv, most), 1;
                many += batch > 64;
              } else if (units * p.places != p.pieces) {
                return std::printf("%lld workgroups of %lld\n", p.pieces, units * p.places), 1;
              }
              for (int b = 0; b < batch; ++b) {
                const int n = ckv::unit_blocks(length[b]), parts = ckv::unit_parts(n, share);
                if (parts < 1 || parts > n || (parts > 1 && !p.split) || (p.share && parts > p.places)) return std::printf("%d parts of %d blocks\n", parts, n), 1;
                if (kind < 4 && b > 4) continue;
                int at = 0;
                for (int i = 0; i < parts && i < 300; ++i) {
                  const int first = ckv::part_begin(n, parts, i), last = ckv::part_begin(n, parts, i + 1);
                  if (first != at || last <= first || last - first > share || last - first < n / parts) return std::printf("part %d of %d: %d .. %d\n", i, parts, first, last), 1;
                  at = last;
                }
                if (parts <= 300 && at != n) return std::printf("%d of %d blocks\n", at, n), 1;
                cut += parts > 1;
              }
            }
          }
        }
  if (!enlarged || !cut || !many) return std::printf("%lld %lld %lld\n", enlarged, cut, many), 1;""")


# ------------------------------------------------------------------ refusals
@pytest.mark.parametrize("heads,picked,change,said", [
    (7, 0, {}, b"multiple of n_kv_heads"), (0, 0, {}, b"multiple of n_kv_heads"), (34, -1, {}, b"16 query heads"), (8, -2, {}, b"n_picked"), (8, 1 << 27, {}, b"pages picked"),
    (8, 0, dict(batch=1 << 22, columns=1 << 20, table_stride=1 << 20, max_length=1 << 24), b"too many entries")])
def test_a_workspace_s_refusal_says_what_is_wrong(good, heads, picked, change, said):  # noqa: F811
    """Not what another call was refused for before, nor nothing."""
    lib = ckv.load()
    pages, seqs = good[:2]
    for k, v in change.items():
        setattr(seqs, k, v)
    assert lib.ckv_paged_append(None, None, None, None) == ckv.EINVAL and b"NULL" in lib.ckv_last_error(None)
    assert lib.ckv_paged_workspace_bytes(C.addressof(pages), C.addressof(seqs), heads, picked) == 0
    assert said in lib.ckv_last_error(None)


def test_batches_beyond_what_a_launch_takes_are_refused(good):  # noqa: F811
    """2^32 threads on an axis: refused by the host's checks, not by the launch."""
    lib = ckv.load()
    pages, seqs, rows, query = good
    p, s, r, q = (C.addressof(x) for x in good)
    select = lambda: lib.ckv_paged_select(p, s, q, 3, 1, 1, 4096, 4096, 1 << 62, None)  # noqa: E731
    attend = lambda: lib.ckv_paged_attend(p, s, q, 0.1, None, 0, 4096, ckv.BF16, None, 4096, 1 << 62, None)  # noqa: E731
    for batch, columns, calls in ((1 << 23, 4, (lambda: lib.ckv_paged_append(p, s, r, None), lambda: lib.ckv_paged_read(p, s, r, None), attend, select)),
                                  ((1 << 23) - 1, 100, (attend, select)), (1 << 22, 4, (select,)), (1 << 21, 2049, (select,))):
        seqs.batch, seqs.columns, seqs.table_stride, seqs.max_length = batch, columns, columns, 16 * columns
        for call in calls:
            assert call() == ckv.EINVAL, (batch, columns)
            assert b"2^2" in lib.ckv_last_error(None)


def test_scales_whose_product_with_a_logarithm_is_infinite_are_refused(good):  # noqa: F811
    lib = ckv.load()
    p, s, _, q = (C.addressof(x) for x in good)
    for scale in (2.4e38, 3.4e38):
        assert lib.ckv_paged_attend(p, s, q, scale, None, 0, 4096, ckv.BF16, None, 4096, 1 << 30, None) == ckv.EINVAL
        assert b"softmax_scale" in lib.ckv_last_error(None)
