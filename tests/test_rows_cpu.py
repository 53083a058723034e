"""Several rows per sequence of a cache in pages without a GPU: what the definitions say of small cases, the index arithmetic of the kernels (compiled on its own), and what the entry points refuse."""
import ctypes as C
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

from oracle import paged as ref
from paper_2601_16986_amd import ckv
from tests.test_kernel_resources_cpu import _tool
from tests.test_paged_cpu import good  # noqa: F401


# ------------------------------------------------------------------ definitions
def test_turning_by_hand():
    x = np.zeros((1, 1, 128))
    x[0, 0, [0, 1, 8, 9, 16]] = 1.0, 2.0, 3.0, 4.0, 5.0
    f = np.zeros(8)
    f[:2] = np.pi / 2, np.pi / 4
    y = ref.rotate(x, np.array([1]), f, magnitude=2.0)[0, 0]                     # dimensions 0 and 8 by a quarter, 1 and 9 by two eighths at position 1
    r = np.sqrt(0.5)
    assert np.allclose(y[[0, 8, 1, 9, 16]], [-6, 2, 2 * (2 * r - 4 * r), 2 * (4 * r + 2 * r), 5])
    y = ref.rotate(x, np.array([2]), f, interleaved=True)[0, 0]                  # 0 and 1 by a half
    assert np.allclose(y[[0, 1, 8, 9, 16]], [-1, -2, 3, 4, 5])
    assert np.array_equal(ref.rotate(x, np.array([0]), f), x)


def test_what_rows_see_by_hand():
    assert ref.sees(2, 2).astype(int).tolist() == [[1, 1, 1, 0], [1, 1, 1, 1]]
    assert ref.sees(4, 2, window=2).astype(int).tolist() == [[0, 0, 0, 1, 1, 0], [0, 0, 0, 0, 1, 1]]
    assert ref.sees(4, 2, window=2, sinks=1).astype(int).tolist() == [[1, 0, 0, 1, 1, 0], [1, 0, 0, 0, 1, 1]]
    assert ref.sees(0, 2, window=1, sinks=9).astype(int).tolist() == [[1, 0], [1, 1]]       # a sink that is yet to come is not seen
    tree = [[1, 0, 0], [1, 1, 0], [1, 0, 1]]
    assert ref.sees(2, 3, tree=tree).astype(int).tolist() == [[1, 1, 1, 0, 0], [1, 1, 1, 1, 0], [1, 1, 1, 0, 1]]
    # both children stand at position 3: of the four entries before them and themselves a window of 3 leaves out the first
    assert ref.sees(2, 3, window=3, tree=tree).astype(int).tolist() == [[1, 1, 1, 0, 0], [0, 1, 1, 1, 0], [0, 1, 1, 0, 1]]


def test_rows_of_a_full_mask_are_what_one_token_gets():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((3, 128)), rng.standard_normal((20, 128)), rng.standard_normal((20, 128))
    o, lse, _, _ = ref.attend_rows(q, k, v, np.ones((3, 20), bool), 0.1)
    for i in range(3):
        one = ref.attend(q[i], k, v, 0.1)
        assert np.allclose(o[i], one[0], rtol=1e-12, atol=0) and np.isclose(lse[i], one[1])
    o, lse, _, _ = ref.attend_rows(q, k, v, np.zeros((3, 20), bool), 0.1)
    assert not o.any() and np.isneginf(lse).all()


# ------------------------------------------------------------------ index arithmetic
def _run(tmp_path, body):
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("no host compiler")
    src, exe = tmp_path / "rows.cpp", tmp_path / "rows"
    src.write_text('#include <climits>\n#include <cstdio>\n#include <initializer_list>\n#include <vector>\n#include "ckv_rows.h"\nint main() {\n' + body + "\n  return 0;\n}\n")
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2601_16986_amd", "csrc")
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined,address", "-fno-sanitize-recover=all", "-I", include, str(src), "-o", str(exe)], check=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0, res.stdout + res.stderr


def test_tiles_of_a_block_hold_what_its_rows_see(tmp_path):
    """Every entry of the window's and the sinks' in one tile, ascending, none twice, and no tile without one."""
    _run(tmp_path, r"""
  for (int size : {32, 64, 128})
    for (int end : {0, 1, 31, 32, 33, 64, 100, 128, 129, 400, 1000})
      for (int oldest : {0, 1, 5, 31, 32, 33, 63, 64, 65, 100, 127, 128, 300, 999})
        for (int sinks : {0, 1, 4, 31, 32, 33, 100, 128, 500, INT_MAX}) {
          const ckv::RowTiles t = ckv::row_tiles(oldest, end, sinks, size);
          std::vector<int> in(end + 1, 0);
          int before = -1;
          for (int n = 0; n < t.count; ++n) {
            const int at = t.tile(n);
            bool any = false;
            if (at <= before) return std::printf("tile %d after %d\n", at, before), 1;
            before = at;
            for (int e = at * size; e < (at + 1) * size; ++e)
              if (e < end) ++in[e], any = any || e >= oldest || e < sinks;
            if (!any && oldest < end) return std::printf("size %d end %d oldest %d sinks %d: tile %d for nothing\n", size, end, oldest, sinks, at), 1;
          }
          for (int e = 0; e < end; ++e)
            if (in[e] > 1 || ((e >= oldest || e < sinks) && !in[e])) return std::printf("size %d end %d oldest %d sinks %d: entry %d in %d tiles\n", size, end, oldest, sinks, e, in[e]), 1;
        }
  const ckv::RowTiles far = ckv::row_tiles(INT_MAX - 5, INT_MAX, INT_MAX, 32);
  if (far.count < 1) return 1;""")


def test_bits_of_entries_between_two(tmp_path):
    _run(tmp_path, r"""
  for (long long e0 : {0ll, 1ll, 64ll, 1000ll, (1ll << 31) - 40})
    for (long long lo = e0 - 70; lo < e0 + 70; lo += 3)
      for (long long hi = lo - 3; hi < lo + 140; hi += 7) {
        const unsigned long long bits = ckv::bits_between(e0, lo, hi);
        for (int i = 0; i < 64; ++i)
          if ((int)(bits >> i & 1) != (e0 + i >= lo && e0 + i < hi)) return std::printf("%lld: %lld .. %lld bit %d\n", e0, lo, hi, i), 1;
      }""")


def test_every_block_of_rows_has_one_workgroup(tmp_path):
    """Whatever the numbers of units and blocks; a unit's blocks go to one of the chip's eight parts as long as units make full rounds."""
    _run(tmp_path, r"""
  for (unsigned units : {1u, 2u, 7u, 8u, 9u, 15u, 16u, 63u, 64u, 100u, 257u})
    for (unsigned each : {1u, 2u, 3u, 8u, 13u, 64u}) {
      const unsigned grid = ckv::rows_grid(units, each);
      if (grid < units * each || grid >= units * each + 8 || grid != (unsigned)ckv::rows_grid<long long>(units, each)) return std::printf("grid %u\n", grid), 1;
      std::vector<int> seen(units * each, 0);
      for (unsigned i = 0; i < grid; ++i) {
        const unsigned piece = ckv::rows_piece(i, units, each);
        if (ckv::rows_piece<long long>(i, units, each) != (piece == ~0u ? -1ll : (long long)piece)) return std::printf("two numbers for %u\n", i), 1;
        if (piece == ~0u) continue;
        if (piece >= units * each || seen[piece]++) return std::printf("%u units of %u: %u twice or none\n", units, each, piece), 1;
        if (piece / each < units / 8 * 8 && piece / each % 8 != i % 8) return std::printf("unit %u on part %u\n", piece / each, i % 8), 1;
      }
      for (int n : seen)
        if (n != 1) return std::printf("%u units of %u: a block left out\n", units, each), 1;
    }""")


def test_every_piece_has_a_group(tmp_path):
    """All units' first pieces come before all second ones; few units' pieces go round the chip's eight parts, those of many that make full rounds stay on one."""
    _run(tmp_path, r"""
  for (unsigned units : {1u, 2u, 3u, 7u, 8u, 9u, 12u, 16u, 64u, 100u, 255u})
    for (unsigned places : {1u, 2u, 8u, 9u, 24u}) {
      std::vector<int> on(units * places, -1);
      for (unsigned g = 0; g < units * places; ++g) {
        const ckv::RowsGroup r = ckv::rows_group(g, units);
        if (r.part != g / units || r.unit >= units || on[r.part * units + r.unit] >= 0) return std::printf("group %u of %u\n", g, units), 1;
        on[r.part * units + r.unit] = (int)(g % 8);
      }
      for (unsigned u = 0; u < units; ++u)
        for (unsigned i = 1; i < places; ++i)
          if ((on[i * units + u] == on[(i - 1) * units + u]) != (units % 8 == 0 && units > 8)) return std::printf("%u units: piece %u of %u\n", units, i, u), 1;
    }""")


def test_pieces_fit_their_places(tmp_path):
    """Whatever share the lengths lead to, a block has no more pieces than places, they are its tiles one after another, and a call has not many more workgroups than find room."""
    _run(tmp_path, r"""
  for (long long units : {1, 4, 8, 32, 100, 256, 1000, 5000})
    for (int rows : {1, 2, 7, 8, 31, 64, 500, 9000})
      for (int group : {1, 4, 5, 16})
        for (int entries : {1, 20, 700, 9350, 131072, 1 << 30}) {
          const ckv::RowsPlan p = ckv::rows_plan(units, rows, group, entries, 256);
          const int each = 32 * p.wide, size = ckv::rows_tile(p.wide);
          if ((long long)p.blocks * each < (long long)rows * group || (long long)(p.blocks - 1) * each >= (long long)rows * group) return std::printf("blocks\n"), 1;
          if (each < 128 && p.blocks != 1) return std::printf("narrow blocks though there are more rows\n"), 1;
          if (p.places < 1 || p.least < 1 || p.pieces != units * p.blocks * p.places) return std::printf("places\n"), 1;
          if (p.places > 1 && p.pieces > 4 * 256 + 2 * units * p.blocks) return std::printf("%lld pieces of %lld blocks\n", p.pieces, units * p.blocks), 1;
          for (int tiles : {1, 2, 3, 30, entries / size + 2})
            for (int share : {1, 2, 5, 100, INT_MAX}) {
              const int s = ckv::rows_share(tiles, share, p.places), parts = ckv::unit_parts(tiles, s);
              if (parts < 1 || parts > p.places) return std::printf("%d tiles, share %d, places %d: %d parts\n", tiles, share, p.places, parts), 1;
              int at = 0;
              for (int i = 0; i < parts; ++i) {
                if (ckv::part_begin(tiles, parts, i) != at) return std::printf("a gap\n"), 1;
                at = ckv::part_begin(tiles, parts, i + 1);
                if (at <= ckv::part_begin(tiles, parts, i)) return std::printf("a piece of nothing\n"), 1;
              }
              if (at != tiles) return std::printf("tiles left out\n"), 1;
            }
        }""")


def test_a_page_s_heads_are_shared_where_pages_are_few(tmp_path):
    _run(tmp_path, r"""
  for (long long pages : {1ll, 3ll, 32ll, 128ll, 129ll, 256ll, 257ll, 1ll << 40})
    for (int rows : {1, 16, 17, 64, 1 << 30})
      for (int group : {1, 4, 16}) {
        const int by = ckv::turned_by(pages, rows, group, 256);
        if (by < 1 || by > group + 1 || (by > 1 && (rows <= 16 || pages * by > 256))) return std::printf("%d for %lld pages\n", by, pages), 1;
      }
  if (ckv::turned_by(32, 64, 7, 256) != 8 || ckv::turned_by(200, 64, 7, 256) != 1) return 1;""")


def test_two_workgroups_find_room_on_a_compute_unit(tmp_path):
    """Of its 160 KB of LDS and 512 registers a lane of each SIMD, as the share of a call's pieces counts on."""
    fat, part, co = (str(tmp_path / x) for x in ("fat", "part", "co"))
    subprocess.run([_tool("llvm-objcopy"), f"--dump-section=.hip_fatbin={fat}", ckv.LIB_PATH, str(tmp_path / "copy.so")], check=True)
    with open(fat, "rb") as f:
        bundles = f.read().split(b"__CLANG_OFFLOAD_BUNDLE__")[1:]         # one of each source
    got = {}
    for bundle in bundles:
        with open(part, "wb") as f:
            f.write(b"__CLANG_OFFLOAD_BUNDLE__" + bundle)
        subprocess.run([_tool("clang-offload-bundler"), "--type=o", "--unbundle", f"--input={part}", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", f"--output={co}"], check=True)
        notes = subprocess.run([_tool("llvm-readelf"), "--notes", co], check=True, capture_output=True, text=True).stdout
        for block in re.split(r"\n  - ", notes):
            name = re.search(r"\.name:\s+(_Z\S+)", block)
            if name and "paged_rows_kernel" in name.group(1):
                got[name.group(1)] = {k: int(v) for k, v in re.findall(r"\.(\w+):\s+(\d+)$", block, re.M)}
    assert len(got) == 8
    for n, k in got.items():
        assert k["group_segment_fixed_size"] <= 80 * 1024 and k["vgpr_count"] <= 256, n


# ------------------------------------------------------------------ refusals
def _rotated(g, positions=None, q=None, out=None, rotation=None):
    r = rotation or ckv.RotationParams(4096, 64, 0, 1.0)
    return ckv.load().ckv_paged_append_rotated(*(C.addressof(x) for x in g[:3]), C.addressof(r), positions, C.addressof(q) if q else None, C.addressof(out) if out else None, None)


def _heads(**how):
    h = ckv.Heads(4096, 8 * 1024, 1024, 128, 8)
    for k, v in how.items():
        setattr(h, k, v)
    return h


def _attend(g, queries=None, mask=None, scale=0.1, out=4096, dtype=ckv.BF16, work=4096, size=1 << 40):
    q, m = queries or _queries(), mask or ckv.Mask(0, 0, None, 0, 0)
    return ckv.load().ckv_paged_attend_rows(C.addressof(g[0]), C.addressof(g[1]), C.addressof(q), C.addressof(m), scale, out, dtype, None, work, size, None)


def _queries(**how):
    q = ckv.RowQueries(4096, None, None, 8 * 1024, 1024, 128, 8, 0, 8)
    for k, v in how.items():
        setattr(q, k, v)
    return q


def _bytes(g, rows=8, heads=8, mask=None):
    m = mask or ckv.Mask(0, 0, None, 0, 0)               # held until the call is over
    return ckv.load().ckv_paged_rows_workspace_bytes(C.addressof(g[0]), C.addressof(g[1]), rows, heads, C.addressof(m))


POOLS = [("n_pages", 0), ("page_size", 48), ("dtype", 0), ("k", None), ("page_stride", 0), ("scales", None)]
SEQS = [("table", None), ("lengths", None), ("batch", 0), ("columns", 0), ("max_length", 65), ("batch", 1 << 24)]


@pytest.mark.parametrize("which,field,bad", [(0, *x) for x in POOLS] + [(1, *x) for x in SEQS])
def test_pools_and_sequences_that_are_refused(good, which, field, bad):
    setattr(good[which], field, bad)
    assert _rotated(good) == _rotated(good, q=_heads(), out=_heads()) == _attend(good) == ckv.EINVAL
    assert _bytes(good) == 0 and ckv.load().ckv_last_error(None) != b""


@pytest.mark.parametrize("field,bad", [("k", None), ("v", 4098), ("rows", 0), ("row_stride", 260), ("head_stride", 64), ("seq_stride", -256)])
def test_rows_to_be_turned_that_are_refused(good, field, bad):
    setattr(good[2], field, bad)
    assert _rotated(good) == ckv.EINVAL


@pytest.mark.parametrize("field,bad", [("frequencies", None), ("frequencies", 4100), ("n_pairs", 0), ("n_pairs", 4), ("n_pairs", 12), ("n_pairs", 72), ("n_pairs", -8), ("interleaved", 2), ("interleaved", -1),
                                       ("magnitude", 0.0), ("magnitude", -1.0), ("magnitude", float("nan")), ("magnitude", float("inf"))])
def test_rotations_that_are_refused(good, field, bad):
    r = ckv.RotationParams(4096, 64, 0, 1.0)
    setattr(r, field, bad)
    assert _rotated(good, rotation=r) == ckv.EINVAL
    lib = ckv.load()
    assert lib.ckv_paged_append_rotated(*(C.addressof(x) for x in good[:3]), None, None, None, None, None) == ckv.EINVAL


@pytest.mark.parametrize("field,bad", [("q", None), ("q", 4104), ("n_q_heads", 7), ("n_q_heads", 0), ("n_q_heads", 34), ("seq_stride", 0), ("row_stride", 64), ("row_stride", 1028), ("head_stride", 132)])
def test_heads_to_be_turned_that_are_refused(good, field, bad):
    assert _rotated(good, q=_heads(**{field: bad}), out=_heads()) == ckv.EINVAL
    assert _rotated(good, q=_heads(), out=_heads(**{field: bad})) == ckv.EINVAL
    assert _rotated(good, q=_heads()) == _rotated(good, out=_heads()) == _rotated(good, q=_heads(), out=_heads(n_q_heads=4)) == ckv.EINVAL


@pytest.mark.parametrize("field,bad", [("q", None), ("q", 4104), ("n_q_heads", 7), ("n_q_heads", 0), ("n_q_heads", 34), ("rows", 0), ("rows", -3), ("rows", (1 << 30) + 1), ("seq_stride", 0), ("row_stride", 64),
                                       ("head_stride", 132)])
def test_row_queries_that_are_refused(good, field, bad):
    assert _attend(good, _queries(**{field: bad})) == ckv.EINVAL
    assert _attend(good, _queries(starts=4096, total=-1)) == ckv.EINVAL


@pytest.mark.parametrize("mask,rows", [((-1, 0, None, 0, 0), 8), ((4, -1, None, 0, 0), 8), ((0, 4, None, 0, 0), 8), ((0, 0, 4096, 64, 7), 8), ((0, 0, 4096, -1, 8), 8), ((7, 0, 4096, 64, 8), 8),
                                       ((0, 0, 4096, 0, 513), 513), ((0, 0, 4096, 1 << 62, 8), 8), ((0, 0, 4096, 64, 1 << 62), 8)])
def test_masks_that_are_refused(good, mask, rows):
    m = ckv.Mask(*mask)
    assert _attend(good, _queries(rows=rows), m) == ckv.EINVAL and _bytes(good, rows, 8, m) == 0


def test_other_arguments_of_an_attention_of_rows(good):
    lib = ckv.load()
    assert {_attend(good, scale=0.0), _attend(good, scale=float("nan")), _attend(good, scale=float("inf")), _attend(good, scale=-1.0), _attend(good, out=None), _attend(good, out=4100),
            _attend(good, dtype=ckv.E4M3), _attend(good, dtype=0)} == {ckv.EINVAL}
    queries, mask = _queries(), ckv.Mask(0, 0, None, 0, 0)
    p, s, q, m = (C.addressof(x) for x in (good[0], good[1], queries, mask))
    for args in ((None, s, q, m), (p, None, q, m), (p, s, None, m), (p, s, q, None)):
        assert lib.ckv_paged_attend_rows(*args, 0.1, 4096, ckv.BF16, None, 4096, 1 << 40, None) == ckv.EINVAL
    assert lib.ckv_paged_rows_workspace_bytes(p, s, 8, 8, None) == 0
    good[1].columns, good[1].table_stride, good[1].max_length = 40000, 40000, 640000
    n = _bytes(good)
    assert n > 256 and n % 256 == 0
    assert {_attend(good, work=None), _attend(good, work=4100), _attend(good, size=n - 1)} == {ckv.EWORKSPACE}
    good[1].max_length = 1 << 30
    good[1].columns = good[1].table_stride = 1 << 26
    assert _attend(good, _queries(rows=1 << 30)) == ckv.EINVAL         # 2^30 rows of 4 heads


def test_calls_with_nothing_to_do_are_not_launched(good):
    """A call whose sequences have no entries, or that has no packed rows, returns without looking at a device."""
    assert _attend(good, _queries(starts=4096, total=0)) == ckv.OK
    good[2].starts, good[2].total = 4096, 0
    assert _rotated(good) == ckv.OK
    good[1].max_length = 0
    assert _attend(good) == ckv.OK and _rotated(good) == ckv.OK
