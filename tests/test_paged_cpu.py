"""The cache in pages without a GPU: its definitions, the index arithmetic that kernels use (compiled on its own, also for tables and lengths that
are wrong), and what the entry points refuse."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import paged as ref
from paper_2601_16986_amd import ckv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ------------------------------------------------------------------ definitions
def test_codes_are_the_format_s():
    """Values and roundings against torch's own conversion, at every midpoint between neighbours too."""
    v = torch.arange(256, dtype=torch.int16).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(v, ref.E4M3, equal_nan=True)
    grid = ref.E4M3[:127]
    x = np.concatenate([grid, (grid[1:] + grid[:-1]) / 2, np.nextafter((grid[1:] + grid[:-1]) / 2, 0), np.nextafter((grid[1:] + grid[:-1]) / 2, 999)])
    x = np.concatenate([x, -x]).astype(np.float32)
    assert np.array_equal(ref.e4m3_codes(x.astype(np.float64)), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


@pytest.mark.parametrize("big,e", [(448.0, 0), (449.0, 1), (896.0, 1), (1.0, -8), (1.75, -8), (1.76, -7), (0.0, -100), (3e38, 120), (1e-36, -100), (2.0 ** -92, -100), (2.0 ** -91, -99)])
def test_exponent_is_the_smallest_that_fits(big, e):
    x = np.zeros((1, 128))
    x[0, 5] = -big
    codes, got = ref.quantise(x)
    assert got[0] == e
    assert abs(ref.dequantise(codes, got)[0, 5] + big) <= max(2.0 ** -4 * big, 2.0 ** -110)


def test_picking_by_hand():
    s = np.array([0, 5, 1, 5, np.nan, -np.inf, 3, 9], np.float32)
    assert ref.pick(s, 4, 1, 1).tolist() == [0, 1, 4, 7]          # the first, the last, what is no number, the lower of two equals
    assert ref.pick(s, 3, 0, 0).tolist() == [1, 4, 7]
    assert ref.pick(s, 10, 1, 1).tolist() == [0, 1, 2, 3, 4, 5, 6, 7, -1, -1]
    assert ref.pick(s, 2, 1, 1).tolist() == [0, 7]


def test_attention_by_hand():
    k, v = np.zeros((2, 128)), np.zeros((2, 128))
    k[0, 0], v[0, 0], v[1, 0] = 2.0, 1.0, 3.0
    q = np.zeros(128)
    q[0] = 1.5
    o, lse, _, _ = ref.attend(q, k, v, 1.0)
    w = 1 / (1 + np.exp(-3.0))
    assert np.isclose(o[0], w + 3 * (1 - w)) and np.isclose(lse, np.log(np.exp(3.0) + 1))
    assert ref.attend(q, k[:0], v[:0], 1.0)[1] == -np.inf


# ------------------------------------------------------------------ index arithmetic
def _run(tmp_path, body):
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("no host compiler")
    src, exe = tmp_path / "paged.cpp", tmp_path / "paged"
    src.write_text('#include <climits>\n#include <cstdio>\n#include <initializer_list>\n#include "ckv_paged.h"\nint main() {\n' + body + "\n  return 0;\n}\n")
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "paper_2601_16986_amd", "csrc"),
                    str(src), "-o", str(exe)], check=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0, res.stdout + res.stderr


def test_pages_that_a_table_names_are_in_the_pool(tmp_path):
    _run(tmp_path, r"""
  for (int n : {1, 5, 1000, INT_MAX})
    for (int page : {INT_MIN, -7, -1, 0, 4, 5, 999, 1000, INT_MAX - 1, INT_MAX})
      if (ckv::page_there(page, n) != (page >= 0 && page < n)) return std::printf("page %d of %d\n", page, n), 1;
  for (int shift = 4; shift <= 8; ++shift)
    for (int length : {0, 1, 15, 16, 17, 255, 256, 257, 1 << 30})
      for (int page : {0, 1, 2, 15, 16, 17, (1 << 30) >> shift, INT_MAX}) {
        const long long left = length - ((long long)page << shift);
        const int want = left <= 0 ? 0 : left > (1 << shift) ? 1 << shift : (int)left;
        if (ckv::page_fill(length, page, shift) != want) return std::printf("length %d page %d of %d\n", length, page, 1 << shift), 1;
      }""")


def test_rows_of_a_call_lie_within_the_sequence_and_the_caller_s_rows(tmp_path):
    _run(tmp_path, r"""
  const int far[] = {INT_MIN, -5, -1, 0, 1, 7, 63, 64, 65, 1 << 30, INT_MAX};
  for (int length : {0, 1, 7, 64, 1 << 30})
    for (int most : {1, 7, 64, 1 << 30})
      for (int has = 0; has < 2; ++has)
        for (int first : far)
          for (int packed = 0; packed < 2; ++packed)
            for (int start : far)
              for (int stop : far)
                for (int total : {0, 7, 64, 1 << 30}) {
                  const ckv::RowSpan s = ckv::row_span(length, most, has, first, packed, start, stop, total);
                  if (s.count < 0 || s.first < 0 || s.count > most || (long long)s.first + s.count > length) return std::printf("outside the sequence\n"), 1;
                  if (packed && s.count > 0 && (start < 0 || (long long)start + s.count > total || start + s.count > stop)) return std::printf("outside the rows\n"), 1;
                  const bool bad = (has && (first < 0 || first > length)) || (packed && (start < 0 || stop < start || stop > total));
                  if (s.bad != bad || (bad && s.count)) return std::printf("bad rows not seen\n"), 1;
                  if (!bad && !packed && !has && s.count != (length < most ? length : most)) return std::printf("rows lost\n"), 1;
                }""")


def test_pieces_of_an_attention_have_their_places(tmp_path):
    """Whatever the lengths turn out to be, there are as many workgroups as pieces, and parts of the workspace for each."""
    _run(tmp_path, r"""
  unsigned seed = 1;
  auto random = [&](int n) { seed = seed * 1664525u + 1013904223u; return (int)((seed >> 8) % (unsigned)n); };
  for (long long units = 1; units < 5000; units = units * 3 / 2 + 1)
    for (long long most = 0; most <= (1 << 30) && units * ckv::unit_blocks((int)most) <= (1 << 30); most = most * 3 / 2 + 1)
      for (bool same : {false, true}) {
        const ckv::AttendPlan p = ckv::attend_plan(units, (int)most, same, 256);
        if (p.pieces < units || p.pieces > 2 * 1024 + 2 * units) return std::printf("%lld pieces of %lld units\n", p.pieces, units), 1;
        for (int kind = 0; kind < 4; ++kind) {
          long long pieces = 0, blocks = 0;
          const int n = units < 100 ? (int)units : 100;          // units of so many lengths, each as often as the others
          int length[100];
          for (int i = 0; i < n; ++i) {
            length[i] = kind == 0 || same ? (int)most : kind == 1 ? 0 : kind == 2 ? random((int)most + 1) : i ? random((int)most / 50 + 1) : (int)most;
            blocks += ckv::unit_blocks(length[i]);
          }
          if (n < units) continue;
          const int share = p.share ? p.share : ckv::attend_share((int)blocks, p.workers);
          for (int i = 0; i < n; ++i) {
            const int parts = ckv::unit_parts(ckv::unit_blocks(length[i]), share);
            if (parts < 1 || (parts > 1 && !p.split) || (p.share && parts > p.places)) return std::printf("%d parts\n", parts), 1;
            pieces += p.share ? p.places : parts;
          }
          if (pieces > p.pieces) return std::printf("%lld pieces, %lld places, %lld units of up to %lld\n", pieces, p.pieces, units, most), 1;
        }
      }""")


# ------------------------------------------------------------------ refusals
@pytest.fixture()
def good():
    """Arguments that are in order, on addresses that nothing looks at."""
    n = 16 * 128
    pages = ckv.Pages(10, 16, 2, 128, ckv.E4M3, 2 * n, n, 128, 64, 32, 512, 256, 4096, 8192, 4096, 4096, None)
    seqs = ckv.Seqs(4096, 4096, 4, 3, 4, 64)
    rows = ckv.Rows(4096, 4096, None, None, 8 * 256, 256, 128, 8, 0)
    query = ckv.Query(4096, 8 * 128, 128, 8)
    return pages, seqs, rows, query


def _calls(pages, seqs, rows, query, only=None):
    lib, p, s, r, q = ckv.load(), C.addressof(pages), C.addressof(seqs), C.addressof(rows), C.addressof(query)
    calls = {"append": lambda: lib.ckv_paged_append(p, s, r, None), "read": lambda: lib.ckv_paged_read(p, s, r, None),
             "attend": lambda: lib.ckv_paged_attend(p, s, q, 0.1, None, 0, 4096, ckv.BF16, None, 4096, 1 << 30, None),
             "select": lambda: lib.ckv_paged_select(p, s, q, 3, 1, 1, 4096, 4096, 1 << 30, None)}
    return {k: f() for k, f in calls.items() if only is None or k in only}


ALL = ("append", "read", "attend", "select")


@pytest.mark.parametrize("field,bad", [
    ("n_pages", 0), ("page_size", 8), ("page_size", 48), ("page_size", 512), ("n_kv_heads", 0), ("head_dim", 64), ("dtype", ckv.F32), ("dtype", 0), ("k", None), ("v", 4104),
    ("page_stride", 0), ("page_stride", -2048), ("head_stride", 120), ("slot_stride", 136 + 4), ("slot_stride", 1 << 28), ("page_stride", 1 << 41), ("scales", None), ("scales", 4100),
    ("scale_page_stride", 30), ("scale_head_stride", 36), ("bounds", 4104), ("bounds_page_stride", 128), ("bounds_head_stride", 260)])
def test_pools_that_are_refused(good, field, bad):
    setattr(good[0], field, bad)
    assert set(_calls(*good).values()) == {ckv.EINVAL}
    assert ckv.load().ckv_last_error(None) != b""
    assert ckv.load().ckv_paged_workspace_bytes(C.addressof(good[0]), C.addressof(good[1]), 8, 0) == 0


@pytest.mark.parametrize("field,bad", [("table", None), ("lengths", None), ("batch", 0), ("columns", 0), ("table_stride", 3), ("max_length", -1), ("max_length", 65), ("batch", 1 << 24)])
def test_sequences_that_are_refused(good, field, bad):
    setattr(good[1], field, bad)
    assert set(_calls(*good).values()) == {ckv.EINVAL}


@pytest.mark.parametrize("field,bad", [("k", None), ("v", 4098), ("rows", 0), ("rows", -1), ("row_stride", 0), ("row_stride", 260), ("head_stride", 64), ("seq_stride", -256)])
def test_rows_that_are_refused(good, field, bad):
    setattr(good[2], field, bad)
    assert set(_calls(*good, only=("append", "read")).values()) == {ckv.EINVAL}


@pytest.mark.parametrize("field,bad", [("q", None), ("q", 4104), ("n_q_heads", 7), ("n_q_heads", 0), ("n_q_heads", 34), ("seq_stride", 0), ("head_stride", 132)])
def test_queries_that_are_refused(good, field, bad):
    setattr(good[3], field, bad)
    assert set(_calls(*good, only=("attend", "select")).values()) == {ckv.EINVAL}


def test_other_arguments_that_are_refused(good):
    lib = ckv.load()
    p, s, r, q = (C.addressof(x) for x in good)

    def attend(scale=0.1, picked=None, n=0, out=4096, dtype=ckv.BF16, work=4096, size=1 << 30):
        return lib.ckv_paged_attend(p, s, q, scale, picked, n, out, dtype, None, work, size, None)

    def select(keep=3, first=1, last=1, picked=4096, work=4096, size=1 << 30):
        return lib.ckv_paged_select(p, s, q, keep, first, last, picked, work, size, None)

    assert {attend(scale=0.0), attend(scale=float("nan")), attend(scale=float("inf")), attend(n=4), attend(picked=4096), attend(picked=4096, n=-1), attend(picked=4096, n=1 << 27),
            attend(out=None), attend(out=4100), attend(dtype=ckv.E4M3)} == {ckv.EINVAL}
    assert {select(keep=0), select(keep=1), select(first=-1), select(last=-1), select(first=4, last=0), select(first=2 ** 31 - 1, last=2 ** 31 - 1), select(picked=None), select(keep=40000)} == {ckv.EINVAL}
    good[0].bounds = None
    assert select() == ckv.EINVAL
    good[0].bounds = 4096
    good[1].columns, good[1].table_stride, good[1].max_length = 40000, 40000, 640000
    assert {attend(work=None), attend(work=4100), attend(size=256)} == {ckv.EWORKSPACE}
    assert select() == ckv.EINVAL                                   # more pages than a selection takes
    good[1].max_length = 16 * 32768
    assert {select(work=None), select(size=1024), select(work=4352 + 8)} == {ckv.EWORKSPACE}
    for args in ((None, s, r), (p, None, r), (p, s, None)):
        assert lib.ckv_paged_append(*args, None) == ckv.EINVAL and lib.ckv_paged_read(*args, None) == ckv.EINVAL
    assert lib.ckv_paged_workspace_bytes(p, s, 7, 0) == 0 and lib.ckv_paged_workspace_bytes(p, s, 8, -2) == 0 and lib.ckv_paged_workspace_bytes(p, s, 8, -1) == 4 * 6 * 32768


def test_pools_of_the_binding_that_are_refused():
    k = torch.zeros((3, 2, 16, 128), dtype=torch.bfloat16)
    c = k.to(torch.float8_e4m3fn)
    scales, bounds = torch.zeros((3, 2, 16, 2), dtype=torch.uint8), torch.zeros((3, 2, 2, 128), dtype=torch.bfloat16)
    for args in (dict(k=k.float(), v=k.float()), dict(k=k, v=k[:2]), dict(k=k, v=k.transpose(1, 2).contiguous().transpose(1, 2)), dict(k=k, v=k, scales=scales), dict(k=c, v=c),
                 dict(k=c, v=c, scales=scales[:2]), dict(k=c, v=c, scales=scales.float()), dict(k=k, v=k, bounds=bounds.float()), dict(k=k, v=k, bounds=bounds[:, :1]),
                 dict(k=k[0], v=k[0]), dict(k=k, v=k)):                # the last is in order, but not on a GPU
        with pytest.raises(ckv.CkvError):
            ckv.PagedCache(**args)
