"""Where the rows of a call go in a cache in pages, and what a page's extremes cover: packed rows without their positions, lengths beyond the most that the
call was told, rows written again."""
import numpy as np
import pytest
import torch

from oracle import paged as ref
from tests.paged import DEV, Filled, bf16, device
from paper_2601_16986_amd import ckv

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _raw(cache):
    """Every byte that an append may write."""
    return [x.view(torch.uint8).clone() for x in (cache.k, cache.v)] + [x.clone() for x in (cache.scales,) if x is not None] + [cache.bounds.view(torch.int16).clone()]


def _check_rows(f, rows):
    """f's sequences hold `rows[side][b]`, [length][heads][128], in 8 bits as those become."""
    for b, n in enumerate(f.lengths):
        k, v = f.cache.read(f.cache.sequences(f.seqs.table[b:b + 1], f.seqs.lengths[b:b + 1]), max(n, 1), first=_ints([0]))
        for side, got in enumerate((k, v)):
            for h in range(f.hkv):
                assert np.array_equal(got[0, :n, h].double().cpu().numpy(), f.held(rows[side][b][:n, h])), f"sequence {b} head {h}"


def _check_bounds(f, rows):
    bounds = f.cache.bounds.double().cpu().numpy()
    for b, n in enumerate(f.lengths):
        for c in range(-(-n // f.ps)):
            for h in range(f.hkv):
                lo, hi = ref.extremes(f.held(rows[0][b][c * f.ps:min(n, (c + 1) * f.ps), h]))
                got = bounds[f.table[b, c], h]
                assert np.array_equal(got[0], lo) and np.array_equal(got[1], hi), f"sequence {b} page {c} head {h}"


# ------------------------------------------------------------------ packed rows without `first`
@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("ps", [16, 64])
def test_packed_rows_are_the_last_of_their_sequences(e4m3, ps):
    """Chunks of other lengths than the call's `rows` behind entries that are there: what was there stays, each sequence's rows come last."""
    lengths, new = [100, 37, 64, 200, 5], [3, 0, 10, 40, 5]
    f = Filled(lengths, 2, ps, e4m3, seed=3)
    rows = [[x[b, :n].copy() for b, n in enumerate(lengths)] for x in f.rows]
    chunk = [bf16(f.rng.standard_normal((sum(new), 2, 128))) for _ in range(2)]
    starts = np.cumsum([0] + new).tolist()
    for side in (0, 1):
        for b, m in enumerate(new):
            rows[side][b][lengths[b] - m:] = chunk[side][starts[b]:starts[b + 1]]
    for most in (40, 150):                              # `rows` as launches need it, and more than some sequences hold
        f.cache.append(f.seqs, *(device(x) for x in chunk), rows=most, starts=_ints(starts))
        assert f.cache.status() == 0
        _check_rows(f, rows)
        out = tuple(torch.full((sum(new) + 2, 2, 128), 5.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        f.cache.read(f.seqs, most, starts=_ints(starts), out=out)
        for side in (0, 1):
            for h in range(2):
                assert np.array_equal(out[side][:-2, h].double().cpu().numpy(), f.held(chunk[side][:, h]))
            assert (out[side][-2:] == 5.0).all()


def test_packed_rows_of_more_than_a_sequence_holds():
    """As with padded rows: they begin at position 0, those behind the length are left out."""
    f = Filled([6, 20], 1, 16, True, seed=4)
    rows = [[x[b, :n].copy() for b, n in enumerate(f.lengths)] for x in f.rows]
    chunk = [bf16(f.rng.standard_normal((12, 1, 128))) for _ in range(2)]
    f.cache.append(f.seqs, *(device(x) for x in chunk), rows=9, starts=_ints([0, 9, 12]))
    for side in (0, 1):
        rows[side][0][:] = chunk[side][:6]
        rows[side][1][17:] = chunk[side][9:]
    _check_rows(f, rows)


# ------------------------------------------------------------------ lengths beyond max_length
@pytest.mark.parametrize("e4m3", [True, False])
def test_rows_behind_the_largest_length_are_left_out(e4m3):
    """A sequence that outgrew what the call was told: positions below the limit get their rows, the others' go nowhere, and no row moves."""
    f = Filled([48, 30], 2, 16, e4m3, seed=5)
    s = f.cache.sequences(f.seqs.table, f.seqs.lengths, 48)
    one = [bf16(f.rng.standard_normal((2, 2, 128))) for _ in range(2)]
    before = _raw(f.cache)
    for far in (49, 60, 10 ** 9, 2 ** 31 - 1):
        f.seqs.lengths.copy_(_ints([far, 0]))
        f.cache.append(s, *(device(x) for x in one))
        assert f.cache.status() == ckv.BAD_LENGTH
        assert all(torch.equal(a, b) for a, b in zip(_raw(f.cache), before)), far
        f.cache.append(s, *(device(x)[:1] for x in one), rows=1, starts=_ints([0, 1, 1]))
        assert f.cache.status() == ckv.BAD_LENGTH
        assert all(torch.equal(a, b) for a, b in zip(_raw(f.cache), before)), far
        f.cache.append(s, *(device(x) for x in one), first=_ints([far - 1, 0]))
        assert f.cache.status() == ckv.BAD_LENGTH
        assert all(torch.equal(a, b) for a, b in zip(_raw(f.cache), before)), far
    # five rows of which two lie below the limit
    five = [bf16(f.rng.standard_normal((2, 5, 2, 128))) for _ in range(2)]
    rows = [[x[b, :n].copy() for b, n in enumerate(f.lengths)] for x in f.rows]
    for side in (0, 1):
        rows[side][0][46:48], rows[side][1][25:30] = five[side][0, :2], five[side][1]
    f.seqs.lengths.copy_(_ints([51, 30]))
    f.cache.append(s, *(device(x) for x in five))
    assert f.cache.status() == ckv.BAD_LENGTH
    f.seqs.lengths.copy_(_ints(f.lengths))
    _check_rows(f, rows)


def test_rows_read_behind_the_largest_length_are_left_alone():
    f = Filled([48, 30], 1, 16, True, seed=6)
    s = f.cache.sequences(f.seqs.table, f.seqs.lengths, 48)
    f.seqs.lengths.copy_(_ints([51, 30]))
    out = tuple(torch.full((2, 5, 1, 128), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    f.cache.read(s, 5, out=out)
    assert f.cache.status() == ckv.BAD_LENGTH
    for side in (0, 1):
        got = out[side].double().cpu().numpy()
        want = (f.k, f.v)[side]
        assert np.array_equal(got[0, :2, 0], want[0][0][46:48]) and (got[0, 2:] == 3.0).all()
        assert np.array_equal(got[1, :, 0], want[1][0][25:30])


# ------------------------------------------------------------------ rows written again
@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("ps,layout", [(16, "plain"), (64, "layers"), (256, "slots_first")])
def test_a_page_s_first_rows_written_again(e4m3, ps, layout):
    """A page's extremes cover its later rows too, however few of them the call writes, in the middle of a sequence and at its end."""
    lengths = [3 * ps + ps // 2 + 1, ps, 2 * ps - 3]
    f = Filled(lengths, 2, ps, e4m3, layout, seed=ps)
    rows = [[x[b, :n].copy() for b, n in enumerate(lengths)] for x in f.rows]
    for count, first in ((1, [0, 0, ps]), (1, [3 * ps, 0, 0]), (ps // 2, [2 * ps, 0, ps]), (ps + 1, [ps, 0, 0])):
        new = [bf16(f.rng.standard_normal((3, count, 2, 128))) for _ in range(2)]
        for side in (0, 1):
            for b in range(3):
                stop = min(lengths[b], first[b] + count)
                rows[side][b][first[b]:stop] = new[side][b, :stop - first[b]]
        f.cache.append(f.seqs, *(device(x) for x in new), first=_ints(first))
        _check_rows(f, rows)
        bounds = f.cache.bounds.double().cpu().numpy()
        for b, n in enumerate(lengths):
            for c in range(-(-n // ps)):
                for h in range(2):
                    lo, hi = ref.extremes(f.held(rows[0][b][c * ps:min(n, (c + 1) * ps), h]))
                    got = bounds[f.table[b, c], h]
                    assert (got[0] <= lo).all() and (got[1] >= hi).all(), f"{count} rows: sequence {b} page {c} head {h}"
                    if first[b] == c * ps:              # written from its first slot on
                        assert np.array_equal(got[0], lo) and np.array_equal(got[1], hi)
    assert f.cache.status() == 0


def test_a_page_with_a_rewritten_first_row_is_still_picked():
    """The page that holds the one key along the query, behind a first row that is written again."""
    f = Filled([16 * 12], 1, 16, True, seed=8, spread=0.1)
    q = np.ones((1, 1, 128))
    k = f.rows[0].copy()
    k[0, 16 * 5 + 9] = 8.0
    f.cache.append(f.seqs, device(k), device(f.rows[1]))
    assert f.cache.select(f.seqs, device(q), 3).tolist() == [[[0, 5, 11]]]
    f.cache.append(f.seqs, device(k[:, 80]), device(f.rows[1][:, 80]), first=_ints([80]))
    assert f.cache.select(f.seqs, device(q), 3).tolist() == [[[0, 5, 11]]]


@pytest.mark.parametrize("order", [[0, 1, 2], [2, 1, 0]])
def test_a_prompt_in_parts_of_any_order(order):
    """Parts that end inside pages: in ascending order, each with its end as length, extremes are exact; in any order they hold."""
    f, ends = Filled([150], 2, 64, True, seed=9), [0, 40, 90, 150]
    rows = [[x[0, :150]] for x in f.rows]
    for x in (f.cache.k, f.cache.v):
        x.view(torch.uint8).fill_(0x7F)
    f.cache.bounds.fill_(float("nan"))
    for i in order:
        if order[0] == 0:
            f.seqs.lengths.fill_(ends[i + 1])
        f.cache.append(f.seqs, *(device(x[:, ends[i]:ends[i + 1]]) for x in f.rows), first=_ints([ends[i]]))
    _check_rows(f, rows)
    _check_bounds(f, rows)
