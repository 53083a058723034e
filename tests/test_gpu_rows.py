"""Attention of several rows per sequence over a cache in pages on the GPU, against its definition in 64 bits (oracle/paged.py)."""
import numpy as np
import pytest
import torch

from paper_2601_16986_amd import ckv
from tests.paged import DEV, LAYOUTS, Filled, bf16, check_attention, device
from tests.rows import check_rows, random_tree

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.as_tensor(np.asarray(x, np.int32)).to(DEV)


def queries(f, rows, hq, spread=1.0):
    return bf16(f.rng.standard_normal((len(f.lengths), rows, hq, 128)) * spread)


def attend(f, q, counts, poison=True, **how):
    """attend_rows of the last counts[b] rows, padded to q's; outputs behind a sequence's last row must stay as they were."""
    dt = torch.float32 if how.get("f32") else torch.bfloat16
    out = torch.full(q.shape, -77.0, dtype=dt, device=DEV)
    first = ints([n - c for n, c in zip(f.lengths, counts)])
    got, lse = f.cache.attend_rows(f.seqs, device(q), first=first, out=out, **how)
    assert got is out
    for b, c in enumerate(counts):
        assert (out[b, c:] == -77.0).all(), "rows behind a sequence's last were written"
    return out, lse


# ------------------------------------------------------------------ rows over what comes before them
@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("hq,hkv,rows", [(1, 1, 1), (1, 1, 40), (5, 1, 6), (5, 1, 7), (16, 1, 2), (16, 1, 5), (28, 4, 9), (6, 6, 33), (15, 3, 30), (4, 2, 200)])
def test_rows_see_what_comes_before_them(e4m3, f32, hq, hkv, rows):
    """Blocks of 32, 64 and 128 rows, begun and ended inside a token's heads; rows that are more than a sequence has."""
    lengths = [1, 0, 16, 33, 250, rows]
    counts = [min(n, rows) for n in lengths]
    f = Filled(lengths, hkv, 16, e4m3, LAYOUTS[rows % 3], seed=hq + rows)
    q = queries(f, rows, hq)
    out, lse = attend(f, q, counts, f32=f32, lse=True)
    check_rows(f, q, out, counts, lse=lse)
    assert f.cache.status() == 0


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("ps", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("rows,hq", [(3, 4), (12, 4), (70, 6)])
def test_rows_over_lengths_and_pages(e4m3, ps, rows, hq):
    lengths = [700, rows, 2049, 63 if rows < 63 else 1000]
    f = Filled(lengths, 2, ps, e4m3, LAYOUTS[ps // 32 % 3], seed=ps)
    q, counts = queries(f, rows, hq), [rows] * 4
    out, lse = attend(f, q, counts, lse=True)
    check_rows(f, q, out, counts, lse=lse)
    again, none = attend(f, q, counts)
    assert none is None and torch.equal(out, again), "the same call, the same bits"


@pytest.mark.parametrize("batch,length,hkv,rows,g", [(1, 30000, 1, 4, 4), (1, 20000, 2, 16, 4), (2, 9000, 3, 40, 4), (60, 700, 2, 5, 4), (9, 3000, 1, 24, 16), (1, 5000, 1, 1500, 1), (130, 100, 8, 3, 2)])
def test_rows_in_few_and_many_pieces(batch, length, hkv, rows, g):
    """One unit cut into pieces for the whole chip, numbers of units that make no full round of the chip's parts, more units than run at once."""
    rng = np.random.default_rng(batch)
    lengths = [length] + [int(x) for x in rng.integers(0, length + 1, batch - 1)]
    counts = [min(n, rows) for n in lengths]
    f = Filled(lengths, hkv, 64, True, seed=length)
    q = queries(f, rows, g * hkv)
    out, lse = attend(f, q, counts, lse=True, f32=True)
    check_rows(f, q, out, counts, lse=lse, only=[b for b in range(batch) if b < 2 or b % 41 == 0])


@pytest.mark.parametrize("batch,length,rows,g,window", [(100, 5000, 4, 4, 0), (70, 3099, 40, 4, 0), (129, 2500, 15, 4, 700)])
def test_pieces_by_the_lengths_of_more_sequences_than_a_wavefront_has_lanes(batch, length, rows, g, window):
    rng = np.random.default_rng(batch)
    lengths = [length, 0] + [int(x) for x in np.exp(rng.uniform(0, np.log(length), batch - 2))]
    counts = [min(n, rows) for n in lengths]
    f = Filled(lengths, 1, 64, True, seed=batch)
    q = queries(f, rows, g)
    out, lse = attend(f, q, counts, lse=True, f32=True, window=window)
    check_rows(f, q, out, counts, window=window, lse=lse, only=[b for b in range(batch) if b < 2 or b % 23 == 0])
    packed = torch.cat([device(q)[b, :n] for b, n in enumerate(counts)])
    again, _ = f.cache.attend_rows(f.seqs, packed, rows=rows, starts=ints(np.cumsum([0] + counts)), f32=True, window=window)
    assert torch.equal(again, torch.cat([out[b, :n] for b, n in enumerate(counts)]))


def test_peaked_and_large_logits():
    f = Filled([300, 77], 2, 16, True, seed=9, spread=3.0)
    q = queries(f, 20, 8, spread=3.0)
    for scale in (1.0, 0.001):
        out, lse = attend(f, q, [20, 20], scale=scale, lse=True, f32=True)
        check_rows(f, q, out, [20, 20], lse=lse, scale=scale)


def test_scales_of_keys_and_values_across_their_range():
    def make(rng, shape):
        return (bf16(rng.standard_normal(shape) * np.exp2(rng.integers(-20, 4, shape[:-1])[..., None].astype(float))),
                bf16(rng.standard_normal(shape) * np.exp2(rng.integers(-60, 60, shape[:-1])[..., None].astype(float))))

    f = Filled([130, 64, 7], 1, 32, True, seed=4, make=make)
    q = queries(f, 9, 5)
    out, lse = attend(f, q, [9, 9, 7], lse=True, f32=True)
    check_rows(f, q, out, [9, 9, 7], lse=lse)


def test_a_new_token_each_is_what_attend_gives():
    """[batch][heads][128], and rows out of a wider tensor."""
    f = Filled([1, 129, 500], 2, 16, True, seed=2)
    q = f.queries(8)
    fused = torch.zeros((3, 17, 128), dtype=torch.bfloat16, device=DEV)
    fused[:, 1:17:2] = device(q)
    for x in (device(q), fused[:, 1:17:2]):
        out, lse = f.cache.attend_rows(f.seqs, x, lse=True, f32=True)
        assert out.shape == q.shape and lse.shape == q.shape[:2]
        check_attention(f, q, out, lse)


def test_packed_rows():
    """Sequences' rows one after another, the last ones of each by default, one sequence without."""
    lengths, counts = [100, 40, 9, 300], [37, 0, 9, 130]
    f = Filled(lengths, 2, 32, False, seed=13)
    q = queries(f, 130, 6)
    packed = torch.cat([device(q)[b, :n] for b, n in enumerate(counts)])
    starts = ints(np.cumsum([0] + counts))
    for how in ({}, dict(first=ints([63, 40, 0, 170]))):
        out, lse = f.cache.attend_rows(f.seqs, packed, rows=130, starts=starts, lse=True, f32=True, **how)
        assert out.shape == packed.shape and lse.shape == packed.shape[:2]
        y, z = torch.zeros(q.shape, device=DEV), torch.zeros(q.shape[:3], device=DEV)
        for b, n in enumerate(counts):
            y[b, :n], z[b, :n] = out[sum(counts[:b]):][:n], lse[sum(counts[:b]):][:n]
        check_rows(f, q, y, counts, lse=z)


def test_rows_of_the_middle():
    """`first` before the sequence's last rows: they see what comes before them, though more is there."""
    f = Filled([200, 90], 1, 16, True, seed=14)
    q = queries(f, 20, 3)
    out, lse = f.cache.attend_rows(f.seqs, device(q), first=ints([50, 70]), lse=True, f32=True)
    check_rows(f, q, out, [20, 20], first=[50, 70], lse=lse)


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("window,sinks", [(0, 0), (33, 0), (40, 5)])
def test_a_single_row_anywhere(e4m3, window, sinks):
    """One row per sequence at its first, at its last or in between; a sequence without entries, and rows that are not there; the same rows packed."""
    lengths, first = [200, 300, 1, 0, 90, 64, 40], [50, 299, 0, 0, 0, 64, 39]
    counts = [1, 1, 1, 0, 1, 0, 1]
    f = Filled(lengths, 2, 16, e4m3, seed=window)
    q = queries(f, 1, 8)
    out = torch.full(q.shape, -77.0, device=DEV)
    _, lse = f.cache.attend_rows(f.seqs, device(q), first=ints(first), out=out, window=window, sinks=sinks, f32=True, lse=True)
    check_rows(f, q, out, counts, first=first, window=window, sinks=sinks, lse=lse)
    assert (out[3] == -77.0).all() and (out[5] == -77.0).all() and f.cache.status() == 0
    packed = torch.cat([device(q)[b, :c] for b, c in enumerate(counts)])
    some, z = f.cache.attend_rows(f.seqs, packed, rows=1, first=ints(first), starts=ints(np.cumsum([0] + counts)), window=window, sinks=sinks, f32=True, lse=True)
    again, zs = torch.zeros_like(out), torch.zeros_like(lse)
    at = 0
    for b, c in enumerate(counts):
        again[b, :c], zs[b, :c] = some[at:at + c], z[at:at + c]
        at += c
    check_rows(f, q, again, counts, first=first, window=window, sinks=sinks, lse=zs)


# ------------------------------------------------------------------ windows
@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 4), (5, 1), (16, 17), (63, 0), (64, 4), (65, 64), (100, 200), (129, 5), (500, 4), (10 ** 6, 3), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("rows,hq,ps", [(1, 4, 16), (9, 4, 64), (50, 10, 16)])
def test_windows_and_sinks(e4m3, window, sinks, rows, hq, ps):
    lengths = [900, 1, 64, 130, 400]
    counts = [min(n, rows) for n in lengths]
    f = Filled(lengths, 2, ps, e4m3, seed=rows)
    q = queries(f, rows, hq)
    out, lse = attend(f, q, counts, window=window, sinks=sinks, lse=True, f32=True)
    check_rows(f, q, out, counts, window=window, sinks=sinks, lse=lse)
    assert f.cache.status() == 0


@pytest.mark.parametrize("rows,window,sinks", [(1, 100, 4), (1, 100, 0), (8, 40, 20), (100, 64, 4), (300, 200, 33)])
def test_pages_that_have_left_every_window_are_not_looked_at(rows, window, sinks):
    """Their table entries name no page, or another sequence's; what lies there is no number."""
    f = Filled([1000, 777], 2, 16, False, seed=window)
    q = queries(f, rows, 8)
    before, lse0 = attend(f, q, [rows] * 2, window=window, sinks=sinks, lse=True)
    check_rows(f, q, before, [rows] * 2, window=window, sinks=sinks, lse=lse0)
    for b, n in enumerate(f.lengths):
        oldest = max(n - rows - window + 1, 0)
        gone = [c for c in range(-(-sinks // 16), oldest // 16)]
        assert gone
        for c in gone:
            f.cache.k[f.table[b, c]] = float("nan")
            f.cache.v[f.table[b, c]] = float("nan")
            f.seqs.table[b, c] = -1 if c % 2 else f.cache.n_pages + 5
        for c in (-(-sinks // 16) - 1, oldest // 16):           # entries beside the window's and the sinks' in the pages that stay
            for slot in range(16):
                e = 16 * c + slot
                if c >= 0 and sinks <= e < oldest:
                    f.cache.k[f.table[b, c], :, slot], f.cache.v[f.table[b, c], :, slot] = float("nan"), float("inf")
    out, lse = attend(f, q, [rows] * 2, window=window, sinks=sinks, lse=True)
    assert torch.equal(out, before) and torch.equal(lse, lse0) and f.cache.status() == 0


# ------------------------------------------------------------------ trees
@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("rows,hq,hkv", [(1, 4, 1), (5, 5, 1), (8, 28, 4), (17, 2, 2), (63, 8, 2), (64, 4, 4), (65, 3, 1), (130, 16, 1), (512, 1, 1)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (600, 4)])
def test_drafted_tokens(e4m3, rows, hq, hkv, window, sinks):
    lengths = [rows, rows + 3, rows + 700, rows + 64]
    f = Filled(lengths, hkv, 32, e4m3, seed=rows)
    trees = [random_tree(f.rng, rows) for _ in lengths]
    q = queries(f, rows, hq)
    out, lse = attend(f, q, [rows] * 4, tree=torch.from_numpy(np.stack(trees)).to(DEV), window=window, sinks=sinks, lse=True, f32=True)
    check_rows(f, q, out, [rows] * 4, trees=trees, window=window, sinks=sinks, lse=lse)
    assert f.cache.status() == 0


@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 3), (70, 200)])
def test_masks_that_are_no_trees(window, sinks):
    """Any set of the call's rows, later ones too, rows that do not see themselves, rows that see nothing; a sequence with fewer rows than the call, whose mask names some that are not there."""
    rows, lengths = 40, [40, 41, 500, 20, 0]
    counts = [40, 40, 40, 20, 0]
    f = Filled(lengths, 2, 16, True, seed=window)
    trees = f.rng.random((5, rows, rows)) < 0.3
    trees[0, 5] = trees[0, 39] = trees[2, 7] = False
    q = queries(f, rows, 6)
    out, lse = attend(f, q, counts, tree=torch.from_numpy(trees).to(DEV), window=window, sinks=sinks, lse=True, f32=True)
    check_rows(f, q, out, counts, trees=trees, window=window, sinks=sinks, lse=lse)
    assert (out[0, 5] == 0).all() and (lse[0, 5] == -float("inf")).all()


def test_one_tree_for_all_and_lines_with_gaps():
    rows, lengths = 21, [21, 100, 300]
    f = Filled(lengths, 1, 16, True, seed=3)
    tree = random_tree(f.rng, rows)
    wide = torch.ones((30, 50), dtype=torch.uint8, device=DEV) * 3
    wide[2:23, 7:28] = torch.from_numpy(tree).to(DEV) * 2
    q = queries(f, rows, 4)
    for t in (torch.from_numpy(tree).to(DEV), wide[2:23, 7:28]):
        out, lse = attend(f, q, [rows] * 3, tree=t, lse=True)
        check_rows(f, q, out, [rows] * 3, trees=[tree] * 3, lse=lse)
    packed = torch.cat([device(q)[b] for b in range(3)])
    again, _ = f.cache.attend_rows(f.seqs, packed, rows=rows, starts=ints([0, 21, 42, 63]), tree=torch.from_numpy(tree).to(DEV))
    assert torch.equal(again.view(out.shape), out)


# ------------------------------------------------------------------ what must not matter
@pytest.mark.parametrize("rows,hq", [(6, 4), (14, 4), (40, 4)])
@pytest.mark.parametrize("nonsense", [float("nan"), float("inf"), -float("inf"), 3.0e38])
def test_what_lies_behind_a_sequence_does_not_matter(rows, hq, nonsense):
    lengths = [40, 49, 64, 100]
    for e4m3 in (True, False):
        f = Filled(lengths, 1, 16, e4m3, seed=3)
        if not e4m3:
            there = torch.zeros(f.cache.k.shape[:3], dtype=torch.bool)
            for b, n in enumerate(lengths):
                for i in range(n):
                    there[f.table[b, i // 16], :, i % 16] = True
            for x in (f.cache.k, f.cache.v):
                x[~there.to(DEV)] = nonsense
        q = queries(f, rows, hq)
        out, lse = attend(f, q, [rows] * 4, lse=True, f32=True)
        check_rows(f, q, out, [rows] * 4, lse=lse)


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("rows,hq", [(6, 4), (14, 4), (40, 4)])
@pytest.mark.parametrize("kind", ["later", "window", "tree"])
def test_rows_are_not_told_of_entries_that_they_do_not_see(e4m3, rows, hq, kind):
    """Keys that are no numbers and values that are infinite in entries that some rows see and others do not: the others' outputs are bit by bit those of clean entries;
    those that see one get NaN in that value's dimensions (all of them if it is the key)."""
    n, at = 200, 200 - rows // 2
    how, trees = {}, None
    if kind == "window":
        how, at = dict(window=30, sinks=2), 200 - rows - 30 + 1 + rows // 2
    f = Filled([n], 1, 16, e4m3, seed=rows)
    if kind == "tree":
        trees = [random_tree(f.rng, rows)]
        how = dict(tree=torch.from_numpy(trees[0]).to(DEV))
    from oracle import paged as ref
    mask = ref.sees(n - rows, rows, how.get("window", 0), how.get("sinks", 0), None if trees is None else trees[0])
    q = queries(f, rows, hq)
    clean, lse0 = attend(f, q, [rows], lse=True, f32=True, **how)
    page, slot = f.table[0, at // 16], at % 16
    k, v = (x.view(torch.uint8 if e4m3 else torch.int16) for x in (f.cache.k, f.cache.v))
    was = v[page, 0, slot, 7].clone()
    v[page, 0, slot, 7] = 0x7F if e4m3 else 0x7F80
    out, lse = attend(f, q, [rows], lse=True, f32=True, **how)
    told = torch.from_numpy(mask[:, at]).to(DEV)
    assert told.any() and not told.all()
    assert torch.equal(out[0, ~told], clean[0, ~told]) and torch.equal(lse, lse0)
    assert torch.isnan(out[0, told][..., 7]).all() and torch.equal(out[0, told][..., 8:], clean[0, told][..., 8:]) and torch.equal(out[0, told][..., :7], clean[0, told][..., :7])
    v[page, 0, slot, 7] = was
    k[page, 0, slot, 3] = 0x7F if e4m3 else 0x7FC0
    out, lse = attend(f, q, [rows], lse=True, f32=True, **how)
    assert torch.equal(out[0, ~told], clean[0, ~told]) and torch.equal(lse[0, ~told], lse0[0, ~told])
    assert torch.isnan(out[0, told]).all() and torch.isnan(lse[0, told]).all()


def test_keys_of_minus_infinity_weigh_nothing():
    f = Filled([40, 3], 1, 16, False, seed=6)
    rows = [torch.from_numpy(x).clone() for x in f.rows]
    rows[0][0, 5], rows[0][1] = -float("inf"), -float("inf")
    f.cache.append(f.seqs, *(x.to(DEV).bfloat16() for x in rows))
    q = np.abs(queries(f, 3, 2)) + 0.01
    f.k[0][0][5], f.k[1][0][:] = -np.inf, -np.inf
    out, lse = attend(f, q, [3, 3], lse=True)
    check_rows(f, bf16(q), out, [3, 3], lse=lse)
    assert (out[1] == 0).all() and (lse[1] == -float("inf")).all()


# ------------------------------------------------------------------ what the host cannot check
def test_wrong_tables_and_lengths_are_reported_and_left_out():
    f = Filled([100, 50, 64], 1, 16, True, seed=7)
    q = queries(f, 12, 4)
    good = f.seqs.table.clone()
    f.seqs.table[0, 2], f.seqs.table[2, 1] = 10 ** 9, -1
    out, lse = attend(f, q, [12] * 3, lse=True)
    assert f.cache.status() == ckv.BAD_PAGE and f.cache.status() == 0
    g = Filled([100, 50, 64], 1, 16, True, seed=7)
    for b, (lo, hi) in ((0, (32, 48)), (2, (16, 32))):         # as if those keys were of no weight
        g.k[b][0] = g.k[b][0].copy()
        g.lengths = [100, 50, 64]
    from oracle import paged as ref
    for b, (lo, hi) in ((0, (32, 48)), (2, (16, 32))):
        mask = ref.sees(f.lengths[b] - 12, 12)
        mask[:, lo:hi] = False
        for j in range(4):
            o, s, mass, reach = ref.attend_rows(q[b, :, j], f.k[b][0], f.v[b][0], mask, 128 ** -0.5)
            assert np.abs(out[b, :, j].double().cpu().numpy() - o).max() <= 2.0 ** -7 * np.abs(o).max()
    check_rows(f, q, out, [12] * 3, lse=lse, only=[1])
    # lengths beyond what the call was told: rows from there on are left out; below nothing
    f.seqs.table.copy_(good)
    f.seqs.lengths.copy_(ints([10 ** 9, -5, 64]))
    s = f.cache.sequences(f.seqs.table, f.seqs.lengths, 96)
    out = torch.full((3, 12, 4, 128), -77.0, dtype=torch.bfloat16, device=DEV)
    f.cache.attend_rows(s, device(q), first=ints([90, 0, 52]), out=out)
    assert f.cache.status() == ckv.BAD_LENGTH
    f.lengths = [96, 0, 64]
    check_rows(f, q, out, [6, 0, 12])
    assert (out[0, 6:] == -77.0).all() and (out[1] == -77.0).all()
    # rows that do not fit their sequence, packed rows beyond the buffer
    out.fill_(-77.0)
    f.seqs.lengths.copy_(ints([100, 50, 64]))
    f.cache.attend_rows(f.seqs, device(q), first=ints([101, -1, 65]), out=out)
    assert f.cache.status() == ckv.BAD_LENGTH and (out == -77.0).all()
    flat = torch.full((5, 4, 128), -77.0, dtype=torch.bfloat16, device=DEV)
    f.cache.attend_rows(f.seqs, device(q)[0, :5], rows=5, starts=ints([0, 6, 6, 4]), out=flat)
    assert f.cache.status() == ckv.BAD_LENGTH and (flat == -77.0).all()


def test_calls_with_nothing_to_do():
    f = Filled([20, 0], 2, 16, True)
    q = torch.zeros((0, 4, 128), dtype=torch.bfloat16, device=DEV)
    out, lse = f.cache.attend_rows(f.seqs, q, rows=4, starts=ints([0, 0, 0]), lse=True)
    assert out.shape == q.shape and lse.shape == (0, 4)
    s = f.cache.sequences(f.seqs.table, torch.zeros_like(f.seqs.lengths), 0)
    out = torch.full((2, 3, 4, 128), -77.0, dtype=torch.bfloat16, device=DEV)
    f.cache.attend_rows(s, device(np.zeros((2, 3, 4, 128))), out=out)
    assert (out == -77.0).all() and f.cache.status() == 0


def test_refusals_of_the_binding():
    f = Filled([20], 2, 16, True)
    q = device(queries(f, 5, 4))
    tree = torch.ones((1, 5, 5), dtype=torch.bool, device=DEV)
    c, s = f.cache, f.seqs
    for bad in (dict(q=q.float()), dict(q=q[..., :64]), dict(q=q[:, :, :3]), dict(q=q.cpu()), dict(q=q.repeat(2, 1, 1, 1)), dict(window=-1), dict(sinks=-1), dict(sinks=4), dict(window=2 ** 31),
                dict(tree=tree.float()), dict(tree=tree[:, :4]), dict(tree=tree.cpu()), dict(tree=tree.transpose(1, 2).repeat(1, 1, 2)[..., ::2]), dict(tree=tree, window=4), dict(rows=4),
                dict(scale=0.0), dict(scale=float("nan")), dict(scale=-1.0), dict(out=torch.empty_like(q, dtype=torch.float32)), dict(out=q[:, :4].contiguous()), dict(first=torch.zeros(1, device=DEV)),
                dict(starts=ints([0, 5])), dict(q=q[0], starts=ints([0, 5])), dict(q=q[0], starts=ints([0, 5, 6]), rows=5)):
        with pytest.raises(ckv.CkvError):
            c.attend_rows(s, **{**dict(q=q), **bad})
    big = Filled([600], 1, 64, True)
    with pytest.raises(ckv.CkvError):
        big.cache.attend_rows(big.seqs, device(queries(big, 513, 1)), tree=torch.ones((513, 513), dtype=torch.bool, device=DEV))


# ------------------------------------------------------------------ offsets, streams, graphs
def test_pools_beyond_four_gigabytes():
    hkv, ps, n = 8, 256, 18432 // 2
    big = ckv.PagedCache.empty(n, ps, hkv, dtype=ckv.BF16)
    f = Filled([600], hkv, ps, False, seed=2)
    s = big.sequences(ints([[n - 1, 3, n - 2]]), f.seqs.lengths)
    big.append(s, *(device(x) for x in f.rows))
    q = queries(f, 20, 16)
    for how in ({}, dict(window=100, sinks=4)):
        out, lse = big.attend_rows(s, device(q), lse=True, **how)
        check_rows(f, q, out, [20], lse=lse, **how)


def test_calls_on_two_streams_at_once():
    f = Filled([9000, 4000], 2, 64, True, seed=21)
    qs = [device(queries(f, r, 8)) for r in (1, 7, 16, 60)]
    want = [f.cache.attend_rows(f.seqs, q)[0] for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None] * 4
    for _ in range(5):
        for i, q in enumerate(qs):
            with torch.cuda.stream(streams[i % 2]):
                got[i] = f.cache.attend_rows(f.seqs, q)[0]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("e4m3", [True, False])
def test_a_drafting_step_captured_and_replayed(e4m3):
    """Drafts enter turned, are attended by a tree of this step, a window of them too: one graph, replayed while lengths, tree and inputs change, beside another graph and eager calls between the replays."""
    rows, hq, hkv = 9, 8, 2
    f, g = (Filled([900, 63, 0], hkv, 16, e4m3, seed=31, columns=70, spare=40) for _ in range(2))
    for x in (f, g):
        free = [p for p in range(x.cache.n_pages) if p not in set(x.table[x.table >= 0].tolist())]
        for b, held in enumerate((57, 4, 0)):
            for c in range(6):
                x.seqs.table[b, held + c] = free.pop()
    rng = np.random.default_rng(0)
    k, v = (torch.zeros((3, rows, hkv, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    q = torch.zeros((3, rows, hq, 128), dtype=torch.bfloat16, device=DEV)
    tree, positions = torch.zeros((3, rows, rows), dtype=torch.bool, device=DEV), torch.zeros((3, rows), dtype=torch.int32, device=DEV)
    r = ckv.Rotation(torch.from_numpy(10000.0 ** (-np.arange(64) / 64)).to(DEV))

    def step(x):
        turned = x.cache.append_rotated(x.seqs, q, k, v, r, positions=positions)
        a, lse = x.cache.attend_rows(x.seqs, turned, tree=tree, lse=True)
        w, _ = x.cache.attend_rows(x.seqs, turned, tree=tree, window=100, sinks=4, f32=True)
        one, _ = x.cache.attend_rows(x.seqs, turned[:, -1], window=50)
        return turned, a, lse, w, one

    def change():
        for x in (f, g):
            x.seqs.lengths.add_(rows)
        for to in (k, v, q):
            to.copy_(torch.from_numpy(rng.standard_normal(tuple(to.shape))))
        t = np.stack([random_tree(rng, rows) for _ in range(3)])
        tree.copy_(torch.from_numpy(t))
        positions.copy_((f.seqs.lengths[:, None] - rows) + torch.from_numpy(t.sum(2) - 1).to(DEV))

    change()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(f)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = step(f)
        graphs.append((graph, got))
    for n in range(7):
        if n:
            change()
        graph, got = graphs[n % 2]
        graph.replay()
        want = step(g)
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(got, want)):
            assert torch.equal(a, b), f"replay {n} output {i}"
    assert f.cache.status() == 0 and g.cache.status() == 0
