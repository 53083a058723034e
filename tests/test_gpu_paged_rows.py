"""Where the rows of a call go in a cache in pages: packed rows without their positions."""
import numpy as np
import pytest
import torch

from tests.paged import DEV, Filled, bf16, device

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _check_rows(f, rows):
    """f's sequences hold `rows[side][b]`, [length][heads][128], in 8 bits as those become."""
    for b, n in enumerate(f.lengths):
        k, v = f.cache.read(f.cache.sequences(f.seqs.table[b:b + 1], f.seqs.lengths[b:b + 1]), max(n, 1), first=_ints([0]))
        for side, got in enumerate((k, v)):
            for h in range(f.hkv):
                assert np.array_equal(got[0, :n, h].double().cpu().numpy(), f.held(rows[side][b][:n, h])), f"sequence {b} head {h}"


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
