"""Scores of pages whose extremes are infinite, no numbers, or those of no key at all, against their definition."""
import numpy as np
import pytest
import torch

from oracle import paged as ref
from tests.paged import DEV, Filled, bf16, device

pytestmark = pytest.mark.gpu


def _check(f, q, keeps=(3, 5, 9, 20)):
    bounds, g = f.cache.bounds.double().cpu().numpy(), q.shape[1] // f.hkv
    for keep in keeps:
        got = f.cache.select(f.seqs, device(q), keep).cpu().numpy()
        for b, n in enumerate(f.lengths):
            held = -(-n // f.ps)
            for h in range(f.hkv):
                s = ref.scores(q[b, h * g:(h + 1) * g], *(bounds[f.table[b, :held], h, i] for i in (0, 1)))
                assert got[b, h].tolist() == ref.pick(s, keep, 1, 1).tolist(), f"keep {keep} sequence {b} head {h}: {s}"


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("pages", [30, 400])
def test_pages_without_a_number_in_a_dimension(e4m3, pages):
    """Append leaves +inf and -inf as least and largest where none of a dimension's keys is a number (in 8 bits an infinite one is none either): such a page's score is
    infinite, whatever the query's sign there."""
    def make(rng, shape):
        k, v = (bf16(rng.standard_normal(shape)) for _ in range(2))
        for page, dim in ((4, 3), (9, 100), (17, 0), (23, 127)):
            k[:, 16 * page:16 * page + 16, :, dim] = np.nan if page != 9 else np.inf
        k[:, 16 * 12:16 * 12 + 15, :, 5] = np.nan                  # one number is left
        k[:, 16 * 20:16 * 21] = np.nan                             # none anywhere
        return k, v

    f = Filled([16 * pages, 16 * 27 - 5], 2, 16, e4m3, seed=pages, make=make)
    for sign in (1, -1, 0):
        q = f.queries(8)
        if sign:
            q = sign * np.abs(q) + sign * 0.01
        _check(f, bf16(q))
    q = f.queries(2)
    q[:, :, [3, 100, 0, 127]] = 0.0                                # a zero adds nothing, whatever the extremes
    _check(f, q)


def test_extremes_of_one_side_and_of_no_key():
    """Extremes that a caller keeps: no number on one side, infinite ones, those of nothing."""
    f = Filled([16 * 40], 1, 16, False, seed=2)
    rng = np.random.default_rng(3)
    lo, hi = np.sort([bf16(rng.standard_normal((40, 128))) for _ in range(2)], axis=0)
    lo[3, 7], hi[8, 9], lo[11, 0], hi[14, 5], lo[19] = np.nan, np.nan, -np.inf, np.inf, -np.inf
    lo[25, 2], hi[25, 2], lo[28, 4], hi[28, 4], lo[31, 6], hi[31, 6] = np.inf, -np.inf, np.inf, np.inf, -np.inf, -np.inf
    at = torch.from_numpy(f.table[0]).long().to(DEV)
    f.cache.bounds[at, 0, 0], f.cache.bounds[at, 0, 1] = device(lo), device(hi)
    for heads in (1, 3, 16):
        for sign in (1, -1, 0):
            q = bf16(rng.standard_normal((1, heads, 128)))
            _check(f, sign * np.abs(q) if sign else q)
            q[:, :, ::2] = 0.0
            _check(f, sign * np.abs(q) if sign else q)
