"""Rows of the tests of ckv_paged_attend_rows: who sees what, and how far outputs may be off."""
from __future__ import annotations

import numpy as np

from oracle import paged as ref


def check_rows(f, q, out, counts, *, first=None, window=0, sinks=0, trees=None, lse=None, scale=128 ** -0.5, what="", only=None):
    """out [batch][rows][hq][128] against the definition for the last counts[b] rows of each sequence of f (tests.paged.Filled), queries q [batch][rows][hq][128].

    As in tests.paged.check_attention: an entry's logit is a float sum of 128 exact products, off by at most 130 half steps (2^-24) of the sum of their magnitudes, and the exponential's argument
    by a few more of its own size, so that a weight is off by twice 140 * 2^-24 * reach relative to the others.  Weights' terms leave 2^-16 (two, bf16 outputs) or 2^-24 (three).  Into an accumulator go at
    most three products per 16 entries and a factor per 64 (n / 4 in all), into the sum of weights 64 of a tile and one per tile, and joining adds up to a hundred: at most 2^-24 each of the sum of
    |weight * value|.  A bf16 output is rounded by 2^-8 of itself."""
    y = out.double().cpu().numpy()
    z = lse.double().cpu().numpy() if lse is not None else None
    f32 = out.dtype.itemsize == 4
    hq = q.shape[2]
    g = hq // f.hkv
    for b in range(len(f.lengths)) if only is None else only:
        n, r = f.lengths[b], counts[b]
        if r == 0:
            continue
        start = n - r if first is None else first[b]
        mask = ref.sees(start, r, window, sinks, None if trees is None else trees[b])
        for h in range(f.hkv):
            k, v = f.k[b][h][:start + r], f.v[b][h][:start + r]
            for j in range(h * g, (h + 1) * g):
                o, s, mass, reach = ref.attend_rows(q[b, :r, j], k, v, mask, scale)
                bound = ((2 * 140 * reach + n / 4 + 256) * 2.0 ** -24 + 2.0 ** (-24 if f32 else -16))[:, None]
                tol = bound * mass + (0 if f32 else 2.0 ** -8 * (np.abs(o) + bound * mass)) + 1e-30
                off = np.abs(y[b, :r, j] - o)
                assert np.all(off <= tol), f"{what} sequence {b} (rows {r} of {n}) head {j}: off by {np.nanmax(off / tol):.2f} of the bound at row {np.argwhere(~(off <= tol))[0]}"
                if z is not None:
                    none = np.isinf(s)
                    assert np.array_equal(z[b, :r, j][none], s[none]), f"{what} sequence {b} head {j}: lse where nothing is seen"
                    far = np.abs(z[b, :r, j][~none] - s[~none]) > (bound[:, 0] + 2.0 ** -23 * np.abs(s) + 2.0 ** -22)[~none]
                    assert not far.any(), f"{what} sequence {b} head {j}: lse"


def random_tree(rng, rows):
    """Ancestors of drafted tokens with random parents."""
    m = np.zeros((rows, rows), bool)
    for i in range(rows):
        up = rng.integers(-1, i) if i else -1
        if up >= 0:
            m[i] = m[up]
        m[i, i] = True
    return m
