"""Attention of several rows over a cache in pages: the weights' own precision, where values nearly cancel."""
import numpy as np
import pytest
import torch

from tests.paged import DEV, bf16, device, pools

N, HKV, PS = 64, 2, 16


def pieces(x, bits, n):
    """x to nearest as a sum of n numbers of so many bits each."""
    r = []
    for _ in range(n):
        e = np.where(x == 0, 0, np.frexp(x)[1] - bits)
        r.append(np.ldexp(np.rint(np.ldexp(x, -e)), e))
        x = x - r[-1]
    return r


def entries(e4m3, gap):
    """(x, keys, values, what comes out, its tolerance but for bf16's rounding): `ones` entries of logit 0, values adding up to w to 20 bits or more, and one of logit -x and value -1,
    w = exp(-x) in (1/2, 1), each `gap` entries behind the one before; the entries between have logits of -200 and below, weights of nothing.

    The output (sum - w) / (ones + w) is what w's own rounding leaves.  The product -x log2(e) is off by 2 half steps of a float below 1, 2 * 2^-25, and w by 0.7 of that; the exponential
    and its terms are off by 2^-24 each; products with the values are exact, and sums of numbers on one grid of 2^-24 below 4 by at most 2^-24 in all.  That is below 2^-22, and is divided by
    ones + w."""
    ones = 6 if e4m3 else 3
    rng = np.random.default_rng(1)
    x = bf16(rng.uniform(0.25, 0.6, (N, HKV)))                    # q's first dimension; the last key's is -1
    w = np.exp(-x)
    parts = pieces(w, 4 if e4m3 else 8, ones)
    k, v = np.zeros((N, ones * gap + 1, HKV, 128)), np.zeros((N, ones * gap + 1, HKV, 128))
    k[..., 0] = -1024.0
    v[:] = 3.0
    for i, p in enumerate(parts):
        k[:, i * gap] = 0.0
        v[:, i * gap] = p[:, :, None]
    k[:, ones * gap] = 0.0
    k[:, ones * gap, :, 0], v[:, ones * gap] = -1.0, -1.0
    return x, k, v, w, (sum(parts) - w) / (ones + w), 2.0 ** -22 / (ones + w)


@pytest.mark.parametrize("e4m3", [True, False])
def test_two_terms_would_not_do(e4m3):
    """Of weights rounded to two bf16 terms most outputs are off by more than the tolerance of this file, bf16's rounding included."""
    _, _, _, w, want, tol = entries(e4m3, 1)
    two = sum(pieces(w, 8, 2))
    off = np.abs(two - w) / ((6 if e4m3 else 3) + w)
    assert (off > tol + 2.0 ** -8 * np.abs(want)).mean() > 0.5


@pytest.mark.gpu
@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("rows,g", [(1, 4), (7, 1), (20, 4)])
@pytest.mark.parametrize("gap", [1, 37, 211])
@pytest.mark.parametrize("packed", [False, True])
def test_weights_of_several_rows_have_the_bits_of_a_float(e4m3, f32, rows, g, gap, packed):
    """Rows that see what comes before them and nothing of each other, in blocks of 64 and 128 rows, in one piece and several; a row each too, padded and packed."""
    x, k, v, _, want, tol = entries(e4m3, gap)
    n = k.shape[1]
    k, v = (np.concatenate([a, np.zeros((N, rows, HKV, 128))], 1) for a in (k, v))
    held = -(-(n + rows) // PS)
    cache = pools(N * held, HKV, PS, e4m3)
    table = torch.arange(N * held, dtype=torch.int32, device=DEV).view(N, held)
    seqs = cache.sequences(table, torch.full((N,), n + rows, dtype=torch.int32, device=DEV))
    cache.append(seqs, device(k), device(v))
    assert np.array_equal(cache.read(seqs, n + rows)[1].double().cpu().numpy(), v), "the values are what the cache holds"
    q = np.zeros((N, rows, HKV, g, 128))
    q[..., 0] = x[:, None, :, None]
    how = dict(tree=torch.zeros((rows, rows), dtype=torch.bool, device=DEV)) if rows > 1 else dict(first=torch.full((N,), n - 1, dtype=torch.int32, device=DEV))
    flat = device(q.reshape(N, rows, HKV * g, 128))
    if packed:
        flat = flat.view(N * rows, HKV * g, 128)
        how.update(rows=rows, starts=torch.arange(0, N * rows + 1, rows, dtype=torch.int32, device=DEV))
    out, _ = cache.attend_rows(seqs, flat, scale=1.0, f32=f32, **how)
    want, tol = want[:, None, :, None, None], tol[:, None, :, None, None]
    got = out.double().cpu().numpy().reshape(N, rows, HKV, g, 128)
    tol = tol + (2.0 ** -22 if f32 else 2.0 ** -8) * np.abs(want)
    assert (np.abs(got - want) <= tol).all(), f"off by {np.abs(got - want).max() * 2 ** 24:.1f} * 2^-24"
    assert cache.status() == 0
