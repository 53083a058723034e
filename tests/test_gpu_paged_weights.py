"""Attention over a cache in pages: the weights' own precision, where values nearly cancel."""
import numpy as np
import pytest
import torch

from tests.paged import DEV, bf16, device, pools

pytestmark = pytest.mark.gpu


def _pieces(x, bits, n):
    """x to nearest as a sum of n numbers of so many bits each."""
    r = []
    for _ in range(n):
        e = np.where(x == 0, 0, np.frexp(x)[1] - bits)
        r.append(np.ldexp(np.rint(np.ldexp(x, -e)), e))
        x = x - r[-1]
    return r


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("g", [1, 12])
@pytest.mark.parametrize("f32", [False, True])
def test_weights_have_the_bits_of_a_float(e4m3, g, f32):
    """Entries of logit 0, values adding up to w to 20 bits or more, and one of logit -x and value -1, w = exp(-x) in (1/2, 1): the output (sum - w) / (entries + w) is what w's own
    rounding leaves.  The product -x log2(e) is off by 2 half steps of a float below 1, 2 * 2^-25, and w by 0.7 of that; the exponential and its terms are off by 2^-24 each; products with
    the values are exact, and sums of numbers on one grid of 2^-24 below 4 by at most 2^-24 in all.  That is below 2^-22, and is divided by entries + w; an output in bf16 is
    rounded by 2^-8 of itself.  (Weights of 16 bits would be off by up to 2^-18.)"""
    n, hkv, ps, ones = 64, 2, 16, 6 if e4m3 else 3
    rng = np.random.default_rng(1)
    x = bf16(rng.uniform(0.25, 0.6, (n, hkv)))                    # q's first dimension; the last key's is -1
    w = np.exp(-x)
    parts = _pieces(w, 4 if e4m3 else 8, ones)
    k, v = np.zeros((n, ones + 1, hkv, 128)), np.zeros((n, ones + 1, hkv, 128))
    k[:, ones, :, 0], v[:, ones] = -1.0, -1.0
    for i, p in enumerate(parts):
        v[:, i] = p[:, :, None]
    q = np.zeros((n, hkv, g, 128))
    q[..., 0] = x[:, :, None]
    cache = pools(n, hkv, ps, e4m3)
    seqs = cache.sequences(torch.arange(n, dtype=torch.int32, device=DEV)[:, None].contiguous(), torch.full((n,), ones + 1, dtype=torch.int32, device=DEV))
    cache.append(seqs, device(k), device(v))
    back = cache.read(seqs, ones + 1)[1].double().cpu().numpy()
    assert np.array_equal(back, v), "the values are what the cache holds"
    out, _ = cache.attend(seqs, device(q.reshape(n, hkv * g, 128)), scale=1.0, f32=f32)
    want = ((sum(parts) - w) / (ones + w))[:, :, None, None]
    got = out.double().cpu().numpy().reshape(n, hkv, g, 128)
    tol = 2.0 ** -22 / (ones + w)[:, :, None, None] + (2.0 ** -22 if f32 else 2.0 ** -8) * np.abs(want)
    assert (np.abs(got - want) <= tol).all(), f"off by {np.abs(got - want).max() * 2 ** 24:.1f} * 2^-24"
