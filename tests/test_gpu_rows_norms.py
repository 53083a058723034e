"""Attention of several rows over long sequences of a cache in pages: how far all outputs of a call are off together, where bounds of the worst case for each would let a lost term of the weights pass."""
import numpy as np
import pytest
import torch

from oracle import paged as ref
from tests.paged import Filled, bf16, device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("n,rows,hq", [(9000, 40, 4), (9000, 8, 4), (30000, 100, 1)])
def test_errors_of_a_whole_call(e4m3, n, rows, hq):
    """Standard normal queries, keys and values: an output is a sum of weights times values of random signs, so its relative error in 2-norm is the weights' (root of the mean square).  A logit of size 1,
    scaled, comes out of some 32 roundings of partial sums of that size, 2^-24 * 0.58 / 2 each on average, 1 * 10^-7 in all; times log2(e), with the maximum taken off, an argument of size 6
    is rounded twice by up to 2^-22, 2 * 10^-7; the exponential is off by up to 2^-23.  Together 3 * 10^-7; 2^-20 allows three times as much.  A third term of the weights that is lost is
    2^-17 of each at most, 2.4 * 10^-6 on average.
    In bf16 an output then rounds the other way than the exact one if a border, 2^-8 of its binade apart, lies between: of 3 * 10^-7 of the norm 8 * 10^-5 of outputs of the norm's size, and several times as
    many with those that are smaller, whose borders are closer; two terms 2.5 * 10^-3.  One in a thousand is allowed."""
    f = Filled([n], 1, 64, e4m3, seed=rows)
    q = bf16(f.rng.standard_normal((1, rows, hq, 128)))
    mask = ref.sees(n - rows, rows)
    want = np.stack([ref.attend_rows(q[0, :, j], f.k[0][0], f.v[0][0], mask, 128 ** -0.5)[0] for j in range(hq)], 1)
    out, _ = f.cache.attend_rows(f.seqs, device(q), f32=True)
    off = np.linalg.norm(out[0].double().cpu().numpy() - want) / np.linalg.norm(want)
    assert off < 2.0 ** -20, f"floats are off by {off:.2e}"
    out, _ = f.cache.attend_rows(f.seqs, device(q))
    got, nearest = out[0].double().cpu().numpy(), torch.from_numpy(want).bfloat16().double().numpy()
    assert np.linalg.norm(got - want) <= np.linalg.norm(nearest - want) * (1 + 2.0 ** -12)
    other = (got != nearest).mean()
    assert other < 1e-3, f"{other:.2e} of the outputs in bf16 round the other way"
