"""A row of each sequence over a cache in pages: padded, where the attention of one token takes it, it comes out as it does packed, whatever values are not finite or as large as they come."""
import numpy as np
import pytest
import torch

from oracle import paged as ref
from tests.paged import DEV, Filled, bf16, device
from tests.rows import check_rows
from tests.test_gpu_rows_range import LARGE, filled, ints

pytestmark = pytest.mark.gpu


def attend(f, q, packed, **how):
    """One row of each sequence, its last: q [batch][1][hq][128]."""
    x = device(q)
    if packed:
        out, lse = f.cache.attend_rows(f.seqs, x[:, 0], rows=1, starts=ints(np.arange(len(f.lengths) + 1)), lse=True, f32=True, **how)
        return out[:, None], lse[:, None]
    return f.cache.attend_rows(f.seqs, x, lse=True, f32=True, **how)


def spoil(f, b, entries, codes):
    """Values of entries of a sequence as they lie in the cache: {dimension: (code, bf16's bits)}."""
    for e in entries:
        page, slot = f.table[b, e // f.ps], e % f.ps
        for d, (code, half) in codes.items():
            if f.e4m3:
                f.cache.v.view(torch.uint8)[page, :, slot, d] = code
            else:
                f.cache.v.view(torch.int16)[page, :, slot, d] = half


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("g", [2, 12])
@pytest.mark.parametrize("n,window", [(40, 0), (3000, 0), (3000, 1200)])
def test_values_that_are_not_finite_reach_the_heads_that_give_them_weight(packed, e4m3, g, n, window):
    """Entries whose logits are -inf for every other head (a product beyond the floats) and ordinary for the rest: there NaN in their values' dimensions, elsewhere nothing of them."""
    spoilt = [n - 3, n - 20] + ([n - 900] if n > 900 else [])

    def make(rng, shape):
        k, v = bf16(rng.standard_normal(shape)), bf16(rng.standard_normal(shape))
        k[..., 0] = 0.0
        k[0, spoilt] = 0.0
        k[0, spoilt, :, 0] = -1.5 * 2.0 ** 126
        return k, v

    f = Filled([n, 17], 1, 16, e4m3, seed=n + g, make=make)
    spoil(f, 0, spoilt, {7: (0x7F, 0x7F80), 90: (0xFF, 0x7FC0)})
    q = bf16(f.rng.standard_normal((2, 1, g, 128)))
    q[..., 0] = np.where(np.arange(g) % 2, 0.0, 64.0)
    out, lse = attend(f, q, packed, scale=0.1, **(dict(window=window, sinks=2) if window else {}))
    seen = ref.sees(n - 1, 1, window, 2 if window else 0)[0]
    y, z = out.double().cpu().numpy()[0, 0], lse.double().cpu().numpy()[0, 0]
    keep = seen.copy()
    keep[spoilt] = False
    for j in range(g):
        k, v = f.k[0][0], f.v[0][0].copy()
        v[spoilt] = 0.0 if j % 2 == 0 else v[spoilt]
        mine = keep if j % 2 == 0 else seen
        o, s, mass, reach = ref.attend(q[0, 0, j], k[mine], v[mine], 0.1)
        bound = (2 * 140 * reach + n / 4 + 256 + 1) * 2.0 ** -24
        clean = np.ones(128, bool)
        if j % 2:
            clean[[7, 90]] = False
            assert np.isnan(y[j, [7, 90]]).all(), f"head {j} gives weight"
        assert (np.abs(y[j] - o) <= bound * mass + 1e-30)[clean].all(), f"head {j}"
        assert abs(z[j] - s) <= bound + 2.0 ** -23 * abs(s) + 2.0 ** -22
    check_rows(f, q, out, [1, 1], window=window, sinks=2 if window else 0, lse=lse, scale=0.1, only=[1])


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("hq,lengths,window", [(8, [3000, 75, 700], 0), (32, [3000, 75, 700], 0), (8, [9000, 64, 1], 2000)])
@pytest.mark.parametrize("which", ["all", "first half", "now and then"])
def test_large_values_of_a_single_row(packed, e4m3, hq, lengths, window, which):
    large = {"all": lambda e: e >= 0, "first half": lambda e: e < lengths[0] - max(window, 3000) // 2, "now and then": lambda e: e % 29 == 3}[which]
    f = filled(lengths, 2, 64, e4m3, hq, large)
    q = bf16(f.rng.standard_normal((3, 1, hq, 128)))
    how = dict(window=window, sinks=4) if window else {}
    out, lse = attend(f, q, packed, **how)
    check_rows(f, q, out, [1] * 3, lse=lse, **how)


@pytest.mark.parametrize("packed", [False, True])
def test_eight_bits_that_are_infinite_as_bf16(packed):
    """A magnitude from 1.9375 * 2^127 on is read back as infinite, and counts as such: NaN where it has weight, nothing where it has none."""
    def make(rng, shape):
        k, v = bf16(rng.standard_normal(shape)), bf16(rng.standard_normal(shape))
        k[0, 30], k[1, 30] = 0.0, 0.0
        k[1, 30, :, 0] = -1.5 * 2.0 ** 126
        v[:, 30, :, 5] = bf16(1.984375 * 2.0 ** 127)
        return k, v

    f = Filled([50, 50], 1, 16, True, seed=3, make=make)
    assert np.isinf(f.v[0][0][30, 5])
    q = np.abs(bf16(f.rng.standard_normal((2, 1, 4, 128)))) + 0.0
    q[..., 0] = 64.0
    out, _ = attend(f, q, packed)
    assert torch.isnan(out[0, 0, :, 5]).all() and torch.isfinite(out[0, 0, :, 6:]).all() and torch.isfinite(out[0, 0, :, :5]).all() and torch.isfinite(out[1]).all()
    assert LARGE < 1.9375 * 2.0 ** 127
