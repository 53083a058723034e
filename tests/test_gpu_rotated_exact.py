"""Rows that enter the cache in pages with their positions' rotation: keys in 8 bits rounded once from 64 bits, and bounds of pages that held rows before."""
import numpy as np
import pytest
import torch

from oracle import paged as ref
from paper_2601_16986_amd import ckv
from tests.paged import DEV, bf16, device, pools

PAIRS = 56                                   # the last 16 dimensions stay as they are


def ints(x):
    return torch.as_tensor(np.asarray(x, np.int32)).to(DEV)


def halfway(interleaved):
    """(keys [rows][128], frequencies): rows of power 0 by a 448 that does not turn, every pair a number half way between two codes and a small one, which at positions 1, 2, ... turns the
    first by less than a float's last bit, up or down.  (Frequencies times the small number: 2^-10 * 3e-8 * 120 at most, 3.5e-9 * 2^-8 of the smallest first numbers; what the cosine takes off is
    a hundredth of the turn at most.)"""
    rng = np.random.default_rng(0)
    rows = 120
    f = np.exp(rng.uniform(np.log(1e-9), np.log(3e-8), PAIRS))
    mid = (ref.E4M3[56:118] + ref.E4M3[57:119]) / 2              # from 1 on, below 448: bf16 numbers
    x = rng.choice(mid, (rows, PAIRS)) * rng.choice([-1.0, 1.0], (rows, PAIRS))
    z = 2.0 ** -10 * rng.choice([-1.0, 1.0], (rows, PAIRS))
    k = np.zeros((rows, 128))
    first, second = (slice(0, 2 * PAIRS, 2), slice(1, 2 * PAIRS, 2)) if interleaved else (slice(0, PAIRS), slice(PAIRS, 2 * PAIRS))
    swap = rng.random((rows, PAIRS)) < 0.5                        # the number half way is the pair's first or its second
    k[:, first], k[:, second] = np.where(swap, z, x), np.where(swap, x, z)
    k[:, 120] = 448.0
    assert np.array_equal(bf16(k), k)
    return k, f


@pytest.mark.parametrize("interleaved", [False, True])
def test_rounding_twice_would_be_seen(interleaved):
    """Turned in 32 bits first, a quarter of the numbers and more get another code than turned in 64 bits."""
    k, f = halfway(interleaved)
    y = ref.rotate(k[:, None], np.arange(1, len(k) + 1), f, interleaved)[:, 0]
    once, twice = ref.quantise(y)[0], ref.quantise(y.astype(np.float32).astype(np.float64))[0]
    assert (ref.quantise(y)[1] == 0).all() and (once != twice).sum() > 0.25 * len(k) * PAIRS


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("hq", [0, 4])
def test_keys_in_eight_bits_are_rounded_once(interleaved, hq):
    k, f = halfway(interleaved)
    n = len(k)
    c = pools(10, 1, 16, True)
    s = c.sequences(ints([np.arange(10)]), ints([n + 1]))
    r = ckv.Rotation(torch.from_numpy(f).to(DEV), interleaved=interleaved)
    q = device(np.ones((1, n, hq, 128))) if hq else None
    c.append_rotated(s, q, device(k[None, :, None]), device(k[None, :, None]), r)
    codes, e = ref.quantise(ref.rotate(k[:, None], np.arange(1, n + 1), f, interleaved)[:, 0])
    at = np.arange(1, n + 1)
    got, scales = c.k.view(torch.uint8).cpu().numpy()[at // 16, 0, at % 16], c.scales.cpu().numpy()[at // 16, 0, at % 16, 0].astype(int) - 127
    assert np.array_equal(scales, e)
    wrong = got != codes
    assert not wrong.any(), f"{wrong.sum()} codes of {wrong.size}"


@pytest.mark.gpu
def test_a_largest_key_that_turns_past_448_gets_another_power():
    """By less than a float's last bit, in both directions."""
    n, f = 8, np.full(PAIRS, 2e-9)
    k = np.zeros((n, 128))
    k[:, 3], k[:, 3 + PAIRS] = 448.0, np.where(np.arange(n) % 2, 1.0, -1.0) * 2.0 ** -3
    c = pools(2, 1, 16, True)
    s = c.sequences(ints([[0, 1]]), ints([n]))
    c.append_rotated(s, None, device(k[None, :, None]), device(k[None, :, None]), ckv.Rotation(torch.from_numpy(f).to(DEV)))
    y = ref.rotate(k[:, None], np.arange(n), f)[:, 0]
    codes, e = ref.quantise(y)
    assert sorted(set(e.tolist())) == [0, 1] and (y.astype(np.float32)[:, 3] == 448.0).all()
    assert np.array_equal(c.scales.cpu().numpy()[0, 0, :n, 0].astype(int) - 127, e) and np.array_equal(c.k.view(torch.uint8).cpu().numpy()[0, 0, :n], codes)


@pytest.mark.gpu
@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("before", ["append", "append_rotated"])
@pytest.mark.parametrize("batch,hq,hkv,ps,held,rows", [(3, 4, 2, 16, 5, 1), (3, 4, 2, 64, 17, 20), (2, 8, 1, 256, 100, 70), (2, 28, 4, 64, 63, 40), (300, 2, 2, 64, 30, 20), (3, 0, 2, 32, 1, 30), (40, 8, 2, 16, 15, 3)])
def test_bounds_of_pages_that_held_rows_before(e4m3, before, batch, hq, hkv, ps, held, rows):
    """A page begun by one call and filled by the next ones: least and largest of all its keys; by a workgroup of its own or several that share its heads."""
    rng = np.random.default_rng(held)
    columns = -(-(held + 2 * rows + batch) // ps)
    c = pools(batch * columns, hkv, ps, e4m3)
    lengths = torch.zeros(batch, dtype=torch.int32, device=DEV)
    s = c.sequences(ints(rng.permutation(batch * columns).reshape(batch, columns)), lengths)
    r = ckv.Rotation(torch.from_numpy(10000.0 ** (-np.arange(64) / 64)).to(DEV))
    n = held + np.arange(batch) % (batch if batch < 50 else 7)
    for count in (int(n.max()), rows, rows):
        new = [device(rng.standard_normal((batch, count, h, 128)) * 2.0 ** rng.integers(-2, 3)) for h in (max(hq, 1), hkv, hkv)]
        if int(lengths.max()) == 0:
            lengths.copy_(ints(n))
            first = dict(first=torch.zeros_like(lengths))
        else:
            lengths.add_(count)
            first = {}
        if int(n.max()) == count and before == "append" and first:
            c.append(s, *new[1:], **first)
        else:
            c.append_rotated(s, new[0] if hq else None, *new[1:], r, **first)
        told = lengths.tolist()
        keys, _ = c.read(s, max(told), first=torch.zeros_like(lengths))
        keys, bounds, table = keys.double().cpu().numpy(), c.bounds.double().cpu().numpy(), s.table.cpu().numpy()
        for b in range(0, batch, max(1, batch // 9)):
            for p in range(-(-told[b] // ps)):
                for h in range(hkv):
                    lo, hi = ref.extremes(keys[b, p * ps:min((p + 1) * ps, told[b]), h])
                    assert np.array_equal(bounds[table[b, p], h, 0], lo) and np.array_equal(bounds[table[b, p], h, 1], hi), f"page {p} of sequence {b}, head {h}, {told[b]} entries"
    assert c.status() == 0
