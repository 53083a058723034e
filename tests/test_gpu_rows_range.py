"""Attention of several rows over a cache in pages: finite values as large as they come, whose weighted sums are finite only once they are divided by the weights."""
import numpy as np
import pytest
import torch

from tests.paged import DEV, Filled, bf16, device
from tests.rows import check_rows

pytestmark = pytest.mark.gpu

LARGE = 1.5 * 2.0 ** 127                     # e4m3 times a power of two has it


def ints(x):
    return torch.as_tensor(np.asarray(x, np.int32)).to(DEV)


def filled(lengths, hkv, ps, e4m3, seed, large, signs=(1.0,)):
    """Values between LARGE / 2 and LARGE, of these signs, in the entries of which `large` (a function of positions) holds; of size 1 in the others."""
    def make(rng, shape):
        k, v = bf16(rng.standard_normal(shape)), bf16(rng.standard_normal(shape))
        at = np.broadcast_to(large(np.arange(shape[1]))[None, :, None, None], shape)
        return k, np.where(at, bf16(rng.uniform(0.5, 1.0, shape) * rng.choice(signs, shape) * LARGE), v)

    return Filled(lengths, hkv, ps, e4m3, seed=seed, make=make)


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("rows,hq,packed", [(1, 8, True), (3, 4, False), (9, 10, False), (70, 6, True)])
@pytest.mark.parametrize("which", ["all", "first half", "now and then"])
def test_large_values(e4m3, f32, rows, hq, packed, which):
    """Whole sequences of them, in one piece and in many; beside pieces without; a few in every tile."""
    large = {"all": lambda e: e >= 0, "first half": lambda e: e < 1500, "now and then": lambda e: e % 29 == 3}[which]
    lengths = [3000, 75, 700]
    f = filled(lengths, 2, 64, e4m3, rows, large)
    assert all(np.isfinite(v).all() for s in f.v for v in s)
    q = bf16(f.rng.standard_normal((3, rows, hq, 128)))
    x = device(q)
    if packed:
        x = x.view(3 * rows, hq, 128)
        out, lse = f.cache.attend_rows(f.seqs, x, rows=rows, starts=ints(np.arange(4) * rows), f32=f32, lse=True)
        out, lse = out.view(q.shape), lse.view(q.shape[:3])
    else:
        out, lse = f.cache.attend_rows(f.seqs, x, f32=f32, lse=True)
    check_rows(f, q, out, [rows] * 3, lse=lse)


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("rows,hq", [(1, 8), (3, 4), (9, 10), (70, 6)])
@pytest.mark.parametrize("packed", [False, True])
def test_large_values_of_both_signs(e4m3, rows, hq, packed):
    """Sums that would be infinite one way and the other, which is no number; logits that rise from tile to tile so that weights above 1 meet them."""
    lengths = [900, 75]
    f = filled(lengths, 2, 64, e4m3, rows, lambda e: e % 3 > 0, signs=(-1.0, 1.0))
    keys, values = f.rows
    keys[..., 0] = bf16(np.arange(900) / 16)[None, :, None]
    f.cache.append(f.seqs, *(torch.from_numpy(x).to(DEV).bfloat16() for x in (keys, values)))
    f.k = [[f.held(keys[b, :n, h]) for h in range(2)] for b, n in enumerate(lengths)]
    q = bf16(f.rng.standard_normal((2, rows, hq, 128)))
    q[..., 0] = 4.0
    if packed:
        out, lse = f.cache.attend_rows(f.seqs, device(q).view(2 * rows, hq, 128), rows=rows, starts=ints(np.arange(3) * rows), f32=True, lse=True)
        out, lse = out.view(q.shape), lse.view(q.shape[:3])
    else:
        out, lse = f.cache.attend_rows(f.seqs, device(q), f32=True, lse=True)
    assert torch.isfinite(out).all()
    check_rows(f, q, out, [rows] * 2, lse=lse)


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("rows,hq", [(1, 8), (3, 4), (70, 6)])
@pytest.mark.parametrize("packed", [False, True])
def test_sums_that_are_no_number_and_nowhere_large(e4m3, rows, hq, packed):
    """One dimension alone, large and positive in the first tiles, large and negative, with weights of 2^7 relative to those, in the later ones: what it would add up to is infinity less infinity, in no
    other place anything is large.  So many sequences (all of the same pages) that none is cut."""
    batch = 700
    f = Filled([256 + rows], 2, 64, e4m3, seed=rows)
    keys, values = f.rows
    keys[0, :128, :, 0], keys[0, 128:256, :, 0], keys[0, 256:, :, 0] = 0.0, 5.0, -5.0
    values[0, :128, :, 7], values[0, 128:256, :, 7] = LARGE, -LARGE
    f.cache.append(f.seqs, *(torch.from_numpy(x).to(DEV).bfloat16() for x in f.rows))
    f.k, f.v = ([[f.held(x[0, :, h]) for h in range(2)]] for x in (keys, values))
    seqs = f.cache.sequences(torch.from_numpy(f.table[[0] * batch]).to(DEV), torch.full((batch,), f.lengths[0], dtype=torch.int32, device=DEV))
    q = bf16(f.rng.standard_normal((1, rows, hq, 128)) / 16)
    q[..., 0] = 1.0
    x = device(q).expand(batch, rows, hq, 128).contiguous()
    if packed:
        out, lse = f.cache.attend_rows(seqs, x.view(batch * rows, hq, 128), rows=rows, starts=ints(np.arange(batch + 1) * rows), scale=1.0, f32=True, lse=True)
        out, lse = out.view(x.shape), lse.view(x.shape[:3])
    else:
        out, lse = f.cache.attend_rows(seqs, x, scale=1.0, f32=True, lse=True)
    assert torch.isfinite(out).all() and torch.equal(out[0], out[699])
    check_rows(f, q, out[:1], [rows], lse=lse[:1], scale=1.0)


@pytest.mark.parametrize("e4m3", [True, False])
def test_weights_above_one_of_large_values(e4m3):
    """The running maximum follows logits with some slack: entries of logit 0, then one of 5.4 (2^7.8) with a value of 2^123, which 2^7.8 times would not be finite."""
    n, at = 200, 150
    f = Filled([n], 1, 16, e4m3, seed=1, make=lambda rng, shape: (np.zeros(shape), np.zeros(shape)))
    k, v = (np.zeros((1, n, 1, 128)) for _ in range(2))
    k[0, at, 0, 0], v[0, at, 0, :] = 5.5, 2.0 ** 123
    f.cache.append(f.seqs, device(k), device(v))
    f.k, f.v = ([[f.held(x[0, :, 0])]] for x in (k, v))
    q = np.zeros((1, 3, 2, 128))
    q[..., 0] = 1.0
    out, lse = f.cache.attend_rows(f.seqs, device(q), scale=5.4 / 5.5, f32=True, lse=True)
    assert torch.isfinite(out).all()
    check_rows(f, q, out, [3], lse=lse, scale=5.4 / 5.5)


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("rows,hq", [(6, 4), (40, 4)])
@pytest.mark.parametrize("n", [200, 3000])
def test_rows_are_not_told_of_large_values_that_they_do_not_see(e4m3, rows, hq, n):
    """Drafts in two branches, of which one sees large values: the other's outputs are bit by bit those without them."""
    i = np.arange(rows)
    trees = [(i[:, None] >= i) & ((i[:, None] - i) % 2 == 0)]
    f = Filled([n], 1, 16, e4m3, seed=rows)
    q = bf16(f.rng.standard_normal((1, rows, hq, 128)))
    how = dict(tree=torch.from_numpy(np.stack(trees)).to(DEV), lse=True, f32=True)
    clean, lse0 = f.cache.attend_rows(f.seqs, device(q), **how)
    at = [1, 3, 5]
    told = torch.from_numpy(trees[0][:, at].any(1)).to(DEV)
    assert told.any() and not told.all()
    spread = torch.from_numpy(f.rows[1]).bfloat16()
    for j in at:
        spread[0, n - rows + j] = LARGE
        f.v[0][0][n - rows + j] = LARGE
    f.cache.append(f.seqs, torch.from_numpy(f.rows[0]).bfloat16().to(DEV), spread.to(DEV))
    out, lse = f.cache.attend_rows(f.seqs, device(q), **how)
    assert torch.equal(out[0, ~told], clean[0, ~told]) and torch.equal(lse, lse0)
    check_rows(f, q, out, [rows], trees=trees, lse=lse)
