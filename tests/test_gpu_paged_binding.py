"""The binding of the cache in pages as the readme uses it."""
import numpy as np
import torch
import pytest

from paper_2601_16986_amd import ckv
from tests.paged import DEV, Filled, bf16, device

pytestmark = pytest.mark.gpu


def test_the_readme_s_loop():
    """A prompt in, tokens one by one, all entries or picked pages, and the last rows into a budgeted context."""
    batch, hq, hkv, prompt, steps = 2, 8, 2, 200, 70
    n = prompt + steps
    f = Filled([n, n], hkv, 64, True, seed=1)                      # the same rows at once
    rows = [device(x) for x in f.rows]
    rng = np.random.default_rng(2)
    c = ckv.PagedCache.empty(12, 64, hkv, dtype=ckv.E4M3, bounds=True)
    table = torch.arange(10, dtype=torch.int32, device=DEV).view(2, 5)
    lengths = torch.full((batch,), prompt, dtype=torch.int32, device=DEV)
    s = c.sequences(table, lengths, n)
    c.append(s, *(x[:, :prompt] for x in rows))
    for t in range(steps):
        lengths += 1
        c.append(s, *(x[:, prompt + t].contiguous() for x in rows))
    q = device(bf16(rng.standard_normal((batch, hq, 128))))
    picked = c.select(s, q, 4)
    assert torch.equal(picked, f.cache.select(f.seqs, q, 4))
    for pages in (None, picked):
        assert torch.equal(c.attend(s, q, pages=pages)[0], f.cache.attend(f.seqs, q, pages=pages)[0])
    P = 150
    k, v = (torch.empty(batch, hkv, P, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    got = c.read(s, P, out=(k.transpose(1, 2), v.transpose(1, 2)))
    want = c.read(s, P)
    for a, b, x in zip(got, want, (k, v)):
        assert torch.equal(a, b) and torch.equal(x, b.transpose(1, 2))
    g = ckv.CrystalKV(1, batch, hq, hkv, 128, 256, np.full((1, batch, hkv), 200), t0=P, budget_max=255)
    g.load_prompt(0, k, v)
    e = g.export_unit(0, 1, 1)
    order = np.argsort(e["pos"])
    for side, x in (("K", k), ("V", v)):
        assert np.array_equal(e[side][order], x[1, 1].float().cpu().numpy())
    assert c.status() == 0 and g.status() == 0


def test_numbers_beyond_32_bits_are_refused():
    """Their lowest bits are numbers that the calls would take."""
    f = Filled([20], 2, 16, True)
    q, one = device(f.queries(4)), torch.zeros((1, 2, 128), dtype=torch.bfloat16, device=DEV)
    starts = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    before = f.cache.k.view(torch.uint8).clone()
    for bad in (lambda: f.cache.sequences(f.seqs.table, f.seqs.lengths, 2 ** 32 + 20), lambda: f.cache.append(f.seqs, one, one, rows=2 ** 32 + 1, starts=starts),
                lambda: f.cache.read(f.seqs, 2 ** 32 + 1, starts=starts, total=1), lambda: f.cache.select(f.seqs, q, 2, first=2 ** 32, last=0), lambda: f.cache.select(f.seqs, q, 2, first=0, last=2 ** 32 + 1),
                lambda: f.cache.sequences(f.seqs.table, f.seqs.lengths, -2 ** 32 + 20)):
        with pytest.raises(ckv.CkvError):
            bad()
    assert torch.equal(before, f.cache.k.view(torch.uint8))
