"""A cache in pages on the device beside its definition on the CPU: pools, tables and rows for the tests of ckv_paged_*."""
from __future__ import annotations

import numpy as np
import torch

from oracle import paged as ref
from paper_2601_16986_amd import ckv

DEV = "cuda:0"
LAYOUTS = ("plain", "slots_first", "layers")


def bf16(x):
    """Numbers on the bf16 grid, float64."""
    return torch.as_tensor(np.asarray(x, np.float32)).bfloat16().double().numpy()


def pools(n_pages, hkv, ps, e4m3, layout="plain", bounds=True, poison=True):
    """Pools in one of three orders, filled with NaN codes and with scales and bounds of nonsense, as memory that held something else may be."""
    dt = torch.float8_e4m3fn if e4m3 else torch.bfloat16

    def rows():
        if layout == "plain":
            x = torch.zeros((n_pages, hkv, ps, 128), dtype=dt, device=DEV)
        elif layout == "slots_first":
            x = torch.zeros((n_pages, ps, hkv, 128), dtype=dt, device=DEV).permute(0, 2, 1, 3)
        else:                                    # one of three layers that share an allocation, and heads with a gap between slots
            x = torch.zeros((n_pages, 3, hkv, ps, 144), dtype=dt, device=DEV)[:, 1, :, :, 16:]
        if poison:
            x.view(torch.uint8 if e4m3 else torch.int16).fill_(0x7F if e4m3 else 0x7FC0)
        return x

    some = (lambda *shape: (shape[0], 3, *shape[1:])) if layout == "layers" else (lambda *shape: shape)
    mine = (lambda x: x[:, 2]) if layout == "layers" else (lambda x: x)
    scales = mine(torch.full(some(n_pages, hkv, ps, 2), 255, dtype=torch.uint8, device=DEV)) if e4m3 else None
    b = mine(torch.full(some(n_pages, hkv, 2, 128), float("nan"), dtype=torch.bfloat16, device=DEV)) if bounds else None
    return ckv.PagedCache(rows(), rows(), scales=scales, bounds=b)


class Filled:
    """Sequences of the given lengths in a cache, their rows on both sides: k, v[b][h] = float64 [length][128], what the cache holds."""

    def __init__(self, lengths, hkv, ps, e4m3, layout="plain", seed=0, spread=1.0, columns=None, make=None, spare=3):
        rng = np.random.default_rng(seed)
        self.lengths, self.hkv, self.ps, self.e4m3, self.rng = list(lengths), hkv, ps, e4m3, rng
        held = [-(-n // ps) for n in lengths]
        n_pages = sum(held) + spare
        self.cache = pools(n_pages, hkv, ps, e4m3, layout)
        order = rng.permutation(n_pages)[:sum(held)]
        columns = columns or max(max(held), 1)
        table = np.full((len(lengths), columns), -7, np.int32)
        at = 0
        for b, n in enumerate(held):
            table[b, :n] = order[at:at + n]
            at += n
        self.table = table
        self.seqs = self.cache.sequences(torch.from_numpy(table).to(DEV), torch.tensor(self.lengths, dtype=torch.int32, device=DEV))
        most = max(max(lengths), 1)
        self.rows = [bf16(rng.standard_normal((len(lengths), most, hkv, 128)) * spread) for _ in range(2)] if make is None else make(rng, (len(lengths), most, hkv, 128))
        self.k, self.v = ([[self.held(side[b, :n, h]) for h in range(hkv)] for b, n in enumerate(self.lengths)] for side in self.rows)
        self.cache.append(self.seqs, *(torch.from_numpy(x).to(DEV).bfloat16() for x in self.rows))

    def held(self, x):
        return ref.dequantise(*ref.quantise(x)) if self.e4m3 else np.asarray(x, np.float64)

    def queries(self, hq, spread=1.0):
        return bf16(self.rng.standard_normal((len(self.lengths), hq, 128)) * spread)

    def page_rows(self, b, pages):
        """Row numbers of pages of a sequence, in the list's order."""
        return np.concatenate([np.arange(p * self.ps, min(self.lengths[b], (p + 1) * self.ps)) for p in pages if p >= 0] or [np.zeros(0)]).astype(int)


def device(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV).bfloat16()


def check_attention(f, q, out, lse=None, picked=None, scale=128 ** -0.5, what=""):
    """Outputs against the definition.  An entry's logit is a float sum of 128 products: off by at most 130 half steps (2^-24) of the sum of their
    magnitudes, and the exponential's argument by a few more of its own size, so a weight relative to the others by twice that, 2 * 2^-24 * 140 * reach. The weight's terms leave
    2^-8 each of what the one before left (two terms for bf16, three for float outputs), and at most 2^-24 per addition of some 512 that a wavefront or the join makes one after another
    (32 entries each at once).  All of that times the sum of |weight * value|; a bf16 output is rounded by 2^-8 of itself."""
    f32 = out.dtype == torch.float32
    y, hq = out.double().cpu().numpy(), q.shape[1]
    g = hq // f.hkv
    for b in range(len(f.lengths)):
        for i in range(hq):
            h = i // g
            k, v = f.k[b][h], f.v[b][h]
            if picked is not None:
                at = f.page_rows(b, picked[b][h])
                k, v = k[at], v[at]
            o, s, mass, reach = ref.attend(q[b, i], k, v, scale)
            bound = (2 * 140 * reach + 512) * 2.0 ** -24 + 2.0 ** (-24 if f32 else -16)
            tol = bound * mass + (0 if f32 else 2.0 ** -8 * (np.abs(o) + bound * mass)) + 1e-30
            off = np.abs(y[b, i] - o)
            assert np.all(off <= tol), f"{what} sequence {b} ({len(k)} entries) head {i}: off by {(off / tol).max():.2f} of the bound"
            if lse is not None:
                z = float(lse[b, i])
                if np.isinf(s):
                    assert z == s, f"{what} sequence {b} head {i}: lse {z}"
                else:
                    assert abs(z - s) <= bound + 2.0 ** -23 * abs(s) + 2.0 ** -22, f"{what} sequence {b} head {i}: lse {z}, {s} expected"
