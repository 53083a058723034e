"""Attention of several rows where one sequence is much longer than the others: its blocks fall into pieces for the whole chip, others into few or none."""
import numpy as np
import pytest
import torch

from oracle import paged as ref
from tests.paged import DEV, bf16, device, pools
from tests.rows import check_rows, random_tree

pytestmark = pytest.mark.gpu

# batch, KV heads, query heads for each, rows, longest, e4m3
CASES = [(20, 4, 5, 25, 40000, False), (70, 2, 4, 64, 30000, True), (70, 1, 4, 8, 95000, False), (600, 1, 1, 9, 40000, True), (16, 1, 4, 300, 40000, True)]


def ints(x):
    return torch.as_tensor(np.asarray(x, np.int32)).to(DEV)


class Ragged:
    """Sequences of the given lengths in a cache, as tests.paged.Filled, their rows appended packed: nothing is as large as the batch times the longest."""

    def __init__(self, lengths, hkv, ps, e4m3, seed):
        self.rng = np.random.default_rng(seed)
        self.lengths, self.hkv = list(lengths), hkv
        held = [-(-n // ps) for n in lengths]
        self.cache = pools(sum(held) + 3, hkv, ps, e4m3)
        order = self.rng.permutation(sum(held) + 3)
        self.table = np.full((len(lengths), max(held)), -7, np.int32)
        starts = np.cumsum([0, *held])
        for b, n in enumerate(held):
            self.table[b, :n] = order[starts[b]:starts[b + 1]]
        self.seqs = self.cache.sequences(ints(self.table), ints(self.lengths))
        rows = [torch.from_numpy(self.rng.standard_normal((sum(lengths), hkv, 128), np.float32)).bfloat16() for _ in range(2)]
        starts = np.cumsum([0, *lengths])
        self.cache.append(self.seqs, *(x.to(DEV) for x in rows), rows=max(lengths), starts=ints(starts))
        held = (lambda x: ref.dequantise(*ref.quantise(x))) if e4m3 else (lambda x: x)
        self.k, self.v = ({b: [held(x[starts[b]:starts[b + 1], h].double().numpy()) for h in range(hkv)] for b in self.some()} for x in rows)

    def some(self):
        """The sequences that are looked at: the first and last, the longest, and a few others."""
        batch = len(self.lengths)
        return sorted({0, 1, int(np.argmax(self.lengths)), batch - 1, *range(3, batch, 97)})


def short(batch, longest, rows, seed):
    """Lengths: an empty one, some shorter than the call's rows, and one that is longest, in the middle."""
    rng = np.random.default_rng(seed)
    n = [int(x) for x in rng.integers(0, 300, batch)]
    n[0], n[batch // 2] = min(5, rows - 1), longest
    if batch > 4:
        n[1], n[-1] = 0, 700
    return n


@pytest.mark.parametrize("batch,hkv,g,rows,longest,e4m3", CASES)
@pytest.mark.parametrize("tree", [False, True])
def test_one_long_sequence(batch, hkv, g, rows, longest, e4m3, tree):
    if tree and rows > 64:
        rows = 64
    lengths = short(batch, longest, rows, longest)
    counts = [min(n, rows) for n in lengths]
    f = Ragged(lengths, hkv, 64, e4m3, batch)
    q = bf16(f.rng.standard_normal((batch, rows, hkv * g, 128)))
    out = torch.full(q.shape, -77.0, device=DEV)
    trees = [random_tree(f.rng, rows) for _ in lengths] if tree else None
    how = dict(f32=True, lse=True, **(dict(tree=torch.from_numpy(np.stack(trees)).to(DEV)) if tree else {}))
    first = ints([n - c for n, c in zip(lengths, counts)])
    _, lse = f.cache.attend_rows(f.seqs, device(q), first=first, out=out, **how)
    check_rows(f, q, out, counts, trees=trees, lse=lse, only=f.some())
    for b in range(batch):
        assert (out[b, counts[b]:] == -77.0).all(), "rows behind a sequence's last were written"
    assert torch.isfinite(out).all() and f.cache.status() == 0
    again = torch.full(q.shape, -77.0, device=DEV)
    f.cache.attend_rows(f.seqs, device(q), first=first, out=again, **how)
    assert torch.equal(out, again), "the same call, the same bits"
    packed = torch.cat([device(q)[b, :n] for b, n in enumerate(counts)])
    rag, _ = f.cache.attend_rows(f.seqs, packed, rows=rows, starts=ints(np.cumsum([0] + counts)), **how)
    assert torch.equal(rag, torch.cat([out[b, :n] for b, n in enumerate(counts)]))


def test_the_long_one_changes_between_replays():
    """One captured call; lengths swap among sequences that share their pages, so that now one and now another is long, none is, or all are."""
    batch, rows, g, longest = 200, 8, 4, 40000
    f = Ragged([longest] + [64] * 3, 1, 64, True, 4)
    table = torch.from_numpy(f.table[[0] * batch]).to(DEV)
    lengths = torch.full((batch,), 300, dtype=torch.int32, device=DEV)
    seqs = f.cache.sequences(table, lengths, longest)
    q = bf16(f.rng.standard_normal((batch, rows, g, 128)))
    x = device(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        f.cache.attend_rows(seqs, x, f32=True, lse=True)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = f.cache.attend_rows(seqs, x, f32=True, lse=True)
    k, v = f.k[0][0], f.v[0][0]
    for turn in range(6):
        n = [300 + 7 * b for b in range(batch)]
        if turn in (1, 3):
            n[turn * 51] = longest
        if turn == 4:
            n = [longest - 13 * b for b in range(batch)]
        lengths.copy_(ints(n))
        out.fill_(-77.0)
        graph.replay()
        want, sums = f.cache.attend_rows(seqs, x, f32=True, lse=True)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, sums), f"replay {turn}"
        f.lengths, f.k, f.v = n, [[k[:m]] for m in n], [[v[:m]] for m in n]
        check_rows(f, q, out, [rows] * batch, lse=lse, only=[0, 51, 153, batch - 1])


def test_lengths_that_are_wrong_beside_a_long_one():
    """Reported, left out, and the others' pieces found all the same."""
    f = Ragged([200] * 78 + [60000, 100], 2, 64, True, 8)
    lengths = f.seqs.lengths.clone()
    lengths[3], lengths[7] = -4, 10 ** 9
    seqs = f.cache.sequences(f.seqs.table, lengths, 60000)
    q = bf16(f.rng.standard_normal((80, 16, 8, 128)))
    first = ints([n - 16 for n in f.lengths])
    first[7] = 59000
    first[5] = 201
    out = torch.full(q.shape, -77.0, device=DEV)
    f.seqs.table[7] = -1
    f.cache.attend_rows(seqs, device(q), first=first, out=out, f32=True)
    assert f.cache.status() & 2
    assert (out[3] == -77.0).all() and (out[5] == -77.0).all()
    check_rows(f, q, out, [16] * 80, only=[0, 1, 78, 79])


@pytest.mark.parametrize("tree", [False, True])
def test_one_long_sequence_through_a_wide_window(tree):
    batch, hkv, g, rows, longest = 70, 2, 4, 64, 30000
    lengths = short(batch, longest, rows, 1)
    counts = [min(n, rows) for n in lengths]
    f = Ragged(lengths, hkv, 64, True, 5)
    q = bf16(f.rng.standard_normal((batch, rows, hkv * g, 128)))
    trees = [random_tree(f.rng, rows) for _ in lengths] if tree else None
    how = dict(window=20000, sinks=70, f32=True, lse=True, **(dict(tree=torch.from_numpy(np.stack(trees)).to(DEV)) if tree else {}))
    out, lse = f.cache.attend_rows(f.seqs, device(q), first=ints([n - c for n, c in zip(lengths, counts)]), **how)
    check_rows(f, q, out, counts, window=20000, sinks=70, trees=trees, lse=lse, only=f.some())
    assert f.cache.status() == 0
