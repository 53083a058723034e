"""Rows that enter the cache in pages with their positions' rotation, on the GPU against the definition in 64 bits (oracle/paged.py)."""
import numpy as np
import pytest
import torch

from oracle import paged as ref
from paper_2601_16986_amd import ckv
from tests.paged import DEV, LAYOUTS, bf16, device, pools

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.as_tensor(np.asarray(x, np.int32)).to(DEV)


def frequencies(n, base=10000.0):
    return base ** (-np.arange(n) / n)


def rotation(f, **how):
    return ckv.Rotation(torch.from_numpy(np.asarray(f, np.float64)).to(DEV), **how)


def off(x, f, interleaved, magnitude):
    """How far a turned value may be from the definition before its rounding: sine and cosine are rounded to float (2^-24 each relative), so are the smaller product and
    the sum: at most 3 * 2^-24 of |x| + |y|, and angles of up to 2^31 * 1 rad in 64 bits are off by 2^31 * 2^-52 of it."""
    return ref.pair_size(x, len(f), interleaved) * magnitude * (3 * 2.0 ** -24 + 2.0 ** -21)


def check_bf16(got, x, y, b, what):
    """bf16 values: the definition's, rounded by at most 2^-8 of itself."""
    bad = np.abs(got - y) > b + 2.0 ** -8 * (np.abs(y) + b)
    assert not bad.any(), f"{what}: {got[bad][:4]}, {y[bad][:4]} expected"


def check_codes(codes, e, y, b, what):
    """A row's codes and power of two: those of values within the bound of the definition's."""
    big, slack = np.abs(y).max(-1), b.max(-1)
    for i in np.ndindex(e.shape):
        lo = ref.quantise(np.array([max(big[i] - slack[i], 0)]))[1]
        hi = ref.quantise(np.array([big[i] + slack[i]]))[1]
        assert lo <= e[i] <= hi, f"{what}: 2^{e[i]} for a magnitude of {big[i]}"
    scale = np.exp2(e.astype(float))[..., None]
    v = ref.E4M3[codes]
    for sign in (-1, 1):
        near = ref.E4M3[ref.e4m3_codes(np.clip((y + sign * b) / scale, -448, 448))]
        assert (sign * v <= sign * near).all(), f"{what}: a code is not that of its value"


class Setup:
    """A cache of poisoned pools with sequences of the given lengths, and rows for it: the last counts[b] of each."""

    def __init__(self, lengths, counts, hq, hkv, ps, e4m3, layout="plain", seed=0, bounds=True, spread=1.0):
        rng = np.random.default_rng(seed)
        self.lengths, self.counts, self.hq, self.hkv, self.ps, self.e4m3 = lengths, counts, hq, hkv, ps, e4m3
        held = [-(-n // ps) for n in lengths]
        self.cache = pools(sum(held) + 2, hkv, ps, e4m3, layout, bounds)
        order, at = rng.permutation(sum(held) + 2), 0
        self.table = np.full((len(lengths), max(max(held), 1)), -3, np.int32)
        for b, n in enumerate(held):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.seqs = self.cache.sequences(ints(self.table), ints(lengths))
        self.most = max(max(counts), 1)
        shape = (len(lengths), self.most)
        self.q, self.k, self.v = (bf16(rng.standard_normal((*shape, h, 128)) * spread) for h in (hq, hkv, hkv))
        self.first = [n - c for n, c in zip(lengths, counts)]
        self.at = np.array(self.first)[:, None] + np.arange(self.most)

    def check(self, turned, positions, f, interleaved=False, magnitude=1.0, whole=True):
        """turned: the queries, [batch][most][hq][128] with -77 where nothing may have been written."""
        c = self.cache
        raw = [x.view(torch.uint8 if self.e4m3 else torch.int16).cpu().numpy() for x in (c.k, c.v)]
        scales = c.scales.cpu().numpy().astype(int) if self.e4m3 else None
        bounds = c.bounds.double().cpu().numpy() if c.bounds is not None else None
        seen = np.zeros(raw[0].shape[:3], bool)
        got_q = turned.double().cpu().numpy() if turned is not None else None
        for b, (n, count) in enumerate(zip(self.lengths, self.counts)):
            mine = np.asarray(positions[b][:count])
            if got_q is not None:
                y = ref.rotate(self.q[b, :count], mine, f, interleaved, magnitude)
                check_bf16(got_q[b, :count], self.q[b, :count], y, off(self.q[b, :count], f, interleaved, magnitude), f"queries of sequence {b}")
                assert (got_q[b, count:] == -77.0).all(), "queries behind a sequence's last were written"
            y, slack = ref.rotate(self.k[b, :count], mine, f, interleaved, magnitude), off(self.k[b, :count], f, interleaved, magnitude)
            for i in range(count):
                page, slot = self.table[b, (self.first[b] + i) // self.ps], (self.first[b] + i) % self.ps
                seen[page, :, slot] = True
                key, value = raw[0][page, :, slot], raw[1][page, :, slot]
                if self.e4m3:
                    check_codes(key, scales[page, :, slot, 0] - 127, y[i], slack[i], f"key {i} of sequence {b}")
                    codes, e = ref.quantise(self.v[b, i])
                    assert np.array_equal(value, codes) and np.array_equal(scales[page, :, slot, 1] - 127, e), f"value {i} of sequence {b}"
                else:
                    check_bf16(torch.from_numpy(key).view(torch.bfloat16).double().numpy(), None, y[i], slack[i], f"key {i} of sequence {b}")
                    assert np.array_equal(torch.from_numpy(value).view(torch.bfloat16).double().numpy(), self.v[b, i])
            if bounds is not None and whole:                   # extremes of the keys as they lie there now
                for p0 in range(self.first[b] // self.ps * self.ps, self.first[b] + count if count else 0, self.ps):
                    page = self.table[b, p0 // self.ps]
                    a, z = max(p0, self.first[b]) - p0, min(p0 + self.ps, self.lengths[b]) - p0
                    if a:
                        continue                               # what its bounds were before is poison here
                    for h in range(self.hkv):
                        rows = raw[0][page, h, a:z]
                        rows = ref.dequantise(rows, scales[page, h, a:z, 0] - 127) if self.e4m3 else torch.from_numpy(rows).view(torch.bfloat16).double().numpy()
                        lo, hi = ref.extremes(rows)
                        assert np.array_equal(bounds[page, h, 0], lo) and np.array_equal(bounds[page, h, 1], hi), f"extremes of sequence {b} head {h} from {p0}"
        for side in (0, 1):
            assert (raw[side][~seen] == (0x7F if self.e4m3 else 0x7FC0)).all(), "a row outside the call's was written"


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("hq,hkv,pairs,ps,lengths,counts", [
    (1, 1, 64, 16, [1], [1]), (8, 2, 64, 16, [5, 33, 0, 16], [5, 33, 0, 16]), (28, 4, 32, 64, [100, 64, 65, 7], [3, 64, 1, 0]), (5, 5, 8, 256, [300, 257], [200, 257]),
    (16, 1, 56, 32, [40, 70], [17, 15]), (40, 8, 64, 128, [129, 1000], [2, 13]), (9, 3, 40, 16, [90], [90])])
def test_rows_are_turned_and_written(e4m3, interleaved, hq, hkv, pairs, ps, lengths, counts):
    s = Setup(lengths, counts, hq, hkv, ps, e4m3, LAYOUTS[hq % 3], seed=hq)
    f = frequencies(pairs)
    out = torch.full((len(lengths), s.most, hq, 128), -77.0, dtype=torch.bfloat16, device=DEV)
    got = s.cache.append_rotated(s.seqs, device(s.q), device(s.k), device(s.v), rotation(f, interleaved=interleaved), first=ints(s.first), out=out)
    assert got is out
    s.check(out, s.at, f, interleaved)
    assert s.cache.status() == 0


@pytest.mark.parametrize("e4m3", [True, False])
def test_packed_rows_positions_of_their_own_and_a_magnitude(e4m3):
    """Drafted tokens: several rows share a position; far ones and negative ones too."""
    lengths, counts = [70, 9, 40], [20, 0, 33]
    s = Setup(lengths, counts, 6, 2, 16, e4m3, seed=3)
    rng = np.random.default_rng(5)
    positions = [rng.integers(-5, 200000, s.most) for _ in lengths]
    positions[0][:4] = [2 ** 31 - 1, -2 ** 31, 0, 1048577]
    f = frequencies(64, 1e6)
    packed = [device(np.concatenate([x[b, :n] for b, n in enumerate(counts)])) for x in (s.q, s.k, s.v)]
    starts = ints(np.cumsum([0] + counts))
    got = s.cache.append_rotated(s.seqs, *packed, rotation(f, magnitude=1.25), positions=ints(np.concatenate([p[:n] for p, n in zip(positions, counts)])), rows=33, starts=starts)
    turned = torch.full((3, s.most, 6, 128), -77.0, dtype=torch.bfloat16, device=DEV)
    for b, n in enumerate(counts):
        turned[b, :n] = got[sum(counts[:b]):sum(counts[:b + 1])]
    s.check(turned, positions, f, magnitude=1.25)
    assert s.cache.status() == 0


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("interleaved", [False, True])
def test_single_rows_of_a_fused_projection_in_place(e4m3, interleaved):
    """One token of each sequence, all three out of one tensor, the queries turned where they lie."""
    lengths = [1, 16, 17, 300]
    s = Setup(lengths, [1] * 4, 8, 2, 16, e4m3, seed=4)
    fused = torch.full((4, 14, 128), 5.0, dtype=torch.bfloat16, device=DEV)
    fused[:, 1:9], fused[:, 9:11], fused[:, 11:13] = device(s.q[:, 0]), device(s.k[:, 0]), device(s.v[:, 0])
    f = frequencies(64, 500000.0)
    q = fused[:, 1:9]
    assert s.cache.append_rotated(s.seqs, q, fused[:, 9:11], fused[:, 11:13], rotation(f, interleaved=interleaved), out=q) is q
    s.check(q[:, None], s.at, f, interleaved)
    assert (fused[:, 0] == 5).all() and (fused[:, 13] == 5).all() and torch.equal(fused[:, 9:11], device(s.k[:, 0])) and torch.equal(fused[:, 11:13], device(s.v[:, 0]))


def test_keys_alone_and_no_bounds():
    s = Setup([50, 20], [50, 20], 2, 2, 32, True, seed=6, bounds=False)
    f = frequencies(64)
    assert s.cache.append_rotated(s.seqs, None, device(s.k), device(s.v), rotation(f), first=ints(s.first)) is None
    s.check(None, s.at, f)


@pytest.mark.parametrize("interleaved", [False, True])
def test_no_turn_at_position_nothing_is_a_plain_append(interleaved):
    """Angles of nothing: rows as append writes them, bit by bit, queries as they were; infinities and no numbers stay in their pairs."""
    for e4m3 in (True, False):
        s, t = (Setup([60, 5], [60, 5], 4, 2, 16, e4m3, seed=7, spread=3.0) for _ in range(2))
        out = s.cache.append_rotated(s.seqs, device(s.q), device(s.k), device(s.v), rotation(frequencies(64), interleaved=interleaved),
                                     positions=torch.zeros((2, 60), dtype=torch.int32, device=DEV), first=ints(s.first))
        t.cache.append(t.seqs, device(s.k), device(s.v), first=ints(s.first))
        assert torch.equal(out[0], device(s.q)[0]) and torch.equal(out[1, :5], device(s.q)[1, :5])
        for a, b in ((s.cache.k, t.cache.k), (s.cache.v, t.cache.v)):
            assert torch.equal(a.view(torch.uint8 if e4m3 else torch.int16), b.view(torch.uint8 if e4m3 else torch.int16))
        assert torch.equal(s.cache.bounds.nan_to_num(9), t.cache.bounds.nan_to_num(9))
        if e4m3:
            assert torch.equal(s.cache.scales, t.cache.scales)
    x = torch.ones((1, 1, 2, 128), dtype=torch.bfloat16, device=DEV)
    x[0, 0, 0, 6], x[0, 0, 1, 9], x[0, 0, 1, 126] = float("inf"), float("nan"), -float("inf")
    for e4m3 in (True, False):
        s = Setup([3], [1], 2, 2, 16, e4m3)
        out = s.cache.append_rotated(s.seqs, x, x, x, rotation(frequencies(32), interleaved=interleaved))
        k, _ = s.cache.read(s.seqs, 1)
        mates = (7, 8, 127) if interleaved else (38, 41, 126)
        for y in (out, k):
            odd = ~torch.isfinite(y[0, 0])
            assert sorted(torch.nonzero(odd[0]).flatten().tolist()) == sorted({6, mates[0]})
            assert sorted(torch.nonzero(odd[1]).flatten().tolist()) == sorted({9, mates[1], 126})
            assert (y[0, 0][~odd] != 0).all()


def test_wrong_pages_and_lengths():
    """The indexes are those of append (checked on the CPU): rows without a page are left out of the cache, their queries turned all the same; rows that do not fit are left alone."""
    s = Setup([40, 20], [40, 20], 2, 1, 16, True, seed=8)
    f = frequencies(64)
    good = s.seqs.table.clone()
    s.seqs.table[0, 1] = 10 ** 9
    out = torch.full((2, 40, 2, 128), -77.0, dtype=torch.bfloat16, device=DEV)
    s.cache.append_rotated(s.seqs, device(s.q), device(s.k), device(s.v), rotation(f), first=ints(s.first), out=out)
    assert s.cache.status() == ckv.BAD_PAGE
    y = ref.rotate(s.q[0], s.at[0], f)
    check_bf16(out[0].double().cpu().numpy(), None, y, off(s.q[0], f, False, 1.0), "queries")
    page = int(good[0, 1])
    assert (s.cache.k.view(torch.uint8)[page] == 0x7F).all() and (s.cache.scales[page] == 255).all()
    s.seqs.table.copy_(good)
    t = Setup([40, 20], [40, 20], 2, 1, 16, True, seed=8)
    out.fill_(-77.0)
    t.cache.append_rotated(t.seqs, device(s.q), device(s.k), device(s.v), rotation(f), first=ints([41, -1]), out=out)
    assert t.cache.status() == ckv.BAD_LENGTH and (out == -77.0).all() and (t.cache.k.view(torch.uint8) == 0x7F).all()
    u = Setup([40, 20], [40, 20], 2, 1, 16, True, seed=8)
    u.seqs.lengths[0] = 60                                      # beyond the columns' 48: what lies below is written at its place
    u.cache.append_rotated(u.cache.sequences(u.seqs.table, u.seqs.lengths, 40), device(s.q), device(s.k), device(s.v), rotation(f), first=ints([0, 0]), out=out)
    assert u.cache.status() == ckv.BAD_LENGTH
    u.check(out, u.at, f, whole=False)


def test_a_captured_step_replayed():
    """Tokens enter again and again in a graph, beside eager calls on another cache."""
    s, t = (Setup([60, 33], [1, 1], 4, 2, 16, True, seed=9) for _ in range(2))
    r = rotation(frequencies(64))
    q, k, v = (torch.zeros((2, h, 128), dtype=torch.bfloat16, device=DEV) for h in (4, 2, 2))
    for x in (s, t):
        x.seqs.lengths.copy_(ints([10, 3]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.cache.append_rotated(s.seqs, q, k, v, r)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = s.cache.append_rotated(s.seqs, q, k, v, r)
    t.cache.append_rotated(t.seqs, q, k, v, r)
    rng = np.random.default_rng(1)
    for n in range(6):
        for x in (s, t):
            x.seqs.lengths.add_(1)
        for to in (q, k, v):
            to.copy_(torch.from_numpy(rng.standard_normal(tuple(to.shape))))
        graph.replay()
        want = t.cache.append_rotated(t.seqs, q, k, v, r)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(s.cache.k.view(torch.uint8), t.cache.k.view(torch.uint8)) and torch.equal(s.cache.scales, t.cache.scales)
        assert torch.equal(s.cache.bounds.nan_to_num(7.0), t.cache.bounds.nan_to_num(7.0))
    assert s.cache.status() == 0


def test_refusals_of_the_binding():
    s = Setup([20], [4], 4, 2, 16, True)
    q, k, v = (device(x) for x in (s.q, s.k, s.v))
    r, i = rotation(frequencies(64)), torch.zeros((1, 4), dtype=torch.int32, device=DEV)
    c = s.cache
    for bad in (lambda: c.append_rotated(s.seqs, q[:, :3], k, v, r), lambda: c.append_rotated(s.seqs, q.float(), k, v, r), lambda: c.append_rotated(s.seqs, q[..., :64], k, v, r),
                lambda: c.append_rotated(s.seqs, q[:, :, :3], k, v, r), lambda: c.append_rotated(s.seqs, q.cpu(), k, v, r), lambda: c.append_rotated(s.seqs, q, k, v, r, out=q[:, :2]),
                lambda: c.append_rotated(s.seqs, None, k, v, r, out=q), lambda: c.append_rotated(s.seqs, q, k, v, r, positions=i[:, :3]), lambda: c.append_rotated(s.seqs, q, k, v, r, positions=i.long()),
                lambda: c.append_rotated(s.seqs, q, k, v, r, out=torch.empty_like(q, dtype=torch.float32)), lambda: c.append_rotated(s.seqs, q[0], k[0], v[0], r, starts=torch.zeros(2, dtype=torch.int32, device=DEV)),
                lambda: rotation(frequencies(7)) and c.append_rotated(s.seqs, q, k, v, rotation(frequencies(7))), lambda: c.append_rotated(s.seqs, q, k, v, rotation(frequencies(72))),
                lambda: c.append_rotated(s.seqs, q, k, v, rotation(frequencies(64), magnitude=float("nan"))), lambda: c.append_rotated(s.seqs, q, k, v, rotation(frequencies(64), magnitude=-1.0)),
                lambda: ckv.Rotation(torch.zeros(64, device=DEV)), lambda: ckv.Rotation(torch.zeros((2, 64), dtype=torch.float64, device=DEV)), lambda: ckv.Rotation(torch.zeros(64, dtype=torch.float64))):
        with pytest.raises(ckv.CkvError):
            bad()
