"""The cache in pages on the GPU against its definition in 64 bits (oracle/paged.py)."""
import numpy as np
import pytest
import torch

from oracle import paged as ref
from paper_2601_16986_amd import ckv
from tests.paged import DEV, LAYOUTS, Filled, bf16, check_attention, device, pools

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ rows
def _held(f, b, h, side):
    return (f.k, f.v)[side][b][h]


def _check_pools(f, upto=None):
    """Every row of every sequence bit by bit in the pools, everything else as it was, and the pages' extremes."""
    c = f.cache
    raw = [x.view(torch.uint8 if f.e4m3 else torch.int16).cpu().numpy() for x in (c.k, c.v)]
    scales = c.scales.cpu().numpy() if f.e4m3 else None
    bounds = c.bounds.double().cpu().numpy()
    seen = np.zeros(raw[0].shape[:3], bool)
    for b, n in enumerate(f.lengths):
        for h in range(f.hkv):
            for side in (0, 1):
                x = f.rows[side][b, :n, h]
                codes, e = ref.quantise(x) if f.e4m3 else (torch.from_numpy(x).bfloat16().view(torch.int16).numpy(), None)
                for c0 in range(0, n, f.ps):
                    page, m = f.table[b, c0 // f.ps], min(f.ps, n - c0)
                    got = raw[side][page, h, :m]
                    ok = (got == codes[c0:c0 + m]) if not f.e4m3 else (got == codes[c0:c0 + m]) | ((got & 0x7F) == 0x7F) & ((codes[c0:c0 + m] & 0x7F) == 0x7F)
                    assert ok.all(), f"sequence {b} head {h} side {side}, rows from {c0}"
                    if f.e4m3:
                        assert np.array_equal(scales[page, h, :m, side].astype(int) - 127, e[c0:c0 + m])
                    seen[page, h, :m] = True
                    if side == 0:
                        lo, hi = ref.extremes(_held(f, b, h, 0)[c0:c0 + m])
                        assert np.array_equal(bounds[page, h, 0], lo) and np.array_equal(bounds[page, h, 1], hi), f"extremes of sequence {b} head {h} page {c0 // f.ps}"
    for side in (0, 1):
        assert (raw[side][~seen] == (0x7F if f.e4m3 else 0x7FC0)).all(), "a row outside the sequences was written"
    if f.e4m3:
        assert (scales[~seen] == 255).all()


LENGTHS = [[1], [16, 0, 17, 1], [33, 64, 200, 5], [511, 300]]


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("lengths,hkv,ps", [(LENGTHS[0], 1, 16), (LENGTHS[1], 3, 16), (LENGTHS[2], 2, 64), (LENGTHS[3], 8, 256), (LENGTHS[2], 4, 32), (LENGTHS[3], 1, 128)])
def test_rows_go_in_and_come_back(e4m3, layout, lengths, hkv, ps):
    f = Filled(lengths, hkv, ps, e4m3, layout, seed=len(lengths) + ps)
    _check_pools(f)
    most = max(lengths)
    out = tuple(torch.full((len(lengths), most, hkv, 128), -77.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    f.cache.read(f.seqs, most, out=out)
    for side in (0, 1):
        got = out[side].double().cpu().numpy()
        for b, n in enumerate(lengths):
            for h in range(hkv):
                assert np.array_equal(got[b, :n, h], _held(f, b, h, side))
            assert (got[b, n:] == -77.0).all(), "rows behind a sequence's last are left alone"
    assert f.cache.status() == 0


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("ps", [16, 64])
def test_rows_that_come_in_parts(e4m3, ps):
    """A ragged prompt, then a chunk of another length each, then single tokens: as if written at once.  The parts come packed, padded with heads outermost, and
    as single rows out of a wider tensor."""
    f = Filled([100, 37, 0, 64], 2, ps, e4m3, seed=5)
    g = Filled([100, 37, 0, 64], 2, ps, e4m3, seed=5)
    for x in (g.cache.k, g.cache.v):
        x.view(torch.uint8 if e4m3 else torch.int16).fill_(0x7F if e4m3 else 0x7FC0)
    if e4m3:
        g.cache.scales.fill_(255)
    g.cache.bounds.fill_(float("nan"))
    kv = [device(x) for x in g.rows]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    lengths = g.seqs.lengths
    # packed
    first = [50, 30, 0, 10]
    starts = np.cumsum([0] + first).tolist()
    lengths.copy_(ints(first))
    g.cache.append(g.seqs, *(torch.cat([x[b, :n] for b, n in enumerate(first)]) for x in kv), rows=50, starts=ints(starts))
    # padded, heads outermost, one sequence without new rows
    upto = [90, 31, 0, 60]
    lengths.copy_(ints(upto))
    chunk = [torch.zeros((4, 2, 50, 128), dtype=torch.bfloat16, device=DEV) for _ in kv]
    for to, x in zip(chunk, kv):
        for b in range(4):
            to[b, :, :upto[b] - first[b]] = x[b, first[b]:upto[b]].transpose(0, 1)
    g.cache.append(g.seqs, *(x.transpose(1, 2) for x in chunk), first=ints(first))
    # single tokens, out of a fused projection's rows
    for n in range(90, 100):
        now = [n + 1, min(32 + n - 90, 37), 0, min(61 + n - 90, 64)]
        before = [n, min(31 + n - 90, 37), 0, min(60 + n - 90, 64)]
        lengths.copy_(ints(now))
        fused = torch.full((4, 12, 128), 9.0, dtype=torch.bfloat16, device=DEV)
        for b in range(4):
            if now[b] > 0:
                fused[b, 8:10], fused[b, 10:12] = kv[0][b, now[b] - 1], kv[1][b, now[b] - 1]
        if n % 2:
            g.cache.append(g.seqs, fused[:, 8:10], fused[:, 10:12])
        else:
            g.cache.append(g.seqs, fused[:, 8:10], fused[:, 10:12], first=ints(before))
    lengths.copy_(ints(f.lengths))
    _check_pools(g)
    assert g.cache.status() == 0
    # single rows and middles back, packed
    k, v = g.cache.read(g.seqs, 7, starts=ints([0, 7, 12, 12, 15]), total=20, first=ints([3, 32, 0, 20]), out=tuple(torch.full((20, 2, 128), 5.0, dtype=torch.bfloat16, device=DEV) for _ in kv))
    for side, got in enumerate((k.double().cpu().numpy(), v.double().cpu().numpy())):
        for h in range(2):
            want = np.concatenate([_held(g, 0, h, side)[3:10], _held(g, 1, h, side)[32:37], _held(g, 3, h, side)[20:23]])
            assert np.array_equal(got[:15, h], want)
        assert (got[15:] == 5.0).all()


def test_rows_of_unusual_values():
    """Every binade's largest and smallest magnitudes, halfway cases of every code, zeros, subnormal numbers, infinities and NaN."""
    def make(rng, shape):
        x = bf16(rng.standard_normal(shape) * np.exp2(rng.integers(-130, 120, shape[:-1])[..., None].astype(float)))
        y = bf16(rng.standard_normal(shape))
        grid = ref.E4M3[:127]
        half = np.concatenate([(grid[1:] + grid[:-1]) / 2, [448.0, -448.0]])
        x[0, 0, 0], x[0, 1, 0] = half, bf16(half * 2.0 ** -40)
        x[0, 2] = 0.0
        x[0, 3, 0] = bf16(2.0 ** -130 * np.arange(128))
        x[0, 4, 0, ::3], x[0, 4, 0, 1::3] = np.inf, -np.inf
        x[0, 5, 0, 7] = np.nan
        x[0, 6] = np.nan
        x[0, 7, 0] = bf16(3.3e38)
        x[0, 8, 0], x[0, 8, 0, 0] = 449.0, 3.3e38
        y[0, 9, 0, 3], y[0, 10, 0] = np.inf, np.nan
        return x, y

    f = Filled([200, 18], 2, 16, True, seed=1, make=make)
    _check_pools(f)
    k, v = f.cache.read(f.seqs, 200)
    for side, got in enumerate((k.double().cpu().numpy(), v.double().cpu().numpy())):
        for b, n in enumerate(f.lengths):
            for h in range(2):
                assert np.array_equal(got[b, :n, h], _held(f, b, h, side), equal_nan=True)


def test_writing_again_keeps_extremes_that_hold():
    f = Filled([40], 1, 16, True, seed=2)
    before = f.cache.bounds.clone()
    f.seqs.lengths.fill_(38)
    f.cache.append(f.seqs, torch.zeros((1, 4, 1, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((1, 4, 1, 128), dtype=torch.bfloat16, device=DEV))
    now, page = f.cache.bounds, f.table[0, 2]
    assert torch.equal(now[page, 0, 0], before[page, 0, 0].clamp(max=0)) and torch.equal(now[page, 0, 1], before[page, 0, 1].clamp(min=0))
    rest = [p for p in range(now.shape[0]) if p != page]
    assert torch.equal(now[rest].nan_to_num(9.0), before[rest].nan_to_num(9.0))


# ------------------------------------------------------------------ attention
@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (2, 1), (15, 3), (14, 2), (8, 1), (9, 1), (32, 2)])
@pytest.mark.parametrize("f32", [False, True])
def test_attention_of_groups(e4m3, hq, hkv, f32):
    f = Filled([1, 0, 16, 31, 33, 250], hkv, 16, e4m3, seed=hq)
    q = f.queries(hq)
    out, lse = f.cache.attend(f.seqs, device(q), f32=f32, lse=True)
    check_attention(f, q, out, lse)
    assert f.cache.status() == 0


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("ps,layout", [(16, "slots_first"), (32, "plain"), (64, "layers"), (128, "slots_first"), (256, "plain")])
@pytest.mark.parametrize("lengths", [[127, 128, 129], [700, 1, 2049, 63], [5000]])
def test_attention_over_lengths(e4m3, ps, layout, lengths):
    f = Filled(lengths, 2, ps, e4m3, layout, seed=ps)
    q = f.queries(10)
    out, lse = f.cache.attend(f.seqs, device(q), lse=True)
    check_attention(f, q, out, lse)
    again, none = f.cache.attend(f.seqs, device(q))
    assert none is None and torch.equal(out, again), "the same call, the same bits"


@pytest.mark.parametrize("batch,length,hkv", [(1, 40000, 1), (300, 130, 2), (3, 9000, 8), (64, 3000, 1), (65, 3000, 1), (130, 2100, 2), (300, 900, 1)])
def test_attention_in_few_and_many_pieces(batch, length, hkv):
    """From one unit cut into pieces for the whole chip to more units than workgroups run at once."""
    rng = np.random.default_rng(batch)
    lengths = [length] + [int(x) for x in rng.integers(0, length + 1, batch - 1)]
    f = Filled(lengths, hkv, 64, True, seed=length)
    q = f.queries(4 * hkv)
    out, lse = f.cache.attend(f.seqs, device(q), lse=True, f32=True)
    few = [b for b in range(batch) if b < 2 or b % 37 == 0]
    f.lengths, f.k, f.v = [f.lengths[b] for b in few], [f.k[b] for b in few], [f.v[b] for b in few]
    check_attention(f, q[few], out[few], lse[few])


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("hq,f32", [(16, True), (11, False), (1, True)])
def test_long_attention_of_other_groups(e4m3, hq, f32):
    f = Filled([3333, 1, 6000], 1, 32, e4m3, seed=hq)
    q = f.queries(hq)
    out, lse = f.cache.attend(f.seqs, device(q), lse=True, f32=f32)
    check_attention(f, q, out, lse)


@pytest.mark.parametrize("e4m3", [True, False])
def test_attention_of_peaked_and_large_logits(e4m3):
    """A few keys far above the rest, in any place, queries that make logits of hundreds; a large softmax scale."""
    f = Filled([300, 77], 2, 16, e4m3, seed=9, spread=3.0)
    q = f.queries(8, spread=3.0)
    for scale in (1.0, 0.001):
        out, lse = f.cache.attend(f.seqs, device(q), scale=scale, lse=True, f32=True)
        check_attention(f, q, out, lse, scale=scale)


def test_scales_of_keys_and_values_across_their_range():
    """Rows of very different magnitudes beside one another; values' own powers of two weigh in."""
    def make(rng, shape):
        return (bf16(rng.standard_normal(shape) * np.exp2(rng.integers(-20, 4, shape[:-1])[..., None].astype(float))),
                bf16(rng.standard_normal(shape) * np.exp2(rng.integers(-60, 60, shape[:-1])[..., None].astype(float))))

    f = Filled([130, 64, 7], 1, 32, True, seed=4, make=make)
    q = f.queries(5)
    out, lse = f.cache.attend(f.seqs, device(q), lse=True, f32=True)
    check_attention(f, q, out, lse)


@pytest.mark.parametrize("ps", [16, 64])
@pytest.mark.parametrize("nonsense", [float("nan"), float("inf"), 3.0e38])
def test_what_lies_behind_a_sequence_does_not_matter(ps, nonsense):
    """The pools hold NaN codes and scales of 255 where nothing was written (tests.paged.pools); in bf16 also infinities and huge numbers."""
    for e4m3 in (True, False):
        f = Filled([1, 15, 17, 100], 1, ps, e4m3, seed=3)
        if not e4m3:
            valid = torch.zeros(f.cache.k.shape[:3], dtype=torch.bool)
            for b, n in enumerate(f.lengths):
                for i in range(n):
                    valid[f.table[b, i // ps], :, i % ps] = True
            for x in (f.cache.k, f.cache.v):
                x[~valid.to(DEV)] = nonsense
        q = f.queries(4)
        out, lse = f.cache.attend(f.seqs, device(q), lse=True, f32=True)
        check_attention(f, q, out, lse)


def test_keys_of_minus_infinity_weigh_nothing():
    f = Filled([40, 3], 1, 16, False, seed=6)
    rows = [torch.from_numpy(x).clone() for x in f.rows]
    rows[0][0, 5], rows[0][1] = -float("inf"), -float("inf")
    f.cache.append(f.seqs, *(x.to(DEV).bfloat16() for x in rows))
    q = np.abs(f.queries(2)) + 0.01
    f.k[0][0][5], f.k[1][0][:] = -np.inf, -np.inf
    out, lse = f.cache.attend(f.seqs, device(q), lse=True)
    check_attention(f, bf16(q), out, lse)
    assert (out[1] == 0).all() and (lse[1] == -float("inf")).all()


def test_queries_and_pages_of_other_strides():
    f = Filled([90, 200], 2, 32, True, seed=8)
    q = f.queries(6)
    fused = torch.zeros((2, 17, 128), dtype=torch.bfloat16, device=DEV)
    fused[:, 3:15:2] = device(q)
    out, _ = f.cache.attend(f.seqs, fused[:, 3:15:2])
    want, _ = f.cache.attend(f.seqs, device(q))
    assert torch.equal(out, want)
    wide = torch.full((2, 40), -9, dtype=torch.int32, device=DEV)
    wide[:, :f.seqs.columns] = f.seqs.table
    s = f.cache.sequences(wide[:, :f.seqs.columns], f.seqs.lengths, 200)
    assert torch.equal(f.cache.attend(s, device(q))[0], want)
    shared = f.cache.sequences(torch.stack([f.seqs.table[1]] * 3), torch.tensor([200, 64, 10], dtype=torch.int32, device=DEV))      # three sequences, one prefix
    g = Filled([200, 64, 10], 2, 32, True, seed=8)
    g.k, g.v = ([[side[1][h][:n] for h in range(2)] for n in (200, 64, 10)] for side in (f.k, f.v))
    q3 = g.queries(6)
    check_attention(g, q3, f.cache.attend(shared, device(q3))[0])


# ------------------------------------------------------------------ pages picked
@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("ps", [16, 32, 256])
def test_attention_over_listed_pages(e4m3, ps):
    """Any order, holes, a page twice, the partial last page in the middle, lists of nothing."""
    f = Filled([ps * 9 + 5, 3, 0, ps * 4], 2, ps, e4m3, seed=ps)
    lists = np.array([[[9, 0, -1, 4, 4, 7, -1], [2, -1, -1, -1, -1, -1, -1]],
                      [[-1, -1, -1, -1, -1, -1, 0], [0, 0, 0, -1, 0, -1, -1]],
                      [[-1] * 7, [-1] * 7],
                      [[-1] * 7, [3, 1, 2, 0, -1, -1, -1]]], np.int32)
    q = f.queries(6)
    for f32 in (False, True):
        out, lse = f.cache.attend(f.seqs, device(q), pages=torch.from_numpy(lists).to(DEV), lse=True, f32=f32)
        check_attention(f, q, out, lse, picked=lists)
    assert f.cache.status() == 0


def test_all_pages_listed_are_all_entries():
    f = Filled([3000, 1700], 2, 16, True, seed=12)
    q = f.queries(8)
    lists = np.full((2, 2, 200), -1, np.int32)
    for b, n in enumerate(f.lengths):
        held = -(-n // 16)
        lists[b, :, :held] = np.arange(held)
    out, lse = f.cache.attend(f.seqs, device(q), pages=torch.from_numpy(lists).to(DEV), lse=True, f32=True)
    check_attention(f, q, out, lse)


@pytest.mark.parametrize("hq,hkv,lengths,ps,keep", [
    (8, 2, [1000, 17, 0, 333], 16, 7), (5, 1, [4096, 4095, 4097], 16, 16), (16, 1, [5000], 32, 100), (7, 7, [900, 2000], 64, 3), (8, 1, [16 * 1025, 16 * 1024], 16, 40),
    (4, 1, [16 * 4099], 16, 500), (2, 1, [16 * 8193], 16, 1000), (40, 8, [8192], 256, 12)])
@pytest.mark.parametrize("first,last", [(1, 1), (0, 0), (2, 0)])
def test_pages_are_picked_by_score(hq, hkv, lengths, ps, keep, first, last):
    f = Filled(lengths, hkv, ps, True, seed=keep, spread=1.0)
    q = f.queries(hq)
    got = f.cache.select(f.seqs, device(q), keep, first=first, last=last).cpu().numpy()
    bounds, g = f.cache.bounds.double().cpu().numpy(), hq // hkv
    for b, n in enumerate(lengths):
        held = -(-n // ps)
        for h in range(hkv):
            s = ref.scores(q[b, h * g:(h + 1) * g], *(bounds[f.table[b, :held], h, i] for i in (0, 1)))
            assert got[b, h].tolist() == ref.pick(s, keep, first, last).tolist(), f"sequence {b} head {h}"
    assert f.cache.status() == 0


@pytest.mark.parametrize("batch,hkv,columns", [(3, 2, 320), (3, 2, 321), (40, 8, 512), (40, 8, 513), (40, 8, 320), (2, 1, 1024), (2, 1, 1025), (1, 2, 4097), (1, 1, 8193), (1, 1, 32768), (64, 16, 513)])
def test_picking_where_it_changes_its_way(batch, hkv, columns):
    """Sequences of up to so many pages, all of one small pool in their own order, which bounds alone decide."""
    g = torch.Generator(device=DEV)
    g.manual_seed(columns)
    pages, ps, heads = 700, 16, 2 * hkv
    cache = pools(pages, hkv, ps, True)
    lo, hi = (torch.randn((pages, hkv, 128), generator=g, device=DEV).bfloat16() for _ in range(2))
    cache.bounds[:, :, 0], cache.bounds[:, :, 1] = torch.minimum(lo, hi), torch.maximum(lo, hi)
    table = torch.randint(0, pages, (batch, columns), generator=g, device=DEV).int()
    rng = np.random.default_rng(columns)
    lengths = [columns * ps - 3] + [int(x) for x in rng.integers(1, columns * ps + 1, batch - 1)]
    q = torch.randn((batch, heads, 128), generator=g, device=DEV).bfloat16()
    keep = 29
    got = cache.select(cache.sequences(table, torch.tensor(lengths, dtype=torch.int32, device=DEV)), q, keep).cpu().numpy()
    bounds, t, qd = cache.bounds.double().cpu().numpy(), table.cpu().numpy(), q.double().cpu().numpy()
    for b in range(min(batch, 12)):
        held = -(-lengths[b] // ps)
        for h in range(hkv):
            each = ref.scores(qd[b, 2 * h:2 * h + 2], bounds[:, h, 0], bounds[:, h, 1])        # of the pool's pages; a sequence has some of them again and again: ties
            assert got[b, h].tolist() == ref.pick(each[t[b, :held]], keep, 1, 1).tolist(), f"sequence {b} head {h}"
    assert cache.status() == 0


def test_pages_of_equal_and_of_no_score():
    """Ties go to the lowest page, what is no number comes first, infinities where they belong."""
    f = Filled([16 * 40], 1, 16, False, seed=1)
    lo, hi = (np.zeros((40, 128)) for _ in range(2))
    hi[:, 0] = [3, 1, 2, 2, 2, 1, 1, 9, 2, 2] * 4
    for special in ({}, {5: np.nan, 33: np.inf, 12: -np.inf}):
        for page, x in special.items():
            hi[page, 0] = x
            lo[page, 0] = min(x, 0) if x == x else x
        b = f.cache.bounds
        b.zero_()
        b[torch.from_numpy(f.table[0]).long().to(DEV), 0, 0] = device(lo)
        b[torch.from_numpy(f.table[0]).long().to(DEV), 0, 1] = device(hi)
        q = np.zeros((1, 2, 128))
        q[..., 0] = 1.0
        s = np.asarray([np.nan if np.isnan(x) else 2 * x for x in np.maximum(lo[:, 0], hi[:, 0])], np.float32)
        for keep in (2, 3, 7, 12, 25, 39, 40, 41):
            for first, last in ((1, 1), (0, 0), (0, 2)):
                got = f.cache.select(f.seqs, device(q), keep, first=first, last=last).cpu().numpy()[0, 0]
                assert got.tolist() == ref.pick(s, keep, first, last).tolist(), (special, keep, first, last)
    got = f.cache.select(f.seqs, device(np.zeros((1, 2, 128))), 6).cpu().numpy()[0, 0]
    assert got.tolist()[-1] == 39 and got.tolist()[0] == 0


# ------------------------------------------------------------------ what the host cannot check
def test_wrong_tables_lengths_and_lists_are_reported_and_left_out():
    """The indexes are checked on the CPU in test_paged_cpu.py: none of these reaches memory."""
    f = Filled([100, 50, 64], 1, 16, True, seed=7)
    q = f.queries(4)
    good = f.seqs.table.clone()
    # a page that is not in the pool: its entries are left out
    f.seqs.table[0, 2], f.seqs.table[2, 1] = 10 ** 9, -1
    keep = [[np.r_[0:32, 48:100]], None, [np.r_[0:16, 32:64]]]
    out, lse = f.cache.attend(f.seqs, device(q), lse=True)
    g = Filled([100, 50, 64], 1, 16, True, seed=7)
    for b in (0, 2):
        g.k[b][0], g.v[b][0] = f.k[b][0][keep[b][0]], f.v[b][0][keep[b][0]]
    check_attention(g, q, out, lse)
    assert f.cache.status() == ckv.BAD_PAGE and f.cache.status() == 0
    raw = f.cache.k.view(torch.uint8).clone()
    f.cache.append(f.seqs, *(torch.zeros((3, 100, 1, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)), first=torch.tensor([32, 50, 16], dtype=torch.int32, device=DEV))
    assert f.cache.status() == ckv.BAD_PAGE
    same = (f.cache.k.view(torch.uint8) == raw).all(-1)[:, 0].cpu().numpy()
    changed = {(p, s) for p, s in zip(*np.nonzero(~same))}
    want = {(f.table[0, i // 16], i % 16) for i in range(48, 100)} | {(f.table[2, i // 16], i % 16) for i in range(32, 64)}
    assert changed <= want
    rows = tuple(torch.full((3, 100, 1, 128), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    f.cache.read(f.seqs, 100, out=rows)
    assert f.cache.status() == ckv.BAD_PAGE and (rows[0][0, 32:48] == 3.0).all()
    picked = f.cache.select(f.seqs, device(q), 3).cpu().numpy()
    assert f.cache.status() == ckv.BAD_PAGE and picked[1, 0].tolist()[0] == 0
    # lengths beyond what the call was told, and below nothing
    f.seqs.table.copy_(good)
    h = Filled([100, 50, 64], 1, 16, True, seed=7)
    h.seqs.lengths.copy_(torch.tensor([10 ** 9, -5, 64], dtype=torch.int32, device=DEV))
    out, lse = h.cache.attend(h.cache.sequences(h.seqs.table, h.seqs.lengths, 96), device(q), lse=True)
    assert h.cache.status() == ckv.BAD_LENGTH
    h.lengths, h.k[0], h.v[0], h.k[1], h.v[1] = [96, 0, 64], [h.k[0][0][:96]], [h.v[0][0][:96]], [h.k[1][0][:0]], [h.v[1][0][:0]]
    check_attention(h, q, out, lse)
    # lists of pages that the sequence does not have
    lists = torch.tensor([[[0, 7, -2]], [[3, 4, 10 ** 9]], [[-(2 ** 31), 2 ** 31 - 1, 1]]], dtype=torch.int32, device=DEV)
    h = Filled([100, 50, 64], 1, 16, True, seed=7)
    out, lse = h.cache.attend(h.seqs, device(q), pages=lists, lse=True)
    assert h.cache.status() == ckv.BAD_PICK
    check_attention(h, q, out, lse, picked=[[[0]], [[3]], [[1]]])
    # rows that do not fit their sequence, packed rows beyond the buffer
    for more in (dict(first=torch.tensor([101, 0, -1], dtype=torch.int32, device=DEV)),):
        raw = h.cache.k.view(torch.uint8).clone()
        h.seqs.lengths.copy_(torch.tensor([100, 0, 64], dtype=torch.int32, device=DEV))
        h.cache.append(h.seqs, *(torch.zeros((3, 5, 1, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)), **more)
        assert h.cache.status() == ckv.BAD_LENGTH and torch.equal(raw, h.cache.k.view(torch.uint8))
    raw = h.cache.k.view(torch.uint8).clone()
    h.cache.append(h.seqs, *(torch.zeros((5, 1, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)), rows=5, starts=torch.tensor([0, 6, 6, 4], dtype=torch.int32, device=DEV))
    assert h.cache.status() == ckv.BAD_LENGTH and torch.equal(raw, h.cache.k.view(torch.uint8))


def test_calls_with_nothing_to_do():
    f = Filled([20, 0], 2, 16, True)
    none, starts = torch.zeros((0, 2, 128), dtype=torch.bfloat16, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    before = f.cache.k.view(torch.uint8).clone()
    f.cache.append(f.seqs, none, none, rows=4, starts=starts)
    k, v = f.cache.read(f.seqs, 4, starts=starts, total=0)
    assert k.shape == v.shape == none.shape and torch.equal(before, f.cache.k.view(torch.uint8))
    s = f.cache.sequences(f.seqs.table, torch.zeros_like(f.seqs.lengths), 0)
    q = device(f.queries(4))
    out, lse = f.cache.attend(s, q, lse=True)
    assert (out == 0).all() and (lse == -float("inf")).all()
    assert (f.cache.select(s, q, 3) == -1).all()
    f.cache.append(s, torch.zeros((2, 2, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((2, 2, 128), dtype=torch.bfloat16, device=DEV))
    assert f.cache.status() == 0 and torch.equal(before, f.cache.k.view(torch.uint8))


def test_refusals_of_the_binding():
    f = Filled([20], 2, 16, True)
    q = device(f.queries(4))
    one = torch.zeros((1, 2, 128), dtype=torch.bfloat16, device=DEV)
    for bad in (lambda: f.cache.attend(f.seqs, q.float()), lambda: f.cache.attend(f.seqs, q[:, :3]), lambda: f.cache.attend(f.seqs, q[..., :64]), lambda: f.cache.attend(f.seqs, q.cpu()),
                lambda: f.cache.attend(f.seqs, q, out=torch.empty_like(q, dtype=torch.float32)), lambda: f.cache.attend(f.seqs, q, scale=-1.0), lambda: f.cache.attend(f.seqs, q.repeat(2, 1, 1)),
                lambda: f.cache.attend(f.seqs, q, pages=torch.zeros((1, 1, 2), dtype=torch.int32, device=DEV)), lambda: f.cache.attend(f.seqs, q, pages=torch.zeros((1, 2, 2), device=DEV)),
                lambda: f.cache.attend(f.seqs, q, pages=torch.zeros((1, 2, 0), dtype=torch.int32, device=DEV)),
                lambda: f.cache.select(f.seqs, q, 0), lambda: f.cache.select(f.seqs, q, 1), lambda: f.cache.select(f.seqs, q, 4, out=torch.zeros((1, 2, 3), dtype=torch.int32, device=DEV)),
                lambda: f.cache.append(f.seqs, one, one.float()), lambda: f.cache.append(f.seqs, one[:, :1], one[:, :1]), lambda: f.cache.append(f.seqs, one, one, rows=2),
                lambda: f.cache.append(f.seqs, one, one, starts=torch.zeros(2, dtype=torch.int32, device=DEV)), lambda: f.cache.append(f.seqs, one, one, first=torch.zeros(1, device=DEV)),
                lambda: f.cache.append(f.seqs, one.cpu(), one.cpu()), lambda: f.cache.read(f.seqs, 0), lambda: f.cache.read(f.seqs, 3, starts=torch.zeros(2, dtype=torch.int32, device=DEV)),
                lambda: f.cache.sequences(f.seqs.table.long(), f.seqs.lengths), lambda: f.cache.sequences(f.seqs.table, f.seqs.lengths.repeat(2)), lambda: f.cache.sequences(f.seqs.table.cpu(), f.seqs.lengths.cpu()),
                lambda: f.cache.sequences(f.seqs.table, f.seqs.lengths, 33), lambda: f.cache.sequences(f.seqs.table[:, :0], f.seqs.lengths), lambda: f.cache.sequences(f.seqs.table, f.seqs.lengths, -1)):
        with pytest.raises(ckv.CkvError):
            bad()
    plain = ckv.PagedCache(f.cache.k, f.cache.v, scales=f.cache.scales)
    with pytest.raises(ckv.CkvError):
        plain.select(plain.sequences(f.seqs.table, f.seqs.lengths), q, 2)
    plain.append(plain.sequences(f.seqs.table, f.seqs.lengths), one, one)                  # no bounds to keep


# ------------------------------------------------------------------ offsets, streams, graphs
def test_pools_beyond_four_gigabytes():
    """Pages at the far end of pools of 4.5 GiB each."""
    hkv, ps, n = 8, 256, 18432 // 2
    big = ckv.PagedCache.empty(n, ps, hkv, dtype=ckv.BF16, bounds=True)
    f = Filled([600], hkv, ps, False, seed=2)
    table = torch.tensor([[n - 1, 3, n - 2]], dtype=torch.int32, device=DEV)
    s = big.sequences(table, f.seqs.lengths)
    big.append(s, *(device(x) for x in f.rows))
    q = f.queries(16)
    out, lse = big.attend(s, device(q), lse=True)
    check_attention(f, q, out, lse)
    want = f.cache.select(f.seqs, device(q), 2)
    assert torch.equal(big.select(s, device(q), 2), want)
    assert all(torch.equal(a, b) for a, b in zip(big.read(s, 600), f.cache.read(f.seqs, 600)))


def test_calls_on_two_streams_at_once():
    """Each call's workspace is its own."""
    f = Filled([9000, 4000], 2, 64, True, seed=21)
    qs = [device(f.queries(8)) for _ in range(4)]
    want = [f.cache.attend(f.seqs, q)[0] for q in qs]
    picks = [f.cache.select(f.seqs, q, 20) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None] * 4
    for _ in range(5):
        for i, q in enumerate(qs):
            with torch.cuda.stream(streams[i % 2]):
                got[i] = (f.cache.attend(f.seqs, q)[0], f.cache.select(f.seqs, q, 20))
        torch.cuda.synchronize()
        for i in range(4):
            assert torch.equal(got[i][0], want[i]) and torch.equal(got[i][1], picks[i])


@pytest.mark.parametrize("e4m3", [True, False])
def test_steps_captured_and_replayed(e4m3):
    """Tokens enter, all entries are read, pages are picked and read: one graph, replayed while lengths and inputs change, beside another graph of the same
    cache and eager calls between the replays."""
    f, g = (Filled([200, 63, 0], 2, 16, e4m3, seed=31, columns=40) for _ in range(2))
    for x in (f, g):                         # every sequence's next pages
        free = [p for p in range(x.cache.n_pages) if p not in set(x.table[x.table >= 0].tolist())]
        assert len(free) == 3
        x.seqs.table[0, 13], x.seqs.table[1, 4], x.seqs.table[2, 0] = free
    rng = np.random.default_rng(0)
    k, v = (torch.zeros((3, 2, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    q = torch.zeros((3, 8, 128), dtype=torch.bfloat16, device=DEV)

    def step(x):
        x.cache.append(x.seqs, k, v)
        a, lse = x.cache.attend(x.seqs, q, lse=True)
        picked = x.cache.select(x.seqs, q, 5)
        b, _ = x.cache.attend(x.seqs, q, pages=picked)
        rows = x.cache.read(x.seqs, 4)
        return a, lse, picked, b, *rows

    for x in (f, g):
        x.seqs.lengths.add_(1)
    for to in (k, v, q):
        to.copy_(torch.from_numpy(rng.standard_normal(tuple(to.shape))))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(f)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = step(f)
        graphs.append((graph, got))
    for n in range(7):
        if n:
            for x in (f, g):
                x.seqs.lengths.add_(1)
            for to in (k, v, q):
                to.copy_(torch.from_numpy(rng.standard_normal(tuple(to.shape))))
        graph, got = graphs[n % 2]
        graph.replay()
        want = step(g)
        torch.cuda.synchronize()
        live = [x.clone() for x in got[:4]], [x[:2].clone() for x in got[4:]]
        for i, (a, b) in enumerate(zip(live[0], want[:4])):
            assert torch.equal(a, b), f"replay {n} output {i}"
        for a, b in zip(live[1], want[4:]):
            assert torch.equal(a, b[:2])
        assert torch.equal(f.cache.bounds.nan_to_num(7.0), g.cache.bounds.nan_to_num(7.0))
    assert f.cache.status() == 0 and g.cache.status() == 0


# ------------------------------------------------------------------ together, and beside the budgeted caches
def test_a_paged_prompt_beside_and_into_a_budgeted_cache():
    """A prompt in bf16 pages, attended by the paged call and by an attention-only step of a context loaded from the rows that the pages give back: the
    same entries, the same outputs within the two kernels' bounds.  Then the 8-bit cache, over all entries and over the pages picked."""
    bz, hq, hkv, n = 2, 10, 2, 500
    f = Filled([n, n], hkv, 64, False, seed=40)
    rng = np.random.default_rng(41)
    q = bf16(rng.standard_normal((bz, hq, 128)))
    rows = [x.transpose(1, 2).contiguous() for x in f.cache.read(f.seqs, n)]
    g = ckv.CrystalKV(1, bz, hq, hkv, 128, 512, np.full((1, bz, hkv), 505), t0=n - 1, budget_max=511)
    g.load_prompt(0, *(x[:, :, :n - 1].contiguous() for x in rows))
    step = g.decode_step(device(q)[None], rows[0][None, :, :, n - 1].contiguous(), rows[1][None, :, :, n - 1].contiguous(), attention_only=True, evict=False)[0]
    out, _ = f.cache.attend(f.seqs, device(q), f32=True)
    check_attention(f, q, out)
    assert (out - step).abs().max() <= 2 * 2e-3 * step.abs().max()
    e = Filled([n, n], hkv, 64, True, seed=40)
    picked = e.cache.select(e.seqs, device(q), 4)
    out, _ = e.cache.attend(e.seqs, device(q), pages=picked)
    check_attention(e, q, out, picked=picked.cpu().numpy())
    g8 = ckv.CrystalKV(1, bz, hq, hkv, 128, 512, np.full((1, bz, hkv), 256), t0=n, budget_max=511)
    g8.load_prompt(0, *(x.transpose(1, 2).contiguous() for x in e.cache.read(e.seqs, n)))
    g8.evict()
    assert g8.status() == 0 and (g8.lengths() == 256).all()


def test_rows_of_many_sequences_and_of_many_small_pages():
    """Enough pages that a wavefront takes one each: single rows of 600 sequences, and a long prompt in pages of 16."""
    for lengths, ps, rows in (([1 + i % 60 for i in range(600)], 32, 1), ([9000, 8000], 16, 9000)):
        f = Filled(lengths, 4, ps, True, seed=rows)
        _check_pools(f)
        if rows == 1:
            g = Filled(lengths, 4, ps, True, seed=rows)
            k, v = (torch.from_numpy(np.stack([x[b, n - 1] for b, n in enumerate(lengths)])).to(DEV).bfloat16() for x in f.rows)
            for x in (g.cache.k, g.cache.v):
                for b, n in enumerate(lengths):
                    x.view(torch.uint8)[g.table[b, (n - 1) // ps], :, (n - 1) % ps] = 0
            g.cache.append(g.seqs, k, v)
            _check_pools(g)
