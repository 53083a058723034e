"""Rotated appends and attention of several rows as a decoder with drafted tokens has them one after another: prompts, drafts in a tree, those that are accepted moved up, single tokens through a window."""
import numpy as np
import pytest
import torch

from oracle import paged as ref
from paper_2601_16986_amd import ckv
from tests.paged import DEV, bf16, device, pools
from tests.rows import check_rows, random_tree

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.as_tensor(np.asarray(x, np.int32)).to(DEV)


class Held:
    """What the cache holds, as check_rows takes it."""

    def __init__(self, cache, seqs, lengths, hkv):
        self.lengths, self.hkv = list(lengths), hkv
        k, v = (x.double().cpu().numpy() for x in cache.read(seqs, max(lengths), first=torch.zeros_like(seqs.lengths)))
        self.k, self.v = ([[x[b, :n, h] for h in range(hkv)] for b, n in enumerate(lengths)] for x in (k, v))


@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("hq,hkv,drafts,window,sinks", [(8, 2, 7, 0, 0), (4, 4, 20, 64, 3), (15, 3, 40, 100, 20)])
def test_drafts_are_verified_and_accepted(e4m3, hq, hkv, drafts, window, sinks):
    rng = np.random.default_rng(drafts)
    ps, columns, lengths = 16, 40, [0, 0, 0, 0]
    batch, how = len(lengths), dict(window=window, sinks=sinks)
    c = pools(batch * columns, hkv, ps, e4m3)
    table = ints(rng.permutation(batch * columns).reshape(batch, columns))
    s = c.sequences(table, ints(lengths))
    f = 10000.0 ** (-np.arange(48) / 48)
    r = ckv.Rotation(torch.from_numpy(f).to(DEV))

    def rows(*shape):
        return [bf16(rng.standard_normal((*shape, h, 128))) for h in (hq, hkv, hkv)]

    def entered(held, k, v, positions, b, at, n):
        """Rows as they are in the cache are the definition's, turned and rounded."""
        want = ref.rotate(k, positions, f)
        got = np.stack([held.k[b][h][at:at + n] for h in range(hkv)], 1)
        # half a step of the code's 4 bits below the row's largest, or of bf16; and what a rotation in 32 bits is off by
        tol = np.abs(want).max(-1, keepdims=True) * (2.0 ** -4 if e4m3 else 2.0 ** -8) * (1 + 2.0 ** -8) + 2.0 ** -20 * ref.pair_size(k, 48)
        assert (np.abs(got - want) <= tol).all()
        gv = np.stack([held.v[b][h][at:at + n] for h in range(hkv)], 1)
        assert (np.abs(gv - v) <= (np.abs(v).max(-1, keepdims=True) * 2.0 ** -4 * (1 + 2.0 ** -8) if e4m3 else 0)).all()

    # prompts, packed, one sequence without
    counts = [90, 1, 0, 33]
    q, k, v = rows(sum(counts))
    starts = ints(np.cumsum([0] + counts))
    lengths = list(counts)
    s.lengths.copy_(ints(lengths))
    turned = c.append_rotated(s, device(q), device(k), device(v), r, rows=90, starts=starts)
    out, lse = c.attend_rows(s, turned, rows=90, starts=starts, lse=True, f32=True, **how)
    held = Held(c, s, lengths, hkv)
    tq, to, tl = np.zeros((batch, 90, hq, 128)), torch.zeros((batch, 90, hq, 128), device=DEV), torch.zeros((batch, 90, hq), device=DEV)
    for b, n in enumerate(counts):
        at = sum(counts[:b])
        tq[b, :n], to[b, :n], tl[b, :n] = turned[at:at + n].double().cpu().numpy(), out[at:at + n], lse[at:at + n]
        entered(held, k[at:at + n], v[at:at + n], np.arange(n), b, 0, n)
    check_rows(held, tq, to, counts, lse=tl, what="prompts", **how)

    for step in range(5):
        # a tree of drafts behind each sequence
        base = list(lengths)
        trees = np.stack([random_tree(rng, drafts) for _ in range(batch)])
        positions = np.array(base)[:, None] + trees.sum(2) - 1
        q, k, v = rows(batch, drafts)
        lengths = [n + drafts for n in base]
        s.lengths.copy_(ints(lengths))
        x = device(q)
        turned = c.append_rotated(s, x, device(k), device(v), r, positions=ints(positions), out=x)
        assert turned is x
        out, lse = c.attend_rows(s, turned, tree=torch.from_numpy(trees).to(DEV), lse=True, **how)
        held = Held(c, s, lengths, hkv)
        check_rows(held, turned.double().cpu().numpy(), out, [drafts] * batch, trees=trees, lse=lse, what=f"step {step}", **how)
        for b in range(batch):
            entered(held, k[b], v[b], positions[b], b, base[b], drafts)
        # one draft and those it follows are accepted: their rows, as they are, move up
        taken = [np.flatnonzero(trees[b, rng.integers(drafts)]) for b in range(batch)]
        most = max(map(len, taken))
        rk, rv = c.read(s, drafts, first=ints(base))
        order = ints([list(t) + [0] * (most - len(t)) for t in taken]).long()
        pick = [torch.gather(y, 1, order[:, :, None, None].expand(-1, -1, hkv, 128)).contiguous() for y in (rk, rv)]
        lengths = [n + len(t) for n, t in zip(base, taken)]
        s.lengths.copy_(ints(lengths))
        c.append(s, *pick, first=ints(base))
        after = Held(c, s, lengths, hkv)
        for b in range(batch):
            for h in range(hkv):
                for a, z in ((after.k, held.k), (after.v, held.v)):
                    assert np.array_equal(a[b][h][:base[b]], z[b][h][:base[b]]) and np.array_equal(a[b][h][base[b]:], z[b][h][base[b] + taken[b]])
        # the token that comes of it
        q, k, v = rows(batch)
        lengths = [n + 1 for n in lengths]
        s.lengths.copy_(ints(lengths))
        turned = c.append_rotated(s, device(q), device(k), device(v), r)
        out, lse = c.attend_rows(s, turned, lse=True, **how)
        held = Held(c, s, lengths, hkv)
        check_rows(held, turned.double().cpu().numpy()[:, None], out[:, None], [1] * batch, lse=lse[:, None], what=f"token {step}", **how)
    assert c.status() == 0


def test_a_step_on_a_stream_of_its_own():
    """Rows written on one stream are what another sees once it waits for them, workspaces included: calls of one step on a side stream, beside others on the default one."""
    rng = np.random.default_rng(5)
    c = pools(80, 2, 16, True)
    r = ckv.Rotation(torch.from_numpy(10000.0 ** (-np.arange(64) / 64)).to(DEV))
    s = [c.sequences(ints(np.arange(40 * i, 40 * i + 40)[None]), ints([600])) for i in range(2)]
    q, k, v = (device(bf16(rng.standard_normal((1, 600, h, 128)))) for h in (8, 2, 2))
    tree = torch.from_numpy(random_tree(rng, 30)).to(DEV)

    def step(x):
        turned = c.append_rotated(x, q, k, v, r)
        return c.attend_rows(x, turned, window=100, sinks=4)[0], c.attend_rows(x, turned[:, -30:], tree=tree)[0], c.attend_rows(x, turned[:, -1], window=30)[0]

    want = step(s[0])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(5):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            a = step(s[1])
        b = step(s[0])
        torch.cuda.synchronize()
        for x, y, z in zip(a, b, want):
            assert torch.equal(x, z) and torch.equal(y, z)
