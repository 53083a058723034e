"""Operators of a paged key-value cache for models that rotate positions, look back through a window, or verify drafted tokens, as cases to time.

A case is a dict of plain values; `prepare` builds what a serving program has in hand before the call (page pools in the middle of their life, a table,
lengths, the projections' rows), `run` makes one pass, `exact` says what its floating-point outputs are in 64 bits.  Kinds of case:

  rotate   queries and keys are rotated by their positions, keys and values enter the cache, and the rows are read back
  window   attention of the last rows of each sequence, each over itself, the entries of a window before it and a few first ones (sinks)
  tree     attention of drafted tokens, the last rows of each sequence, over all entries before them (or a window's) and their own ancestors

A row is 128 values.  In 8 bits it is 128 e4m3 codes and a power of two: with E the smallest integer for which the row's largest finite magnitude is at
most 448 * 2^E (from -100 to 120), a code is x / 2^E rounded to e4m3, and the scale byte E + 127.  Pools: k, v [pages][KV heads][slots][128],
scales uint8 [pages][KV heads][slots][2] (key, value), bounds bf16 [pages][KV heads][2][128] (least and largest key of each channel).

Rotation: of the first `rotary` dimensions pair j (j and j + rotary / 2, or 2 j and 2 j + 1 where they are interleaved) turns by position * base^(-2 j / rotary).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
D = 128
SCALE = 1.0 / math.sqrt(D)


def _case(name, kind, batch, hq, hkv, length, page, dtype="e4m3", ragged=True, rows=1, window=0, sinks=0, lse=False, f32=False, rotary=128, base=10000,
          interleaved=False):
    """rows: the last so many rows of each sequence are the call's (0: all); window 0: no limit."""
    return dict(name=name, kind=kind, batch=batch, hq=hq, hkv=hkv, length=length, page=page, dtype=dtype, ragged=ragged, rows=rows, window=window, sinks=sinks,
                lse=lse, f32=f32, rotary=rotary, base=base, interleaved=interleaved)


def listed():
    return [
        # one token of each of 32 sequences enters the cache of one layer: latency is all there is
        _case("rotate_step", "rotate", 32, 32, 8, 2048, 64, base=500000),
        # 64 drafted tokens of each of 4 sequences, far out, positions by their depth in the tree; a model that turns half of its dimensions
        _case("rotate_drafts", "rotate", 4, 28, 4, 131072, 128, dtype="bf16", rows=64, rotary=64, base=1000000, interleaved=True),
        # a batch of 8K-level prompts enters the cache of one 14B layer
        _case("rotate_prompts", "rotate", 8, 40, 8, 9350, 64, rows=0, base=1000000),
        # the smallest call: one token of one short sequence, two KV heads, small pages
        _case("window_tiny", "window", 1, 8, 2, 129, 16, dtype="bf16", window=32, sinks=4),
        # one token of each sequence of a large batch, a layer that looks back 4096 entries
        _case("window_step", "window", 64, 32, 8, 9350, 64, ragged=False, window=4096, sinks=4),
        # the next 512 tokens of 16 prompts that enter chunk by chunk, a 7B layer (G = 7)
        _case("window_chunk", "window", 16, 28, 4, 9350, 64, rows=512, window=2048, sinks=16),
        # whole prompts of a 14B layer at once, in full precision: the largest
        _case("window_prompts", "window", 2, 40, 8, 8192, 64, dtype="bf16", ragged=False, rows=0, window=4096, sinks=4, lse=True),
        # 8 drafted tokens of a few short sequences of a 7B model
        _case("tree_small", "tree", 4, 28, 4, 777, 16, dtype="bf16", rows=8),
        # 64 drafted tokens of each of 32 sequences of many lengths, an 8B layer in 8 bits
        _case("tree_llama8b", "tree", 32, 32, 8, 9350, 64, rows=64),
        # 48 drafted tokens of one sequence of 128K on a 14B layer: the length is all there is to split
        _case("tree_long", "tree", 1, 40, 8, 131072, 256, ragged=False, rows=48, lse=True),
        # 25 drafted tokens of 16 sequences on a layer that looks back 1024 entries, full precision
        _case("tree_window", "tree", 16, 40, 8, 9350, 32, dtype="bf16", rows=25, window=1024, sinks=4, f32=True),
    ]


HEADS = [(8, 2), (28, 4), (40, 8), (32, 8), (16, 16), (12, 4), (64, 8), (4, 1), (16, 1), (5, 5)]


def draw(rng):
    def log_int(lo, hi):
        return int(round(float(lo) * (float(hi) / lo) ** rng.random()))

    kind = rng.choice(["rotate", "rotate", "window", "window", "window", "tree", "tree", "tree"])
    hq, hkv = rng.choice(HEADS)
    batch, length, page = log_int(1, 64), log_int(1, 60000), rng.choice([16, 32, 64, 128, 256])
    rows = log_int(1, 96) if kind == "tree" else rng.choice([0, 1, log_int(1, 64), log_int(1, 2000)])
    limited = kind == "window" or (kind == "tree" and rng.random() < 0.3)
    window = max(log_int(1, 8000), rows if kind == "tree" else 1) if limited else 0
    c = _case("", kind, batch, hq, hkv, length, page, dtype=rng.choice(["e4m3", "bf16"]), ragged=rng.random() < 0.7, rows=rows, window=window,
              sinks=rng.choice([0, 1, 4, 17]) if limited else 0, lse=kind != "rotate" and rng.random() < 0.3, f32=kind != "rotate" and rng.random() < 0.3,
              rotary=rng.choice([128, 128, 64, 32, 112]), base=rng.choice([10000, 500000, 1000000]), interleaved=rng.random() < 0.3)
    del c["name"]

    def costs():
        new = min(length, rows) if rows else length
        if kind == "rotate":
            return batch * max(hkv * length / 4_500_000, new * (hq + 2 * hkv) / 2_200_000)
        return max(batch * hkv * length / 4_500_000, batch * hq * new * length / 1.2e9)

    while costs() > 1:
        if batch > 1:
            batch = (batch + 1) // 2
        else:
            length = length // 2 + 1
    c["batch"], c["length"] = batch, max(length, 1)
    return c


# ------------------------------------------------------------------ inputs
def _lengths(case):
    """Entries per sequence, the call's rows included."""
    n, b = case["length"], case["batch"]
    if not case["ragged"]:
        return [n] * b
    r = np.random.RandomState(17 * b + n % 1009)
    return [n] + [max(1, int(n * 16.0 ** -float(u))) for u in r.random_sample(b - 1)]


def _rows(case):
    """Rows of the call per sequence."""
    return [min(n, case["rows"]) if case["rows"] else n for n in _lengths(case)]


def _tree(rows, turn):
    """Parents of drafted tokens, the best ones first: -1 is the sequence's last accepted token."""
    r = np.random.RandomState((rows + 1000 * turn) % 2 ** 32)
    return [-1 if i == 0 else int(r.randint(max(-1, i // 3 - 4), i)) for i in range(rows)]


def _ancestors(rows, turn):
    """Who sees whom, bool [rows][rows]: a token itself and its ancestors."""
    sees = np.zeros((rows, rows), bool)
    for i, up in enumerate(_tree(rows, turn)):
        if up >= 0:
            sees[i] = sees[up]
        sees[i, i] = True
    return sees


def _quantise(x):
    """Codes and scale bytes of rows."""
    x = x.float()
    mantissa, exponent = torch.frexp(torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1))
    e = torch.where(mantissa > 0, exponent - 9 + (mantissa > 0.875).int(), -100).clamp(-100, 120)
    inverse = ((127 - e) << 23).view(torch.float32)          # 2^-E
    return (x * inverse.unsqueeze(-1)).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _values(codes, scale):
    """What rows stand for, in 32 bits."""
    return codes.float() if scale is None else codes.float() * (scale.int() << 23).view(torch.float32).unsqueeze(-1)


def _pool(case, pages, gen, mean):
    """Pools full of rows: a few heavy keys along the mean query, the others noise."""
    hkv, ps = case["hkv"], case["page"]
    dt = torch.float8_e4m3fn if case["dtype"] == "e4m3" else torch.bfloat16
    k, v = (torch.empty((pages, hkv, ps, D), dtype=dt, device=DEVICE) for _ in range(2))
    scales = torch.empty((pages, hkv, ps, 2), dtype=torch.uint8, device=DEVICE) if case["dtype"] == "e4m3" else None
    step = max(1, (32 << 20) // (hkv * ps * D))
    for a in range(0, pages, step):
        e = min(pages, a + step)
        heavy = (torch.rand((e - a, hkv, ps, 1), generator=gen, device=DEVICE) < 0.01).float()
        for i, (to, x) in enumerate(((k, torch.randn((e - a, hkv, ps, D), generator=gen, device=DEVICE) + 0.75 * heavy * mean),
                                     (v, torch.randn((e - a, hkv, ps, D), generator=gen, device=DEVICE)))):
            if scales is None:
                to[a:e] = x.bfloat16()
            else:
                codes, s = _quantise(x.bfloat16())
                to.view(torch.uint8)[a:e] = codes.view(torch.uint8)
                scales[a:e, :, :, i] = s
    return k, v, scales


def _bounds(case, k, scales, filled):
    """Least and largest keys over the first `filled` rows of every page."""
    hkv, ps, pages = case["hkv"], case["page"], len(k)
    bounds = torch.zeros((pages, hkv, 2, D), dtype=torch.bfloat16, device=DEVICE)
    step = max(1, (32 << 20) // (hkv * ps * D))
    for a in range(0, pages, step):
        e = min(pages, a + step)
        x = _values(k[a:e], None if scales is None else scales[a:e, :, :, 0])
        there = (torch.arange(ps, device=DEVICE) < filled[a:e, None])[:, None, :, None]
        some = (filled[a:e] > 0)[:, None, None]
        bounds[a:e, :, 0] = torch.where(some, torch.where(there, x, math.inf).amin(2), 0.0).bfloat16()
        bounds[a:e, :, 1] = torch.where(some, torch.where(there, x, -math.inf).amax(2), 0.0).bfloat16()
    return bounds


def _frequencies(case):
    return case["base"] ** (-2.0 * torch.arange(case["rotary"] // 2, dtype=torch.float64, device=DEVICE) / case["rotary"])


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    batch, hq, hkv, ps = case["batch"], case["hq"], case["hkv"], case["page"]
    lengths, rows = _lengths(case), _rows(case)
    turn = int(seed) % batch
    lengths, rows = lengths[turn:] + lengths[:turn], rows[turn:] + rows[:turn]
    held = [-(-n // ps) for n in lengths]
    pages, columns = sum(held) + sum(held) // 8 + 4, max(held)
    shuffled = torch.randperm(pages, generator=gen, device=DEVICE)[:sum(held)].int().cpu()
    table, filled = torch.full((batch, columns), -1, dtype=torch.int32), torch.zeros(pages, dtype=torch.int32)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = shuffled[at:at + n]
        filled[table[b, :n].long()] = (lengths[b] - rows[b] - ps * torch.arange(n, dtype=torch.int32)).clamp(0, ps)
        at += n
        if case["window"]:               # pages that nobody will look at again have been given back
            oldest = (lengths[b] - rows[b] - case["window"]) // ps
            table[b, -(-case["sinks"] // ps):max(oldest, 0)] = -1
    mean = torch.randn(D, generator=gen, device=DEVICE)
    mean *= 4.0 / mean.norm()
    k, v, scales = _pool(case, pages, gen, mean)
    starts = [0]
    for n in rows:
        starts.append(starts[-1] + n)
    total = starts[-1]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEVICE)  # noqa: E731
    s = dict(k=k, v=v, scales=scales, bounds=None, table=table.to(DEVICE), lengths=ints(lengths), case=case, total=total, most=max(rows), starts=ints(starts),
             first=ints([n - r for n, r in zip(lengths, rows)]), sees=None, positions=None)
    s["q"] = (torch.randn((total, hq, D), generator=gen, device=DEVICE) + mean).bfloat16()
    if case["kind"] == "rotate":
        s["bounds"] = _bounds(case, k, scales, filled.to(DEVICE))
        s["new_k"], s["new_v"] = (torch.randn((total, hkv, D), generator=gen, device=DEVICE).bfloat16() for _ in range(2))
        s["frequencies"] = _frequencies(case)
        if case["rows"] > 1:             # drafts: positions by depth
            depths = {r: _ancestors(r, int(seed)).sum(1) - 1 for r in set(rows)}
            s["positions"] = ints(np.concatenate([n - r + depths[r] for n, r in zip(lengths, rows)]))
    if case["kind"] == "tree":
        sees = np.zeros((batch, max(rows), max(rows)), bool)
        for b, r in enumerate(rows):
            sees[b, :r, :r] = _ancestors(r, int(seed) + b % 3)
        s["sees"] = torch.from_numpy(sees).to(DEVICE)
    if own:
        from paper_2601_16986_amd import ckv
        s["cache"] = ckv.PagedCache(k, v, scales=scales, bounds=s["bounds"])
        s["seqs"] = s["cache"].sequences(s["table"], s["lengths"], case["length"])
        if case["kind"] == "rotate":
            s["rotation"] = ckv.Rotation(s["frequencies"], interleaved=case["interleaved"])
    return s


# ------------------------------------------------------------------ one pass
def _places(s):
    """Sequence and position of every row of the call."""
    count = s["starts"][1:] - s["starts"][:-1]
    b = torch.repeat_interleave(torch.arange(len(count), device=DEVICE), count, output_size=s["total"])
    return b, s["first"][b] + torch.arange(s["total"], device=DEVICE) - s["starts"][b]


def _turned(x, cos, sin, interleaved):
    """Rows [rows][heads][128] turned, in 32 bits."""
    n = cos.shape[-1]
    x = x.float()
    a, z = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if interleaved else (x[..., :n], x[..., n:2 * n])
    a, z = a * cos - z * sin, z * cos + a * sin
    pairs = torch.stack((a, z), -1).flatten(-2) if interleaved else torch.cat((a, z), -1)
    return torch.cat((pairs, x[..., 2 * n:]), -1)


def _plain_rotate(s):
    case = s["case"]
    b, at = _places(s)
    page, slot = s["table"][b, at // case["page"]].long(), at % case["page"]
    angle = (at if s["positions"] is None else s["positions"]).double()[:, None, None] * s["frequencies"]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    q = _turned(s["q"], cos, sin, case["interleaved"]).bfloat16()
    back = []
    for i, (pool, x) in enumerate(((s["k"], _turned(s["new_k"], cos, sin, case["interleaved"])), (s["v"], s["new_v"]))):
        if s["scales"] is None:
            pool[page, :, slot] = x.bfloat16()
            back.append(pool[page, :, slot])
        else:
            codes, e = _quantise(x)
            pool.view(torch.uint8)[page, :, slot] = codes.view(torch.uint8)
            s["scales"][page, :, slot, i] = e
            back.append(_values(pool.view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn), s["scales"][page, :, slot, i]).bfloat16())
    k, v = back
    bounds = s["bounds"].float()
    begun = torch.zeros(len(bounds), dtype=torch.int32, device=DEVICE).scatter_reduce(0, page, (slot == 0).int(), "amax")[:, None, None] > 0
    rows = page[:, None, None].expand(k.shape)
    s["bounds"][:, :, 0] = torch.where(begun, math.inf, bounds[:, :, 0]).scatter_reduce(0, rows, k.float(), "amin").bfloat16()
    s["bounds"][:, :, 1] = torch.where(begun, -math.inf, bounds[:, :, 1]).scatter_reduce(0, rows, k.float(), "amax").bfloat16()
    return {"q": q, "k": k, "v": v, "bounds": s["bounds"]}


def _plain_attend(s):
    case, table = s["case"], s["table"]
    batch, hq, hkv, ps, most = case["batch"], case["hq"], case["hkv"], case["page"], s["most"]
    page = table.long().clamp(min=0)[:, None]
    head = torch.arange(hkv, device=DEVICE)[None, :, None]
    k, v = (_values(pool.view(torch.uint8)[page, head].view(pool.dtype) if s["scales"] is not None else pool[page, head],
                    s["scales"][page, head][..., i] if s["scales"] is not None else None).reshape(batch, hkv, -1, D) for i, pool in enumerate((s["k"], s["v"])))
    b, at = _places(s)
    i = at - s["first"][b]
    q = torch.zeros((batch, most, hq, D), device=DEVICE)
    q[b, i] = s["q"].float() * SCALE
    # who sees whom, [batch][rows][entries]
    e, row = torch.arange(k.shape[2], device=DEVICE), torch.arange(most, device=DEVICE)
    first, length = s["first"][:, None, None], s["lengths"][:, None, None]
    p = first + row[None, :, None]
    if s["sees"] is None:
        sees = e <= p
    else:
        p = first + s["sees"].sum(-1, keepdim=True) - 1
        mine = s["sees"].gather(2, (e - first).clamp(0, most - 1).expand(batch, most, -1))
        sees = (e < first) | mine
    sees = sees & (e < length)
    if case["window"]:
        sees = sees & ((e > p - case["window"]) | (e < case["sinks"]))
    q = q.view(batch, most, hkv, -1, D).permute(0, 2, 1, 3, 4).reshape(batch, hkv, -1, D)
    logits = torch.matmul(q, k.transpose(2, 3).contiguous()).view(batch, hkv, most, hq // hkv, -1)
    logits.masked_fill_(~sees[:, None, :, None], -math.inf)
    top = logits.amax(-1, keepdim=True)
    w = logits.sub_(torch.where(torch.isinf(top), 0.0, top)).exp_()
    weight = w.sum(-1, keepdim=True)
    out = torch.matmul(w.view(batch, hkv, -1, w.shape[-1]), v).view(batch, hkv, most, -1, D) / torch.where(weight > 0, weight, 1.0)
    out, lse = (x.permute(0, 2, 1, 3, 4).reshape(batch, most, hq, -1)[b, i] for x in (out, top + torch.log(weight)))
    return out.to(torch.float32 if case["f32"] else torch.bfloat16), lse[..., 0]


def run(s):
    case = s["case"]
    if case["kind"] == "rotate":
        if own:
            q = s["cache"].append_rotated(s["seqs"], s["q"], s["new_k"], s["new_v"], s["rotation"], positions=s["positions"], rows=s["most"], first=s["first"], starts=s["starts"])
            k, v = s["cache"].read(s["seqs"], rows=s["most"], first=s["first"], starts=s["starts"], total=s["total"])
            return {"q": q, "k": k, "v": v, "bounds": s["bounds"]}
        return _plain_rotate(s)
    if own:
        if case["rows"] == 1:            # a decode step: one token of every sequence
            out, lse = s["cache"].attend_rows(s["seqs"], s["q"], window=case["window"], sinks=case["sinks"], tree=s["sees"], f32=case["f32"], lse=case["lse"])
        else:
            out, lse = s["cache"].attend_rows(s["seqs"], s["q"], window=case["window"], sinks=case["sinks"], tree=s["sees"], rows=s["most"], starts=s["starts"],
                                              f32=case["f32"], lse=case["lse"])
    else:
        out, lse = _plain_attend(s)
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def _pairs(case):
    """Per sequence: entries that some row sees, and pairs of a row and an entry that it sees."""
    found = []
    for n, r in zip(_lengths(case), _rows(case)):
        first, window = n - r, case["window"] or n + r + 1
        if case["kind"] == "tree":
            sees = _ancestors(r, 0)
            p, upto, more = first + sees.sum(1) - 1, np.full(r, first), sees.sum(1)
        else:
            p = first + np.arange(r)
            upto, more = p + 1, np.zeros(r, np.int64)
        low = np.minimum(np.maximum(p - window + 1, 0), upto)
        sinks = np.minimum(low, case["sinks"])
        found.append((int(n - low.min() + sinks.max()), int((upto - low + sinks + more).sum())))
    return found


def work(case):
    hq, hkv, rows = case["hq"], case["hkv"], _rows(case)
    row = 2 * D + 2 if case["dtype"] == "e4m3" else 4 * D                  # key and value as they are cached
    q = sum(rows) * hq * D
    if case["kind"] == "rotate":
        touched = sum((n - 1) // case["page"] - (n - r) // case["page"] + 1 for n, r in zip(_lengths(case), rows))
        turned = sum(rows) * (hq + hkv) * case["rotary"]
        return {"bytes": 4 * q + hkv * (sum(rows) * (4 * D + row + row + 4 * D) + touched * 4 * D), "flops": 3 * turned}
    pairs = _pairs(case)
    return {"bytes": hkv * sum(n for n, _ in pairs) * row + q * (6 if case["f32"] else 4), "flops": 4.0 * D * hq * sum(n for _, n in pairs)}


# ------------------------------------------------------------------ 64 bits
def _power(e):
    """2 to the whole power e, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_row(x):
    """What rows become in 8 bits."""
    x = x.double()
    big = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(-1, keepdim=True)
    e = torch.frexp(big / 448.0)[1].clamp(-100, 120)                       # big / 448 < 2^e; one less where it is a power of two
    e = torch.where((big <= 448 * _power(e - 1)) & (e > -100), e - 1, e)
    y = x / _power(e)
    step = _power((torch.frexp(y)[1] - 1).clamp(min=-6) - 3)
    y = torch.round(y / step) * step
    return torch.where(torch.isfinite(y), y, torch.full_like(y, math.nan)) * _power(e)


def _exact_rotation(x, position, case):
    """One sequence's rows [rows][heads][128] as complex numbers that turn."""
    n = case["rotary"] // 2
    x = x.double()
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if case["interleaved"] else (slice(0, n), slice(n, 2 * n))
    z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous())
    z = z * torch.polar(torch.ones((), dtype=torch.float64, device=DEVICE), torch.outer(position.double(), _frequencies(case)))[:, None]
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_rotate(case, s):
    starts, first, lengths = s["starts"].tolist(), s["first"].tolist(), s["lengths"].tolist()
    ps, sides, bounds = case["page"], ([], [], []), s["bounds"].double()
    held = _exact_row if s["scales"] is not None else (lambda x: x.double())
    for b, n in enumerate(lengths):
        mine = slice(starts[b], starts[b + 1])
        position = torch.arange(first[b], n, device=DEVICE) if s["positions"] is None else s["positions"][mine]
        sides[0].append(_exact_rotation(s["q"][mine], position, case))
        sides[1].append(held(_exact_rotation(s["new_k"][mine], position, case)))
        sides[2].append(held(s["new_v"][mine]))
        new, row = sides[1][-1], first[b]
        while row < n:
            stop = min(n, (row // ps + 1) * ps)
            part, page = new[row - first[b]:stop - first[b]], int(s["table"][b, row // ps])
            lo, hi = part.amin(0), part.amax(0)
            if row % ps:
                lo, hi = torch.minimum(lo, bounds[page, :, 0]), torch.maximum(hi, bounds[page, :, 1])
            bounds[page, :, 0], bounds[page, :, 1], row = lo, hi, stop
    return {"q": torch.cat(sides[0]), "k": torch.cat(sides[1]), "v": torch.cat(sides[2]), "bounds": bounds}


def _exact_entries(s, i, b, head, at):
    """Keys (i = 0) or values (1) of entries `at` of a sequence, [entries][128]."""
    page, slot = s["table"][b, at // s["case"]["page"]].long(), at % s["case"]["page"]
    if s["scales"] is None:
        return (s["k"], s["v"])[i][page, head, slot].double()
    raw = (s["k"], s["v"])[i].view(torch.uint8)[page, head, slot].view(torch.float8_e4m3fn).double()
    return raw * _power(s["scales"][page, head, slot, i].long() - 127)[:, None]


def exact(case, seed):
    if case["batch"] * case["hkv"] > 2048:
        return None
    s = prepare(dict(case), seed)
    if case["kind"] == "rotate":
        return _exact_rotate(case, s)
    g, window, sinks = case["hq"] // case["hkv"], case["window"], case["sinks"]
    starts = s["starts"].tolist()
    out = torch.zeros((s["total"], case["hq"], D), dtype=torch.float64, device=DEVICE)
    lse = torch.zeros((s["total"], case["hq"]), dtype=torch.float64, device=DEVICE)
    for b, n in enumerate(s["lengths"].tolist()):
        first, r = int(s["first"][b]), starts[b + 1] - starts[b]
        for lo in range(0, r, 1024):                     # so many rows at once, over what any of them sees
            hi = min(r, lo + 1024)
            own_rows = torch.arange(lo, hi, device=DEVICE)
            oldest = max(0, first + (0 if case["kind"] == "tree" else lo) - window) if window else 0
            end = n if case["kind"] == "tree" else first + hi
            at = torch.cat((torch.arange(min(sinks, oldest), device=DEVICE), torch.arange(oldest, end, device=DEVICE)))
            if case["kind"] == "tree":
                mask = torch.cat((torch.ones((hi - lo, first), dtype=torch.bool, device=DEVICE), s["sees"][b, lo:hi, :r]), 1)[:, at]
                position = first + s["sees"][b, lo:hi, :r].sum(1) - 1
            else:
                position = first + own_rows
                mask = at[None] <= position[:, None]
            if window:
                mask = mask & ((position[:, None] - at[None] < window) | (at[None] < sinks))
            for h in range(case["hkv"]):
                k, v = (_exact_entries(s, i, b, h, at) for i in (0, 1))
                q = s["q"][starts[b] + lo:starts[b] + hi, h * g:(h + 1) * g].double()
                for j in range(g):
                    z = torch.where(mask, q[:, j] @ k.T / math.sqrt(D), -math.inf)
                    total = torch.logsumexp(z, 1)
                    out[starts[b] + lo:starts[b] + hi, h * g + j] = torch.exp(z - total[:, None]) @ v
                    lse[starts[b] + lo:starts[b] + hi, h * g + j] = total
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}
