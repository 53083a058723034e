"""Plain CPU definitions of the cache in pages (ckv_paged_* of include/ckv.h) in 64 bits: what rows become in 8 bits, a page's extremes,
attention of one token and of several rows, the pages that scores pick, and positions' rotations.  numpy; test infrastructure only."""
from __future__ import annotations

import math

import numpy as np

D = 128


def e4m3_values():
    """The 256 codes' values: sign, four bits of exponent (bias 7, 0 subnormal), three of mantissa; all ones is NaN, there is no infinity."""
    v = np.zeros(256)
    for c in range(128):
        e, m = c >> 3, c & 7
        v[c] = math.nan if c == 127 else m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[c + 128] = -v[c]
    return v


E4M3 = e4m3_values()
_GRID = E4M3[:127]                       # ascending, 0 .. 448


def e4m3_codes(y):
    """Nearest code of each value (|y| <= 448), ties to the even code; NaN for what is not finite."""
    a = np.abs(np.where(np.isfinite(y), y, 0.0))
    hi = np.clip(np.searchsorted(_GRID, a), 1, 126)
    lo = hi - 1
    below, above = a - _GRID[lo], _GRID[hi] - a
    c = np.where(below < above, lo, np.where(above < below, hi, np.where(lo % 2 == 0, lo, hi)))
    return np.where(np.isfinite(y), c + 128 * np.signbit(y), 127).astype(np.uint8)


def quantise(x):
    """(codes, E) of rows [..., 128]."""
    x = np.asarray(x, np.float64)
    big = np.where(np.isfinite(x), np.abs(x), 0.0).max(-1)
    e = np.full(big.shape, -100)
    for i, b in np.ndenumerate(big):
        n = -100
        if b > 448 * 2.0 ** -100:
            n = math.frexp(b / 448)[1] - 1           # 2^n <= b / 448
            while b > math.ldexp(448.0, n):
                n += 1
        e[i] = min(n, 120)
    return e4m3_codes(np.ldexp(x, -e[..., None])), e


def dequantise(codes, e):
    """Values as bf16 has them: all codes times 2^E but one are its numbers (4 bits, exponents within its range); what a magnitude from 1.9375 * 2^127 on
    rounds to, 2^128, is infinite there as in a float."""
    x = np.ldexp(E4M3[codes], np.asarray(e)[..., None])
    return np.where(np.abs(x) >= 2.0 ** 128, np.copysign(np.inf, x), x)


def extremes(k):
    """Least and largest of each dimension over rows [n][128], NaN left out (+inf, -inf where nothing is left)."""
    k = np.asarray(k, np.float64)
    return np.where(np.isnan(k), np.inf, k).min(0), np.where(np.isnan(k), -np.inf, k).max(0)


def attend(q, k, v, scale):
    """One head: q [128], k, v [n][128] -> (out [128], lse, sum of |weight * value| [128], largest sum |q k| scale)."""
    if len(k) == 0:
        return np.zeros(D), -np.inf, np.zeros(D), 0.0
    s = (k * q).sum(1) * scale
    m = s.max()
    if m == -np.inf:
        return np.zeros(D), -np.inf, np.zeros(D), 0.0
    w = np.exp(s - m)
    w_sum = w.sum()
    reach = float((np.abs(k) * np.abs(q))[s > -np.inf].sum(1).max() * scale)
    return (w[:, None] * v).sum(0) / w_sum, m + math.log(w_sum), (w[:, None] * np.abs(v)).sum(0) / w_sum, reach


def sees(first, rows, window=0, sinks=0, tree=None):
    """Which of the first + rows entries of a sequence each of its last `rows` rows sees, bool [rows][first + rows]."""
    e, i = np.arange(first + rows)[None], np.arange(rows)[:, None]
    if tree is None:
        p = first + i
        m = e <= p
    else:
        tree = np.asarray(tree, bool)[:rows, :rows]
        p = first + tree.sum(1, keepdims=True) - 1
        m = np.concatenate([np.ones((rows, first), bool), tree], 1)
    return m & ((e > p - window) | ((e < sinks) & (e <= p) if tree is None else (e < sinks))) if window else m


def attend_rows(q, k, v, mask, scale):
    """Rows q [rows][128] over entries k, v [n][128] as far as mask [rows][n] says: outputs, lse, sums of |weight * value|, largest sum |q k| scale of each row."""
    n = len(q)
    if k.shape[0] == 0:
        return np.zeros((n, D)), np.full(n, -np.inf), np.zeros((n, D)), np.zeros(n)
    with np.errstate(invalid="ignore", divide="ignore"):
        s = np.where(mask, (q @ np.where(mask.any(0)[:, None], k, 0.0).T) * scale, -np.inf)
        m = s.max(1, keepdims=True)
        w = np.exp(s - np.where(np.isinf(m), 0.0, m))
        total = w.sum(1)
        some = np.where(total > 0, total, 1.0)
        clean = np.where(np.isfinite(v), v, 0.0)
        out, mass = w @ clean / some[:, None], w @ np.abs(clean) / some[:, None]
        reach = np.where(s > -np.inf, (np.abs(q) @ np.abs(np.where(np.isfinite(k), k, 0.0)).T) * scale, 0.0).max(1)
        return out, np.where(total > 0, m[:, 0] + np.log(some), -np.inf), mass, reach


def scores(q, lo, hi):
    """Scores of pages: q [G][128], lo, hi [pages][128].  A zero of a query adds nothing, whatever the extremes."""
    q = np.asarray(q, np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        return np.where(q[:, None] == 0, 0.0, np.maximum(q[:, None] * lo[None], q[:, None] * hi[None])).sum(-1).sum(0).astype(np.float32)


def pick(score, keep, first, last):
    """Pages picked by score [held], ascending, -1 behind."""
    held = len(score)
    out = np.full(keep, -1, np.int32)
    if held <= keep:
        out[:held] = np.arange(held)
        return out
    forced = [i for i in range(held) if i < first or i >= held - last]
    rest = sorted((i for i in range(held) if first <= i < held - last), key=lambda i: (0 if np.isnan(score[i]) else 1, 0.0 if np.isnan(score[i]) else -float(score[i]), i))
    out[:] = sorted(forced + rest[:keep - len(forced)])
    return out


def rotate(x, positions, frequencies, interleaved=False, magnitude=1.0):
    """Rows x [..., rows, heads, 128] turned by their positions [..., rows]."""
    x, n = np.asarray(x, np.float64), len(frequencies)
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    angle = (np.asarray(positions, np.float64)[..., None] * np.asarray(frequencies, np.float64))[..., None, :]
    c, s = magnitude * np.cos(angle), magnitude * np.sin(angle)
    y = x.copy()
    y[..., first], y[..., second] = x[..., first] * c - x[..., second] * s, x[..., second] * c + x[..., first] * s
    return y


def pair_size(x, n, interleaved=False):
    """|x| + |y| of the pair that each dimension is in (0 where it is in none), of which a rounded rotation is off by a share."""
    a = np.abs(np.asarray(x, np.float64))
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    y = np.zeros_like(a)
    y[..., first] = y[..., second] = a[..., first] + a[..., second]
    return y
