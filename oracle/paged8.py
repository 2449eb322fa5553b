"""Oracle: slots of a paged cache, its rows held in 8 bits, and attention over them -- TEST
INFRASTRUCTURE.

What is computed, in float64 and whole numbers, one sequence, row and page after another:

* E4M3: the numbers of the 8-bit type (1 sign, 4 exponent with bias 7, 3 mantissa bits; the
  last magnitude is NaN, there is no infinity), from the definition; nearest: the nearest
  of them, ties to the one with an even last bit.
* scale_of: the least power of two, 2^-126 at least, at which values fit.
* append: new rows of one sequence and head in blocks that share a scale.
* attend: softmax attention of a sequence's newest tokens, each up to its own row.
* extend: pages given back and taken, with the maps of the new rows.
"""

from __future__ import annotations

import math

import numpy as np

from . import paged


def _numbers():
    out = []
    for code in range(0x7f):
        e, m = code >> 3, code & 7
        out.append(m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return np.array(out)


E4M3 = _numbers()       # of codes 0 .. 0x7e, ascending


def nearest(x):
    """The nearest e4m3 number to each x, |x| <= 448; NaN for what is not finite."""
    x = np.asarray(x, np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    assert a.max(initial=0.0) <= 448.0
    hi = np.clip(np.searchsorted(E4M3, a), 1, len(E4M3) - 1)
    lo = hi - 1
    to_lo, to_hi = a - E4M3[lo], E4M3[hi] - a
    take = np.where(to_lo < to_hi, lo, np.where(to_hi < to_lo, hi, np.where(lo % 2 == 0, lo, hi)))
    return np.where(np.isfinite(x), np.copysign(E4M3[take], x), np.nan)


def scale_of(x):
    """2^e with the least e >= -126 at which all finite |x| <= 448 2^e."""
    x = np.asarray(x, np.float64)
    most = np.abs(x[np.isfinite(x)]).max(initial=0.0)
    e = -126
    while most > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def append(rows, scales, block, start, new):
    """rows [n, D] (e4m3 numbers; those before start count) and scales [blocks] of one
    sequence and head; new [m, D] behind the first start.  Returns the rows up to the last
    new one and the scales."""
    rows, scales = np.array(rows, np.float64), np.array(scales, np.float64)
    end = start + len(new)
    out = np.zeros((end, new.shape[1]))
    out[:start] = rows[:start]
    for j in range(start // block, -(-end // block) if len(new) else 0):
        at = range(max(start, j * block), min(end, (j + 1) * block))
        x = np.stack([new[r - start] for r in at])
        s = scale_of(x)
        if j * block < start:
            if not scales[j] >= s:
                for r in range(j * block, start):
                    out[r] = nearest(out[r] * (scales[j] / s))
            else:
                s = scales[j]
        with np.errstate(invalid="ignore"):
            out[at.start:at.stop] = nearest(x / s)
        scales[j] = s
    return out, scales


def attend(q, k, v, scale=None, visible=None):
    """q [m, H, D] the last m tokens over k, v [n, H_kv, D] -> o [m, H, D], lse [m, H]; a
    token without rows to see: zeros and -inf.  visible [n]: rows that count (default all)."""
    m, n = len(q), len(k)
    o, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    for i in range(m):
        upto = max(0, n - (m - 1 - i))
        seen = None if visible is None else visible[:upto]
        o[i], lse[i], _ = paged.decode(q[i], k[:upto], v[:upto], scale, seen)
    return o, lse


def extend(table, length, page, add, free, n_rows, first_pos=None):
    """table (lists, changed), length, free (lists, changed) -> start, cu, seq, slot, pos
    (lists) and whether all were served."""
    up = lambda n: -(-n // page)  # noqa: E731
    batch = len(add)
    start, fine = [0] * batch, True
    for b, a in enumerate(add):
        if a <= 0:
            n = max(length[b] + a, 0)
            for j in range(up(n), up(length[b])):
                free.append(table[b][j])
                table[b][j] = -1
            length[b] = start[b] = n
    cu, seq, slot, pos, dry = [0], [], [], [], False
    for b, a in enumerate(add):
        cu.append(min(cu[-1] + max(a, 0), 2 ** 31 - 1))
        if a <= 0:
            continue
        have, want = up(length[b]), up(length[b] + a)
        ok = want <= len(table[b]) and cu[-1] <= n_rows
        if ok and want > have:
            dry = dry or want - have > len(free)
            ok = not dry
        if ok:
            for j in range(have, want):
                table[b][j] = free.pop()
        start[b] = length[b] if ok else -1
        fine = fine and ok
        for i in range(min(a, n_rows - len(seq))):
            seq.append(b)
            slot.append(start[b] + i if ok else -1)
            pos.append(slot[-1] if first_pos is None else first_pos[b] + i)
        length[b] += a if ok else 0
    for x in (seq, slot, pos):
        x += [-1] * (n_rows - len(x))
    return start, cu, seq, slot, pos, fine


def attend_tolerances(q, k, v, scale, dtype, o):
    """Bounds of o [m, H, D] and lse [m, H] for float32 arithmetic over dequantised k, v
    [n, H_kv, D].

    A score is a float32 sum of D exact products (e4m3 by bf16; of 3 D for float32 queries,
    which enter in three bf16 parts), times the block's scale: off by at most (3 D + 5) or
    (D + 5) 2^-24 of its terms' absolute sum, e below (the 5: the block's scale, the
    softmax scale, log2 e, the difference to the maximum and its exponential).  The sums
    over the rows run in partial sums of at most n / 16 + 64 terms: d below.  A weight is
    then relatively off by 2 (e + d), and o by that times the largest |v|; weights times the
    block's scale (2^-24) enter in two bf16 parts, off by 2^-16 of them, or three for float32,
    2^-24.  The output is rounded once.  lse is off by e + d and by the rounding of its
    logarithm and products, 2^-22 of its absolute terms."""
    m, H, D = q.shape
    n, K = k.shape[:2]
    terms = np.zeros((m, H))
    for h in range(H):
        terms[:, h] = scale * (np.abs(k[:, h // (H // K)]) @ np.abs(q[:, h]).T).max(0, initial=0.0)
    e = terms * ((D if dtype == "bf16" else 3 * D) + 5) * 2.0 ** -24
    d = (n / 16 + 64) * 2.0 ** -24
    rel = 2 * (e + d) + 2.0 ** -23 + (2.0 ** -16 if dtype == "bf16" else 0.0)
    half = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}[dtype]
    to = rel[..., None] * np.abs(v).max(initial=0.0) + half * (np.abs(o) + 1e-30)
    return to * (1 + 2.0 ** -7), e + d + (terms + math.log(max(n, 1))) * 2.0 ** -22
