"""Oracle: rotary positions, attention over a paged cache and its eviction -- TEST
INFRASTRUCTURE.

What is computed, in float64:

* turns: revolutions per position of the pairs of a head, theta^(-2i/R) / (2 pi),
  scaled for contexts longer than the trained one by interpolating all positions
  ("linear"), by changing theta so that the slowest pair is interpolated and the
  fastest is not ("base"), or by bands of how often a pair turns over the trained
  context ("bands": the YaRN paper's ramp, arXiv 2309.00071 section 3.2).
* rope: every pair turned by 2 pi pos turns, as a complex product; the inverse is the
  conjugate.
* rows: the cached rows of a sequence, page by page.
* decode: softmax attention of one query per head over these rows, and the weight
  every row receives, per KV head.
* keep: the rows that stay when a cache is cut to a budget by accumulated weight.
"""

from __future__ import annotations

import math

import numpy as np


def turns(rot, theta=10000.0, scaling="none", factor=1.0, context=0.0, low=1.0, high=32.0):
    out = []
    for i in range(rot // 2):
        base = theta * factor ** (rot / (rot - 2)) if scaling == "base" else theta
        f = 1.0 / (2.0 * math.pi * base ** (2.0 * i / rot))
        if scaling == "linear":
            f = f / factor
        elif scaling == "bands":
            r = f * context                      # revolutions over the trained context
            if r <= low:
                f = f / factor
            elif r < high:
                g = (r - low) / (high - low)
                f = (1.0 - g) * f / factor + g * f
        out.append(f)
    return np.array(out)


def rope(x, pos, turns_, pairs="interleaved", inverse=False, amplitude=1.0):
    """x [rows, heads, D]; the first 2 len(turns_) elements of every head turned."""
    y = np.array(x, np.float64)
    rot = 2 * len(turns_)
    a = np.multiply.outer(np.asarray(pos, np.float64), turns_)
    z = np.exp(2j * np.pi * (a - np.floor(a)))
    z = amplitude * (z.conj() if inverse else z)[:, None, :]
    re, im = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if pairs == "interleaved" else \
        (np.arange(rot // 2), np.arange(rot // 2, rot))
    w = (y[:, :, re] + 1j * y[:, :, im]) * z
    y[:, :, re], y[:, :, im] = w.real, w.imag
    return y


def rows(pool, table_row, n):
    """Rows 0 .. n-1 of a sequence from a pool [pages, page_rows, ...]."""
    page = pool.shape[1]
    return np.stack([pool[table_row[r // page], r % page] for r in range(n)]) if n else \
        np.zeros((0,) + pool.shape[2:], pool.dtype)


def decode(q, k, v, scale=None, visible=None):
    """q [H, D], k, v [n, H_kv, D] -> o [H, D], lse [H], weight [H_kv, n].  visible [n]:
    rows that count (default all); none: zeros and -inf."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    H, D = q.shape
    n, K = k.shape[:2]
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    seen = np.ones(n, bool) if visible is None else np.asarray(visible, bool)
    o, lse, w = np.zeros((H, D)), np.full(H, -np.inf), np.zeros((K, n))
    if not seen.any():
        return o, lse, w
    for h in range(H):
        g = h // (H // K)
        s = scale * (k[seen, g] @ q[h])
        top = s.max()
        e = np.exp(s - top)
        lse[h] = top + math.log(e.sum())
        p = e / e.sum()
        o[h] = p @ v[seen, g]
        w[g, seen] += p
    return o, lse, w


def keep(weight, budget, recent):
    """Rows kept of a head whose rows have these weights, ascending: the last `recent`
    and the heaviest others, the lower row first among equals, a NaN above all."""
    n = len(weight)
    m = min(n, max(budget, 0))
    recent = min(recent, m)
    old = list(range(n - recent))
    old.sort(key=lambda r: (0, 0.0, r) if math.isnan(weight[r]) else (1, -float(weight[r]), r))
    return sorted(old[:m - recent]) + list(range(n - recent, n))
