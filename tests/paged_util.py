"""Shared helpers of the paged-cache GPU tests (not collected by pytest itself).

Caches are built so that what must not be read hurts if it is: pages in random order,
pages of no sequence and rows past a sequence's length full of NaN, table entries past
a sequence's last page -1.

Rounding: a value rounded to a type is off by at most half a step, 2^-8 of it for bf16
and 2^-24 for float32.
"""

from __future__ import annotations

import numpy as np
import torch

import paper_2511_14694_amd as F
from gpu_util import DEV, to64, torch_dtype  # noqa: F401

HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def values(rng, shape, dtype, scale=1.0):
    """A device tensor of normal values and what it holds, in float64."""
    t = torch.as_tensor((rng.standard_normal(shape) * scale).astype(np.float32)).to(torch_dtype(dtype)).to(DEV)
    return t, to64(t)


class Cache:
    """A paged cache of sequences of `lens` rows, with its rows in float64: k[b], v[b]
    [len, H_kv, D]; spare pages (all NaN) for other tables of the same pool."""

    def __init__(self, rng, lens, kv_heads, dim, page, dtype="bf16", max_pages=None, weight=False, by_head=False,
                 spare=0, padded=False):
        need = [-(-n // page) for n in lens]
        self.page, self.lens = page, list(lens)
        self.max_pages = max(max(need, default=0), 1) if max_pages is None else max_pages
        total = sum(need) + spare + 1
        order = [int(x) for x in rng.permutation(total)]
        self.table = np.full((len(lens), self.max_pages), -1, np.int32)
        pool = [np.full((total, page, kv_heads, dim), np.nan, np.float32) for _ in range(2)]
        self.k, self.v = [], []
        for b, n in enumerate(lens):
            ids = [order.pop() for _ in range(need[b])]
            self.table[b, :need[b]] = ids
            for to, x in ((self.k, pool[0]), (self.v, pool[1])):
                r = torch.as_tensor(rng.standard_normal((n, kv_heads, dim)).astype(np.float32))
                r = r.to(torch_dtype(dtype)).float().numpy()
                to.append(r.astype(np.float64))
                for j in range(need[b]):
                    part = r[j * page:(j + 1) * page]
                    x[ids[j], :len(part)] = part
        self.free = order        # pages of no sequence
        t = [torch.as_tensor(x).to(torch_dtype(dtype)).to(DEV) for x in pool]
        if by_head:
            t = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in t]
        elif padded:             # rows inside a wider pool: [pages, page, 2 H_kv, D]
            both = torch.full((total, page, 2 * kv_heads, dim), float("nan"), dtype=t[0].dtype, device=DEV)
            wide = [both, both.clone()]
            for w, x in zip(wide, t):
                w[:, :, kv_heads:] = x
            t = [w[:, :, kv_heads:] for w in wide]
        w = None
        if weight:
            self.weight = rng.random((len(lens), kv_heads, self.max_pages * page)).astype(np.float32)
            w = torch.as_tensor(self.weight).to(DEV)
        self.dev = F.PagedCache(t[0], t[1], torch.as_tensor(self.table).to(DEV),
                                torch.as_tensor(np.asarray(lens, np.int32)).to(DEV), w)

    def other(self, rng, rows, weight=True):
        """A cache of the same pool with tables of its own for `rows` rows a sequence."""
        per = -(-rows // self.page) if rows else 1
        table = np.array([[self.free.pop() for _ in range(per)] for _ in self.lens], np.int32).reshape(len(self.lens), per)
        w = torch.full((len(self.lens), self.dev.k.shape[2], per * self.page), -1.0, device=DEV) if weight else None
        return F.PagedCache(self.dev.k, self.dev.v, torch.as_tensor(table).to(DEV),
                            torch.full((len(self.lens),), -1, dtype=torch.int32, device=DEV), w)


def paged_rows(cache, b, n, which="k"):
    """Rows 0 .. n-1 of sequence b of a device cache, float64 [n, H_kv, D]."""
    pool = getattr(cache, which)
    page = pool.shape[1]
    table = cache.table.cpu().numpy()
    if n == 0:
        return np.zeros((0,) + tuple(pool.shape[2:]))
    r = np.arange(n)
    return to64(pool[torch.as_tensor(table[b][r // page].astype(np.int64)).to(DEV), torch.as_tensor(r % page).to(DEV)])


def within(got, ref, tol, what):
    """|got - ref| <= tol elementwise, infinities and NaN alike."""
    got, ref, tol = np.broadcast_arrays(np.asarray(got, np.float64), np.asarray(ref, np.float64),
                                        np.asarray(tol, np.float64))
    fine = np.isfinite(ref)
    assert np.array_equal(got[~fine], ref[~fine], equal_nan=True), f"{what}: not finite values differ"
    err = np.abs(got[fine] - ref[fine])
    bad = ~(err <= tol[fine])
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {err[bad].max():.3e} where " \
                          f"{tol[fine][bad][np.argmax(err[bad])]:.3e} is allowed"


def decode_tolerances(q, k, scale, dtype, v, o):
    """Bounds of one sequence's o [H, D], lse [H] and of the relative error of its
    softmax weights [H], for float32 arithmetic.

    A score is a sum of D float32 products (of exact ones for bf16): off by at most
    (D + 4) 2^-24 of its terms' absolute sum, e below (the 4: scale, log2 e, the
    difference to the maximum and its exponential).  The sums over the rows run in
    partial sums of at most n / 16 + 64 terms: d below.  A weight is then relatively off
    by 2 (e + d), and o by that times the largest |v|; the products with v may take the
    weights in two bf16 parts, off by 2^-16 of them.  lse is off by e + d and by the
    rounding of its logarithm and products, 2^-22 of its absolute terms."""
    H, D = q.shape
    n, K = k.shape[:2]
    e = np.zeros(H)
    for h in range(H):
        e[h] = scale * (np.abs(k[:, h // (H // K)]) @ np.abs(q[h])).max(initial=0.0) * (D + 4) * 2.0 ** -24
    d = (n / 16 + 64) * 2.0 ** -24
    rel = 2 * (e + d)
    vmax = np.abs(v).max(initial=0.0)
    to = ((rel + (2.0 ** -16 if dtype == "bf16" else 0.0)) * vmax)[:, None] + HALF_STEP[dtype] * (np.abs(o) + 1e-30)
    to = to * (1 + 2.0 ** -7)
    smax = e / ((D + 4) * 2.0 ** -24) + np.log(max(n, 1))
    return to, e + d + smax * 2.0 ** -22, rel
