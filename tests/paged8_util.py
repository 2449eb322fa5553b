"""Shared helpers of the 8-bit paged-cache GPU tests (not collected by pytest itself).

Caches are built so that what must not be read hurts if it is: pages in random order,
pages of no sequence and rows past a sequence's length full of NaN, scales of blocks
without rows NaN, table entries past a sequence's last page -1.
"""

from __future__ import annotations

import numpy as np
import torch

import paper_2511_14694_amd as F
from gpu_util import DEV
from oracle import paged8 as O

E4M3 = torch.float8_e4m3fn
NAN = 0x7f


def i32(x):
    return torch.as_tensor(np.asarray(x, np.int32)).to(DEV)


def random_rows(rng, shape):
    """Codes of e4m3 numbers, normal values among them, the extremes too."""
    x = torch.as_tensor((rng.standard_normal(shape) * 60.0).astype(np.float32)).clamp(-448, 448)
    x[torch.as_tensor(rng.random(shape) < 0.02)] = 448.0
    x[torch.as_tensor(rng.random(shape) < 0.02)] = -2.0 ** -9
    return x.to(E4M3)


class Cache8:
    """An 8-bit paged cache of sequences of `lens` rows: dev, and in float64 its pools of
    8-bit numbers and scales, (pk, pv) [pages, page, H_kv, D] and (ks, vs) [pages, H_kv,
    blocks]; pages `free` of no sequence."""

    def __init__(self, rng, lens, kv_heads, dim, page, block, max_pages=None, by_head=False, spare=0, padded=False,
                 odd_scales=False):
        need = [-(-n // page) for n in lens]
        self.page, self.block, self.lens = page, block, list(lens)
        self.max_pages = max(max(need, default=0), 1) if max_pages is None else max_pages
        total = sum(need) + spare + 1
        order = [int(x) for x in rng.permutation(total)]
        self.table = np.full((len(lens), self.max_pages), -1, np.int32)
        codes = [torch.full((total, page, kv_heads, dim), NAN, dtype=torch.uint8) for _ in range(2)]
        scales = [torch.full((total, kv_heads, page // block), float("nan")) for _ in range(2)]
        for b, n in enumerate(lens):
            ids = [order.pop() for _ in range(need[b])]
            self.table[b, :need[b]] = ids
            for j, p in enumerate(ids):
                rows = min(page, n - j * page)
                for to, sc in zip(codes, scales):
                    to[p, :rows] = random_rows(rng, (rows, kv_heads, dim)).view(torch.uint8)
                    blocks = -(-rows // block)
                    e = rng.integers(-9, -4, (kv_heads, blocks)).astype(np.float64)
                    s = 2.0 ** e * (rng.uniform(1, 2, e.shape) if odd_scales else 1.0)
                    sc[p, :, :blocks] = torch.as_tensor(s.astype(np.float32))
        self.free = order
        t = [x.to(DEV) for x in codes]
        if by_head:
            t = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in t]
        elif padded:             # rows inside a wider pool: [pages, page, 2 H_kv, D]
            wide = [torch.full((total, page, 2 * kv_heads, dim), NAN, dtype=torch.uint8, device=DEV) for _ in t]
            for w, x in zip(wide, t):
                w[:, :, kv_heads:] = x
            t = [w[:, :, kv_heads:] for w in wide]
        self.dev = F.PagedCache8(*(x.view(E4M3) for x in t), *(s.to(DEV) for s in scales),
                                 torch.as_tensor(self.table).to(DEV), i32(lens))
        self.refresh()

    def refresh(self):
        """The float64 copies, as the device holds them."""
        self.pk, self.pv = (to_codes(getattr(self.dev, n)) for n in "kv")
        self.ks, self.vs = (getattr(self.dev, n).cpu().double().numpy() for n in ("k_scale", "v_scale"))

    def rows(self, b, n, which="k", scaled=True):
        """Rows 0 .. n-1 of sequence b: [n, H_kv, D], dequantised or (scaled False) as 8-bit
        numbers."""
        pool, scale = (self.pk, self.ks) if which == "k" else (self.pv, self.vs)
        r = np.arange(n)
        p = self.table[b][r // self.page]
        x = pool[p, r % self.page]
        return x * scale[p, :, r % self.page // self.block][:, :, None] if scaled else x


def to_codes(t):
    """What an e4m3 tensor holds, float64."""
    return t.cpu().float().double().numpy()


def appended(c, k, v, start, cu):
    """What the pools of c must hold after an append of k, v [rows, H_kv, D] (float64):
    (pk, pv, ks, vs), all else as it was."""
    out = [x.copy() for x in (c.pk, c.pv, c.ks, c.vs)]
    for b in range(len(c.lens)):
        if start[b] < 0 or cu[b + 1] == cu[b]:
            continue
        n = start[b] + cu[b + 1] - cu[b]
        r = np.arange(n)
        p = c.table[b][r // c.page]
        blocks = -(-n // c.block)
        bp, bi = c.table[b][np.arange(blocks) * c.block // c.page], np.arange(blocks) * c.block % c.page // c.block
        for new, pool, scale in ((k, out[0], out[2]), (v, out[1], out[3])):
            for g in range(pool.shape[2]):
                rows, s = O.append(pool[p, r % c.page, g], scale[bp, g, bi], c.block, start[b], new[cu[b]:cu[b + 1], g])
                pool[p, r % c.page, g] = rows
                scale[bp, g, bi] = s
    return out


def same(got, ref, what):
    assert np.array_equal(got, ref, equal_nan=True), f"{what}: {(~((got == ref) | (np.isnan(got) & np.isnan(ref)))).sum()} differ"
