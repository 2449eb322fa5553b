"""focus_paged_append on the GPU against the oracle, element for element: e4m3 numbers and
scales are exact, so nothing is allowed to differ."""

import numpy as np
import pytest
import torch

import paper_2511_14694_amd as F
from gpu_util import DEV, announce
from oracle import paged8 as O
from paged8_util import Cache8, appended, i32, same, to_codes
from paged_util import values

pytestmark = pytest.mark.gpu


def _offsets(counts):
    return [0] + [int(x) for x in np.cumsum(counts)]


def _check(c, k64, v64, start, cu, what=""):
    ref = appended(c, k64, v64, start, cu)
    c.refresh()
    for got, want, name in zip((c.pk, c.pv, c.ks, c.vs), ref, ("k", "v", "k_scale", "v_scale")):
        same(got, want, f"{what} {name}")


def _new(rng, counts, K, D, dtype, spread=6):
    """k, v with a magnitude of its own for each row and head."""
    out = []
    for _ in range(2):
        n = sum(counts)
        x = rng.standard_normal((n, K, D)) * 2.0 ** rng.integers(-spread, spread, (n, K, 1))
        out.append(values(np.random.default_rng(0), (0,), dtype) if n == 0 else None)
        t = torch.as_tensor(x.astype(np.float32)).to(torch.bfloat16 if dtype == "bf16" else torch.float32).to(DEV)
        out[-1] = (t, t.float().cpu().double().numpy())
    return out


@pytest.mark.parametrize("lens,add,K,D,page,block,dtype,by_head", [
    ([0], [1], 1, 16, 8, 8, "bf16", False),
    ([5, 8, 15], [1, 1, 1], 2, 64, 16, 8, "bf16", False),
    ([0, 3, 16, 31], [33, 0, 16, 1], 3, 128, 16, 16, "bf16", True),
    ([7, 100], [250, 3], 8, 128, 64, 32, "bf16", False),
    ([9, 0, 61], [130, 64, 2], 1, 96, 64, 64, "f32", False),
    ([1, 2], [5, 700], 2, 256, 256, 256, "bf16", False),
    ([3], [2100], 1, 64, 1024, 1024, "f32", True),
    ([10, 20, 30], [40, 50, 60], 5, 192, 32, 8, "f32", False),
    ([12], [1030], 4, 128, 128, 128, "bf16", False),
    ([1000], [1], 2, 256, 1024, 512, "f32", False),
    ([3, 70], [130, 200], 3, 128, 64, 64, "bf16", False),
    ([50, 0], [90, 300], 2, 64, 64, 64, "f32", True),
    ([100, 300], [257, 400], 2, 256, 128, 128, "bf16", True),
    ([120], [513], 3, 128, 128, 128, "f32", False),
])
@pytest.mark.parametrize("fused", [False, True])
def test_append_matches_oracle(lens, add, K, D, page, block, dtype, by_head, fused):
    announce(f"append {lens} + {add} {K} x {D} page {page} block {block} {dtype} by_head {by_head} fused {fused}")
    rng = np.random.default_rng(sum(lens) + sum(add) + D)
    ends = [n + a for n, a in zip(lens, add)]
    c = Cache8(rng, ends, K, D, page, block, by_head=by_head, padded=not by_head and fused)
    c.dev.length.copy_(i32(lens))
    (k, k64), (v, v64) = _new(rng, add, K, D, dtype)
    if fused:
        both = torch.cat((k, v), 1)
        k, v = both[:, :K], both[:, K:]
    cu = _offsets(add)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    F.focus_paged_append(k, v, c.dev, i32(lens), i32(cu), err=err)
    _check(c, k64, v64, lens, cu, "first")
    assert c.dev.length.tolist() == [e if a else n for n, a, e in zip(lens, add, ends)] and err.item() == 0
    # the same rows again, from an earlier row on: those behind it are overwritten
    start = [max(0, n - 3) for n in lens]
    F.focus_paged_append(k, v, c.dev, i32(start), i32(cu), err=err)
    _check(c, k64, v64, start, cu, "again")
    assert err.item() == 0


def test_append_one_row_a_sequence_without_offsets():
    rng = np.random.default_rng(5)
    lens = [int(x) for x in rng.integers(0, 70, 300)]
    c = Cache8(rng, [n + 1 for n in lens], 2, 64, 16, 16)
    (k, k64), (v, v64) = _new(rng, [1] * 300, 2, 64, "bf16")
    announce("append 300 sequences")
    F.focus_paged_append(k, v, c.dev, i32(lens))
    _check(c, k64, v64, lens, list(range(301)))


@pytest.mark.parametrize("batch,most", [(70, 3), (600, 9), (5000, 2), (65, 200)])
def test_append_finds_its_sequences(batch, most):
    """Many ragged sequences, many of them without rows."""
    rng = np.random.default_rng(batch)
    lens = [int(x) for x in rng.integers(0, 12, batch)]
    add = [int(x) if y else 0 for x, y in zip(rng.integers(0, most + 1, batch), rng.random(batch) < 0.6)]
    add[-1] = 0
    c = Cache8(rng, [n + a for n, a in zip(lens, add)], 1, 16, 8, 8)
    (k, k64), (v, v64) = _new(rng, add, 1, 16, "f32")
    announce(f"append {batch} ragged sequences")
    F.focus_paged_append(k, v, c.dev, i32(lens), i32(_offsets(add)))
    _check(c, k64, v64, lens, _offsets(add))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_row_by_row_grows_scales(dtype):
    """Rows that grow from the smallest numbers of the type to the largest: every step turns
    the block's rows to the new scale."""
    rng = np.random.default_rng(7)
    D, block = 32, 8
    c = Cache8(rng, [24], 1, D, 8, block)
    c.dev.length.zero_()
    c.dev.k_scale.fill_(float("nan"))
    c.dev.v_scale.fill_(float("nan"))
    c.refresh()
    e = np.linspace(-149 if dtype == "f32" else -133, 127, 24)
    announce(f"append growing {dtype}")
    for r in range(24):
        x = (rng.uniform(-1, 1, (1, 1, D)) * 2.0 ** e[r]).astype(np.float32)
        x[0, 0, 0] = np.float32(2.0 ** np.floor(e[r]))
        t = torch.as_tensor(x).to(torch.bfloat16 if dtype == "bf16" else torch.float32).to(DEV)
        t64 = t.double().cpu().numpy()
        F.focus_paged_append(t, -t, c.dev, i32([r]))
        _check(c, t64, -t64, [r], [0, 1], f"row {r}")
    assert c.dev.length.tolist() == [24]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_special_values(dtype):
    """Zeros, numbers around the edges of a scale, infinities, NaN, subnormal numbers; blocks
    of nothing finite; every bf16 number."""
    rng = np.random.default_rng(8)
    D, K = 128, 2
    inf, nan, tiny = np.inf, np.nan, 2.0 ** -149 if dtype == "f32" else 2.0 ** -133
    x = np.zeros((48, K, D), np.float32)
    x[8, 0, :4] = [448.0, -448.0, 2.0 ** -9, 2.0 ** -10]
    x[8, 1, :4] = [450.0, 1.0, -2.0 ** -10, 464.0]
    x[16, 0, :5] = [inf, -inf, nan, 3.0, -448.0]
    x[16:24, 1] = rng.choice(np.array([inf, -inf, nan], np.float32), (8, D))
    x[24, 0, :3] = [tiny, -tiny, 2.0 ** -126]
    x[24, 1, :3] = [3.38e38, -3.38e38, 1e30]
    x[32:, 1] = rng.standard_normal((16, D)) * 1e-38
    x[32:40, 0, ::2] = -0.0
    c = Cache8(rng, [48, 512], K, D, 16, 8)
    full = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).float().reshape(-1, 1, D)
    full = full[torch.as_tensor(rng.permutation(len(full)))].repeat(1, K, 1).numpy()
    t = torch.as_tensor(np.concatenate([x, full])).to(torch.bfloat16 if dtype == "bf16" else torch.float32).to(DEV)
    t64 = t.cpu().double().numpy()
    announce(f"append special values {dtype}")
    F.focus_paged_append(t, -t, c.dev, i32([0, 0]), i32([0, 48, 560]))
    _check(c, t64, -t64, [0, 0], [0, 48, 560])


def test_append_skips_what_it_cannot_store():
    rng = np.random.default_rng(9)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    K, D, page, block = 2, 64, 16, 8

    def call(lens, add, start, change=None, cu=None, extra=0):
        c = Cache8(rng, [n + a for n, a in zip(lens, add)], K, D, page, block, spare=2)
        (k, k64), (v, v64) = _new(rng, add + [extra], K, D, "bf16")
        c.dev.length.copy_(i32(lens))
        if change:
            change(c)
        err.zero_()
        F.focus_paged_append(k, v, c.dev, i32(start), i32(_offsets(add) if cu is None else cu), err=err)
        return c, k64, v64

    # not served: nothing stored, nothing reported; the others are
    announce("append not served, rows past the last")
    c, k, v = call([5, 6, 7], [4, 30, 9], [5, -1, 7], extra=11)
    _check(c, k, v, [5, -1, 7], [0, 4, 34, 43])
    assert err.item() == 0 and c.dev.length.tolist() == [9, 6, 16]

    # a page outside the pool: its blocks are left out
    announce("append page outside the pool")
    for bad in (-1, 1 << 30):
        def spoil(c):
            c.dev.table[0, 1] = bad
        c, k, v = call([5, 0], [40, 3], [5, 0], spoil)
        keep = [x.copy() for x in (c.pk, c.pv, c.ks, c.vs)]
        p = c.table[0, 1]
        ref = appended(c, k, v, [5, 0], [0, 40, 43])
        for x, y in zip(ref, keep):
            x[p] = y[p]
        c.refresh()
        for got, want in zip((c.pk, c.pv, c.ks, c.vs), ref):
            same(got, want, "others")
        assert err.item() == F.FOCUS_ERR_BOUNDS and c.dev.length.tolist() == [45, 3]
        # the last page: the length ends before it
        err.zero_()
        c.dev.length.zero_()
        c.dev.table[0, 1], c.dev.table[0, 2] = int(p), bad
        (x, _), (y, _) = _new(rng, [43], K, D, "bf16")
        F.focus_paged_append(x, y, c.dev, i32([5, 0]), i32([0, 40, 43]), err=err)
        assert err.item() == F.FOCUS_ERR_BOUNDS and c.dev.length.tolist() == [32, 3]

    # rows past the table
    announce("append past the table")
    c, k, v = call([30, 2], [2, 3], [30, 2])
    err.zero_()
    (x, x64), (y, y64) = _new(rng, [8, 1], K, D, "bf16")
    F.focus_paged_append(x, y, c.dev, i32([28, 2 ** 31 - 1]), i32([0, 8, 9]), err=err)
    c.refresh()
    ref = appended(c, x64[:4], y64[:4], [28, -1], [0, 4, 4])
    F.focus_paged_append(x, y, c.dev, i32([28, 2 ** 31 - 1]), i32([0, 8, 9]), err=err)
    c.refresh()
    for got, want in zip((c.pk, c.pv, c.ks, c.vs), ref):
        same(got, want, "inside")
    assert err.item() == F.FOCUS_ERR_CAPACITY and c.dev.length.tolist() == [32, 5]

    # offsets past the rows are clipped; rows before the first belong to nobody
    announce("append offsets outside the rows")
    c, k, v = call([0, 0], [12, 9], [0, 0], cu=[3, 12, 40])
    _check(c, k, v, [0, 0], [3, 12, 21])
    assert err.item() == F.FOCUS_ERR_BOUNDS
    c, k, v = call([0, 0], [12, 9], [0, 0], cu=[-5, 12, 21])
    _check(c, k, v, [0, 0], [0, 12, 21])
    assert err.item() == F.FOCUS_ERR_BOUNDS
    # offsets that do not ascend: nothing outside the pages, an end
    c, k, v = call([0, 0, 0], [12, 9, 4], [0, 0, 0], cu=[0, 20, 7, 25])
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype,D,block", [("bf16", 128, 64), ("bf16", 128, 128), ("f32", 128, 128), ("bf16", 256, 256)])
def test_append_large_blocks_of_ragged_sequences(dtype, D, block):
    """Parts of several sequences and their blocks follow one another in a workgroup, some with
    infinities and NaN; stored twice, the second time larger, so that first parts are turned."""
    rng = np.random.default_rng(12)
    lens = [int(x) for x in rng.integers(0, 300, 40)]
    announce(f"append large blocks {dtype} {D} {block}")
    parts = [[int(x) if y else 1 for x, y in zip(rng.integers(0, 450, 40), rng.random(40) < 0.5)] for _ in range(2)]
    c = Cache8(rng, [n + a + b for n, a, b in zip(lens, *parts)], 3, D, block, block)
    for i, add in enumerate(parts):
        (k, k64), (v, v64) = _new(rng, add, 3, D, dtype)
        for t, x in ((k, k64), (v, v64)):
            t *= 2.0 ** (8 * i)
            x *= 2.0 ** (8 * i)
            at = tuple(rng.integers(0, n, 30) for n in x.shape)
            bad = rng.choice([np.inf, -np.inf, np.nan], 30)
            x[at] = bad
            t[tuple(torch.as_tensor(j).to(DEV) for j in at)] = torch.as_tensor(x[at], dtype=t.dtype).to(DEV)
        F.focus_paged_append(k, v, c.dev, i32(lens), i32(_offsets(add)))
        _check(c, k64, v64, lens, _offsets(add), f"part {i}")
        lens = [n + a for n, a in zip(lens, add)]
    assert c.dev.length.tolist() == lens


def test_append_nothing():
    rng = np.random.default_rng(10)
    c = Cache8(rng, [5, 9], 2, 64, 16, 8)
    before = [to_codes(x) for x in (c.dev.k, c.dev.v)]
    k = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device=DEV)
    F.focus_paged_append(k, k, c.dev, i32([5, 9]), i32([0, 0, 0]))
    k = torch.ones(7, 2, 64, dtype=torch.bfloat16, device=DEV)
    F.focus_paged_append(k, k, c.dev, i32([5, 9]), i32([0, 0, 0]))
    same(to_codes(c.dev.k), before[0], "k")
    same(to_codes(c.dev.v), before[1], "v")
    assert c.dev.length.tolist() == [5, 9]


def test_append_more_blocks_than_a_launch_has_waves():
    """262 144 rows of 1 024 heads of 16 in blocks of 8: 2^25 of them, one wave each would be more
    threads than a launch may have.  Every head gets the same rows."""
    announce("append 2^25 blocks")
    rows, K, D, page, block = 262_144, 1024, 16, 1024, 8
    pages = rows // page
    rng = np.random.default_rng(11)
    k64 = rng.standard_normal((rows, D)).astype(np.float32)
    k64[:, 0] *= 2.0 ** rng.integers(-8, 9, rows)     # (blocks of different scales)
    k = torch.as_tensor(k64).to(DEV).bfloat16()
    wide = k[:, None, :].expand(rows, K, D)
    pools = [torch.zeros(pages, page, K, D, dtype=torch.float8_e4m3fn, device=DEV) for _ in range(2)]
    scales = [torch.zeros(pages, K, page // block, device=DEV) for _ in range(2)]
    c = F.PagedCache8(*pools, *scales, torch.arange(pages, dtype=torch.int32, device=DEV)[None].flip(1).contiguous(), i32([0]))
    F.focus_paged_append(wide, wide, c, i32([0]), i32([0, rows]))
    # one head by itself, held to the definition elsewhere
    one = F.PagedCache8(*(torch.zeros(pages, page, 1, D, dtype=torch.float8_e4m3fn, device=DEV) for _ in range(2)),
                        *(torch.zeros(pages, 1, page // block, device=DEV) for _ in range(2)), c.table, i32([0]))
    F.focus_paged_append(k[:, None], k[:, None], one, i32([0]), i32([0, rows]))
    assert c.length.item() == one.length.item() == rows
    assert one.k_scale.unique().numel() > 4
    for x, y in ((c.k, one.k), (c.v, one.v)):
        for i in range(0, pages, 32):
            a, b = x.view(torch.uint8)[i:i + 32], y.view(torch.uint8)[i:i + 32]
            assert bool((a == b).all())
    for x, y in ((c.k_scale, one.k_scale), (c.v_scale, one.v_scale)):
        assert bool((x == y).all())
    block0 = k64[:block].astype(np.float64)
    block0 = torch.as_tensor(block0).bfloat16().double().numpy()
    want, scale = O.append(np.zeros((block, D)), np.zeros(1), block, 0, block0)
    assert np.array_equal(to_codes(one.k)[pages - 1, :block, 0], want) and one.k_scale[pages - 1, 0, 0].item() == scale[0]


@pytest.mark.parametrize("batch", [2, 40, 90, 300])
@pytest.mark.parametrize("dtype,D,block", [("bf16", 64, 8), ("f32", 256, 128)])
def test_append_reports_bad_offsets_wherever_they_are(batch, dtype, D, block):
    """Offsets that leave the rows or descend, among others that do neither: reported, and
    nothing written but the pages of the sequences' tables."""
    rng = np.random.default_rng(batch)
    K, page = 2, 128
    add = [int(x) for x in rng.integers(1, 4, batch)]
    n = sum(add)
    fine = _offsets(add)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    announce(f"append bad offsets {batch} {dtype} {D}")
    cases = [(fine, False), (fine[:-1] + [n - 1], False)]
    for at in sorted({1, batch // 2, batch - 1}):
        for value in (n + 1, 2 ** 31 - 1, -1, -2 ** 31, fine[at + 1] + 1, fine[at - 1] - 1):
            cases.append((fine[:at] + [value] + fine[at + 1:], True))
    cases += [(fine[:-1] + [n + 1], True), ([-1] + fine[1:], True), ([fine[1] + 1] + fine[1:], True),
              ([n] + [0] * (batch - 1) + [n], True), ([0] * batch + [-3], True)]
    (k, _), (v, _) = _new(rng, add, K, D, dtype)
    c = Cache8(rng, [page] * batch, K, D, page, block, spare=5)
    outside = torch.as_tensor([p for p in range(c.dev.k.shape[0]) if p not in c.table]).to(DEV)
    keep = [x.view(torch.uint8)[outside].clone() for x in (c.dev.k, c.dev.v, c.dev.k_scale, c.dev.v_scale)]
    for cu, bad in cases:
        err.zero_()
        c.dev.length.zero_()
        F.focus_paged_append(k, v, c.dev, i32([0] * batch), i32(cu), err=err)
        # (a sequence may get more rows by them than its table's one page holds, which is said too)
        most = max(min(y, n) - max(x, 0) for x, y in zip(cu, cu[1:]))
        said = err.item() & ~(F.FOCUS_ERR_CAPACITY if most > page else 0)
        assert said == (F.FOCUS_ERR_BOUNDS if bad else 0), cu[:8]
        for x, y in zip((c.dev.k, c.dev.v, c.dev.k_scale, c.dev.v_scale), keep):
            assert torch.equal(x.view(torch.uint8)[outside], y)
        if not bad:
            assert c.dev.length.tolist() == [y - x for x, y in zip(cu, cu[1:])]
