"""focus_paged_attend on the GPU against the float64 oracle (tolerances:
oracle.paged8.attend_tolerances)."""

import math

import numpy as np
import pytest
import torch

import paper_2511_14694_amd as F
from gpu_util import DEV, announce, to64
from oracle import paged8 as O
from paged8_util import NAN, Cache8, i32
from paged_util import values, within

pytestmark = pytest.mark.gpu


def _check(c, q64, counts, got, dtype, scale=None, visible=None, tol=1.0):
    o, lse = to64(got[0]), to64(got[1])
    D = q64.shape[2]
    sc = D ** -0.5 if scale is None else scale
    at = 0
    for b, (n, m) in enumerate(zip(c.lens, counts)):
        k, v = c.rows(b, n, "k"), c.rows(b, n, "v")
        q = q64[at:at + m]
        seen = np.ones(n, bool) if visible is None else visible[b]
        with np.errstate(invalid="ignore"):
            ro, rl = O.attend(q, k, v, sc, seen)
        to, tl = O.attend_tolerances(q, np.nan_to_num(k[seen]), np.nan_to_num(v[seen]), sc, dtype, np.nan_to_num(ro))
        within(o[at:at + m], ro, to * tol, f"o[{b}]")
        within(lse[at:at + m], rl, tl * tol, f"lse[{b}]")
        at += m


def _offsets(counts):
    return i32(np.concatenate([[0], np.cumsum(counts)]))


CASES = [
    # lens, tokens, H, K, D, page, block, dtype, by_head
    ([1], [1], 1, 1, 64, 8, 8, "f32", False),
    ([1], [1], 32, 8, 128, 64, 16, "bf16", False),
    ([137], [1], 32, 8, 128, 64, 32, "bf16", False),
    ([0, 5, 0], [1, 1, 1], 4, 2, 64, 16, 8, "bf16", False),
    ([31, 32, 33, 7, 8, 9], [1, 2, 3, 1, 0, 2], 6, 2, 128, 8, 8, "bf16", False),
    ([15, 16, 17, 63, 65], [4, 4, 4, 4, 4], 6, 6, 64, 16, 16, "f32", True),
    ([300, 1, 2021], [3, 1, 2], 6, 2, 64, 32, 8, "f32", True),
    ([1000, 129, 127, 128], [5, 5, 5, 5], 8, 8, 128, 128, 64, "bf16", True),
    ([513, 90], [1, 1], 16, 1, 128, 16, 16, "bf16", False),
    ([257, 40], [7, 3], 40, 2, 64, 16, 8, "bf16", False),          # 20 heads of a KV head, 7 tokens: nine tiles
    ([257, 70], [2, 1], 34, 2, 128, 16, 16, "f32", False),
    ([3000], [16], 3, 3, 128, 1024, 256, "bf16", False),
    ([5000, 10, 2500], [1, 4, 2], 8, 2, 128, 64, 16, "bf16", False),
    ([5000, 10, 2500], [2, 2, 2], 4, 4, 128, 16, 8, "f32", False),
    ([3, 2, 9], [3, 5, 12], 2, 1, 64, 8, 8, "bf16", False),         # tokens that see nothing
    ([257, 33], [3, 1], 40, 2, 64, 16, 8, "f32", False),            # two heads a wave, four tiles
    ([700, 5], [9, 2], 8, 8, 64, 32, 32, "bf16", False),            # eight heads a workgroup
    ([700, 5], [2, 1], 5, 5, 64, 32, 32, "bf16", False),            # an odd number of heads of 64
    ([40, 900], [300, 7], 1, 1, 128, 16, 8, "bf16", False),         # more tokens than rows
]


@pytest.mark.parametrize("lens,counts,H,K,D,page,block,dtype,by_head", CASES)
@pytest.mark.parametrize("split", [0, 128, 640])
def test_attend_matches_oracle(lens, counts, H, K, D, page, block, dtype, by_head, split):
    announce(f"attend {lens} {counts} {H}/{K} x {D} page {page} block {block} {dtype} by_head {by_head} split {split}")
    rng = np.random.default_rng(sum(lens) + H + D)
    c = Cache8(rng, lens, K, D, page, block, by_head=by_head, padded=not by_head and D == 64, odd_scales=split == 640)
    q, q64 = values(rng, (sum(counts), H, D), dtype, 1.5)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    cu = None if counts == [1] * len(lens) and split else _offsets(counts)
    got = F.focus_paged_attend(q, c.dev, cu, max_rows=max(counts), split_keys=split, err=err)
    _check(c, q64, counts, got, dtype)
    assert err.item() == 0
    again = F.focus_paged_attend(q, c.dev, cu, max_rows=max(counts), split_keys=split)
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1]), "not deterministic"
    # a greater bound of the tokens changes nothing but the split
    if split and (max(counts) + 3) * H // K <= 512:
        more = F.focus_paged_attend(q, c.dev, cu, max_rows=max(counts) + 3, split_keys=split)
        _check(c, q64, counts, more, dtype)


@pytest.mark.parametrize("batch,top,H,K,dim,dtype,new", [
    (130, 700, 4, 4, 64, "bf16", 2),         # more sequences than a wave has lanes
    (70, 1500, 2, 1, 128, "f32", 1),
    (40, 1100, 8, 8, 128, "bf16", 3),
    (5, 4000, 34, 2, 64, "bf16", 1),         # groups of 17, two KV heads together
    (300, 90, 2, 1, 64, "bf16", 4),
    (3, 9000, 4, 4, 128, "bf16", 8),
    (3, 9000, 32, 8, 128, "bf16", 8),        # 768 columns of many shares
    (16, 4096, 4, 4, 128, "bf16", 1),        # tables long enough for four heads a workgroup
    (17, 4300, 8, 8, 64, "bf16", 1),
    (20, 7000, 8, 4, 128, "f32", 1),
    (17, 3000, 8, 8, 128, "bf16", 2),        # for two
])
def test_attend_chunks_chosen(batch, top, H, K, dim, dtype, new):
    """Lengths from 0 to top in tables long enough to be split, 0 to `new` tokens."""
    announce(f"attend {batch} x {top} {H}/{K} x {dim} {dtype} new {new}")
    rng = np.random.default_rng(batch)
    lens = [top, 0, 1] + [int(x) for x in np.exp(rng.uniform(0, np.log(top), batch - 3))]
    counts = [new] + [int(x) for x in rng.integers(0, new + 1, batch - 1)]
    c = Cache8(rng, lens, K, dim, 64, 16)
    q, q64 = values(rng, (sum(counts), H, dim), dtype)
    got = F.focus_paged_attend(q, c.dev, _offsets(counts), max_rows=new)
    _check(c, q64, counts, got, dtype)


@pytest.mark.parametrize("batch,top,H,K,dim,dtype,new,split", [
    (140, 600, 4, 4, 64, "bf16", 2, 128),
    (140, 700, 2, 1, 128, "f32", 1, 256),
    (150, 600, 40, 1, 128, "bf16", 2, 0),    # 80 columns
    (150, 600, 40, 1, 64, "f32", 1, 128),
    (129, 250, 66, 2, 64, "bf16", 1, 0),     # 33 columns, tables that are not split
    (400, 60, 24, 1, 128, "f32", 1, 0),
    (128, 900, 6, 2, 64, "bf16", 3, 0),      # as many sequences as a wave holds
])
def test_attend_many_sequences(batch, top, H, K, dim, dtype, new, split):
    announce(f"attend {batch} x {top} {H}/{K} x {dim} {dtype} new {new} split {split}")
    rng = np.random.default_rng(batch + H)
    lens = [0, top, 1, 0] + [int(x) for x in rng.integers(0, top + 1, batch - 5)] + [0]
    counts = [int(x) for x in rng.integers(0, new + 1, batch)]
    counts[1] = counts[-1] = new
    c = Cache8(rng, lens, K, dim, 32, 8)
    q, q64 = values(rng, (sum(counts), H, dim), dtype)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = F.focus_paged_attend(q, c.dev, _offsets(counts), max_rows=new, split_keys=split, err=err)
    _check(c, q64, counts, got, dtype)
    assert err.item() == 0


def test_attend_table_far_larger_than_the_lengths():
    rng = np.random.default_rng(31)
    lens = [0, 1, 700, 33]
    c = Cache8(rng, lens, 2, 128, 64, 32, max_pages=1024)
    q, q64 = values(rng, (4, 8, 128), "bf16")
    announce("attend wide table")
    _check(c, q64, [1] * 4, F.focus_paged_attend(q, c.dev), "bf16")


def test_attend_chunk_of_more_pages_than_held():
    """Chunks over more pages than a workgroup holds at a time."""
    rng = np.random.default_rng(32)
    c = Cache8(rng, [20_003], 1, 64, 8, 8)
    q, q64 = values(rng, (3, 2, 64), "bf16")
    announce("attend many pages")
    _check(c, q64, [3], F.focus_paged_attend(q, c.dev, _offsets([3]), max_rows=3, split_keys=128 * 80), "bf16")


def test_attend_a_long_sequence_beside_a_short_one():
    rng = np.random.default_rng(38)
    c = Cache8(rng, [262_144, 3], 1, 64, 128, 64)
    q, q64 = values(rng, (5, 4, 64), "bf16")
    announce("attend 262144 rows")
    _check(c, q64, [3, 2], F.focus_paged_attend(q, c.dev, _offsets([3, 2]), max_rows=3), "bf16")


def test_attend_and_append_in_a_pool_past_32_bits():
    """Pages at the end of pools of 4.6 GB give the bits that they give in a small one."""
    page, K, D, block, pages = 64, 8, 128, 16, 70_000
    rng = np.random.default_rng(39)
    lens = [500, 64, 1]
    (k, _), (v, _), (q, _) = (values(rng, (sum(lens), n, D), "bf16") for n in (K, K, 4 * K))
    cu = _offsets(lens)
    got = []
    announce("attend and append past 32 bits")
    for total in (16, pages):
        pools = [torch.empty(total, page, K, D, dtype=torch.uint8, device=DEV) for _ in range(2)]
        for x in pools:
            x[-16:] = 0x7f
        scales = [torch.full((total, K, page // block), float("nan"), device=DEV) for _ in range(2)]
        table = torch.full((3, 8), -1, dtype=torch.int32, device=DEV)
        table[0], table[1, 0], table[2, 0] = torch.arange(total - 8, total, device=DEV), total - 9, total - 16
        c = F.PagedCache8(*(x.view(torch.float8_e4m3fn) for x in pools), *scales, table, i32([0, 0, 0]))
        F.focus_paged_append(k, v, c, i32([0, 0, 0]), cu)
        o, lse = F.focus_paged_attend(q[:5], c, _offsets([2, 2, 1]), max_rows=2)
        got.append([o, lse, c.length] + [x[-16:].clone() for x in (*pools, *(y.view(torch.int32) for y in scales))])
    assert pools[0].numel() > 2 ** 32 and torch.isfinite(got[0][0].float()).all()
    for x, y in zip(*got):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_strided_queries_scale_and_outputs(dtype):
    rng = np.random.default_rng(33)
    H, K, D = 6, 3, 64
    c = Cache8(rng, [90, 300], K, D, 16, 8)
    qkv, qkv64 = values(rng, (5, H + 2 * K, D), dtype)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    o = torch.full((5, H, D), 7.0, dtype=t, device=DEV)
    lse = torch.full((5, H), 7.0, device=DEV)
    announce(f"attend strided {dtype}")
    # 2 + 2 rows: the fifth belongs to nobody and is left as it was
    F.focus_paged_attend(qkv[:, :H], c.dev, _offsets([2, 2]), max_rows=2, o=o, lse=lse, softmax_scale=0.3)
    _check(c, qkv64[:, :H], [2, 2], (o, lse), dtype, scale=0.3)
    assert (o[4] == 7).all() and (lse[4] == 7).all()
    # rows before the first offset too, and heads before rows
    o.fill_(7.0)
    q2 = qkv[:, :H].transpose(0, 1).contiguous().transpose(0, 1)
    F.focus_paged_attend(q2, c.dev, i32([1, 3, 5]), max_rows=2, o=o, want_lse=False, softmax_scale=0.3)
    _check(c, qkv64[1:, :H], [2, 2], (o[1:], F.focus_paged_attend(q2, c.dev, i32([1, 3, 5]), 2, softmax_scale=0.3)[1][1:]),
           dtype, scale=0.3)
    assert (o[0] == 7).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("split", [0, 128])
def test_attend_nan_only_where_it_is_seen(D, split):
    """A NaN in a row's k, v or scales reaches the tokens that see it, not those before."""
    rng = np.random.default_rng(34)
    announce(f"attend NaN {D} {split}")
    for n in (40, 300, 1027):
        for which in ("k", "v", "k_scale", "v_scale"):
            c = Cache8(rng, [n], 2, D, 16, 8)
            row = n - 2                                   # seen by the last two tokens of four
            p, r = c.table[0][row // 16], row % 16
            if "scale" in which:
                row = n - 1 - (n - 1) % 8
                if row <= n - 4:
                    continue                              # every token sees the block
                p, r = c.table[0][row // 16], row % 16
                getattr(c.dev, which)[p, 0, r // 8] = float("nan")
            else:
                getattr(c.dev, which).view(torch.uint8)[p, r, 0, 5] = NAN
            q, q64 = values(rng, (4, 4, D), "bf16")
            c.refresh()
            o, lse = F.focus_paged_attend(q, c.dev, i32([0, 4]), max_rows=4, split_keys=split)
            first = next(i for i in range(4) if n - 3 + i > row)
            k, v = c.rows(0, n, "k"), c.rows(0, n, "v")
            for i in range(4):
                upto = n - 3 + i
                o_i, lse_i = to64(o[i]), to64(lse[i])
                if i < first:
                    ro, rl = O.attend(q64[i:i + 1], k[:upto], v[:upto])
                    to, tl = O.attend_tolerances(q64[i:i + 1], k[:upto], v[:upto], D ** -0.5, "bf16", ro)
                    within(o_i, ro[0], to[0], f"{which} token {i}")
                    within(lse_i, rl[0], tl[0], f"{which} token {i}")
                else:
                    spoiled = o_i[:2] if "k" in which or "scale" in which else o_i[:2, 5]
                    assert np.isnan(spoiled).all(), (which, i)
                    fine = o_i[2:] if "k" in which or "scale" in which else np.delete(o_i, 5, 1)
                    assert np.isfinite(fine).all() and np.isfinite(o_i[2:]).all(), (which, i)


def test_attend_scales_of_all_sizes():
    """Scales from the least to great ones: scores of some thousands, weights that leave one
    row, values near the end of float32."""
    rng = np.random.default_rng(35)
    c = Cache8(rng, [200], 2, 128, 16, 8)
    c.dev.k_scale.copy_(torch.as_tensor(2.0 ** rng.integers(-126, 0, tuple(c.dev.k_scale.shape))))
    c.dev.v_scale.copy_(torch.as_tensor(2.0 ** rng.integers(-100, 110, tuple(c.dev.v_scale.shape))))
    c.refresh()
    q, q64 = values(rng, (1, 4, 128), "f32")
    announce("attend scales")
    _check(c, q64, [1], F.focus_paged_attend(q, c.dev), "f32")
    c.dev.k_scale.zero_()
    c.dev.v_scale.zero_()
    o, lse = F.focus_paged_attend(q, c.dev)
    assert (o == 0).all() and (lse - math.log(200)).abs().max() < 1e-6


def test_attend_great_queries():
    """The greatest queries whose products with any e4m3 row are float32 numbers, against keys of
    the least scales."""
    rng = np.random.default_rng(37)
    announce("attend great queries")
    for D in (64, 128):
        c = Cache8(rng, [70], 2, D, 16, 8)
        c.dev.k_scale.copy_(torch.as_tensor(2.0 ** rng.integers(-126, -124, tuple(c.dev.k_scale.shape))))
        c.refresh()
        q, q64 = values(rng, (1, 4, D), "f32")
        most = 2.0 ** 111 * (1 - 2.0 ** -24)
        q = (q * 2.0 ** 109).clamp(-most, most)
        q64 = to64(q)
        _check(c, q64, [1], F.focus_paged_attend(q, c.dev, softmax_scale=0.5), "f32", scale=0.5)


def test_attend_pages_outside_the_pool_and_bad_offsets():
    rng = np.random.default_rng(36)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    announce("attend pages outside the pool")
    for split in (0, 128):
        c = Cache8(rng, [600, 40, 20], 2, 64, 16, 8)
        for j, bad in ((2, -1), (3, -2 ** 31), (20, 10 ** 6), (37, 2 ** 31 - 1)):
            c.dev.table[0, j] = bad
        c.dev.table[2, :2] = -1
        seen = [np.ones(600, bool), np.ones(40, bool), np.zeros(20, bool)]
        for j in (2, 3, 20, 37):
            seen[0][16 * j:16 * j + 16] = False
        q, q64 = values(rng, (5, 2, 64), "bf16")
        err.zero_()
        got = F.focus_paged_attend(q, c.dev, i32([0, 2, 4, 5]), max_rows=2, split_keys=split, err=err)
        _check(c, q64, [2, 2, 1], got, "bf16", visible=seen)
        assert err.item() == F.FOCUS_ERR_BOUNDS
    announce("attend lengths outside the table")
    c = Cache8(rng, [32, 16], 2, 64, 16, 8)
    q, q64 = values(rng, (2, 2, 64), "bf16")
    c.dev.length.copy_(i32([99, -4]))
    err.zero_()
    got = F.focus_paged_attend(q, c.dev, err=err)
    c.lens = [32, 0]
    _check(c, q64, [1, 1], got, "bf16")
    assert err.item() == F.FOCUS_ERR_CAPACITY
    announce("attend bad offsets")
    c = Cache8(rng, [32, 300, 40], 2, 64, 16, 8)
    q, q64 = values(rng, (6, 2, 64), "bf16")
    for cu, bit, fine in (([0, 3, 4, 6], F.FOCUS_ERR_CAPACITY, [(1, 3, 4), (2, 4, 6)]),
                          ([4, 2, 3, 5], F.FOCUS_ERR_BOUNDS, [(1, 2, 3), (2, 3, 5)]),
                          ([-1, 1, 2, 9], F.FOCUS_ERR_BOUNDS, [(1, 1, 2)])):
        o, lse = torch.full_like(q, 7.0), torch.full((6, 2), 7.0, device=DEV)
        err.zero_()
        F.focus_paged_attend(q, c.dev, i32(cu), max_rows=2, o=o, lse=lse, err=err)
        assert err.item() == bit
        mine = set()
        for b, r0, r1 in fine:
            one = Cache8.__new__(Cache8)
            one.__dict__.update(c.__dict__, lens=[c.lens[b]], table=c.table[b:b + 1])
            _check(one, q64[r0:r1], [r1 - r0], (o[r0:r1], lse[r0:r1]), "bf16")
            mine |= set(range(r0, r1))
        for t in set(range(6)) - mine:
            assert (o[t] == 7).all() and (lse[t] == 7).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_split_keys_fix_a_sequences_bits(D, dtype):
    """With a given split a sequence's result depends neither on the rest of the batch nor on
    how wide its table is: 127 shares, in tables of 127 and 128 and with sixteen others."""
    rng = np.random.default_rng(40)
    c = Cache8(rng, [127 * 128] + [900, 40, 0, 128] * 4, 2, D, 64, 16, max_pages=256)
    q, q64 = values(rng, (17, 32, D), dtype)
    announce(f"attend given split {D} {dtype}")
    o, lse = F.focus_paged_attend(q, c.dev, split_keys=128)
    _check(c, q64, [1] * 17, (o, lse), dtype)
    for n in (1, 2, 5, 17):
        for width in (254, 256):
            part = F.PagedCache8(c.dev.k, c.dev.v, c.dev.k_scale, c.dev.v_scale, c.dev.table[:n, :width].contiguous(),
                                 c.dev.length[:n])
            o1, l1 = F.focus_paged_attend(q[:n], part, split_keys=128)
            assert torch.equal(o1, o[:n]) and torch.equal(l1, lse[:n]), (n, width)


@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (128, "f32"), (64, "f32")])
def test_attend_split_keys_fix_bits_of_many_shares(D, dtype):
    """The same of sequences of 127, 128 and 150 shares, which are joined in two ways, and of
    shorter ones beside them."""
    rng = np.random.default_rng(44)
    c = Cache8(rng, [127 * 128, 128 * 128, 150 * 128 - 77, 127 * 128 + 1, 300, 1, 0] + [200] * 10, 1, D, 64, 16, max_pages=400)
    q, q64 = values(rng, (17, 32, D), dtype)
    announce(f"attend given split, many shares {D} {dtype}")
    o, lse = F.focus_paged_attend(q, c.dev, split_keys=128)
    _check(c, q64, [1] * 17, (o, lse), dtype)
    for part, width in ((slice(0, 1), 254), (slice(1, 2), 256), (slice(2, 3), 300), (slice(3, 4), 255), (slice(0, 4), 400),
                        (slice(2, 7), 300)):
        one = F.PagedCache8(c.dev.k, c.dev.v, c.dev.k_scale, c.dev.v_scale, c.dev.table[part, :width].contiguous(),
                            c.dev.length[part])
        o1, l1 = F.focus_paged_attend(q[part], one, split_keys=128)
        assert torch.equal(o1, o[part]) and torch.equal(l1, lse[part]), (part, width)


@pytest.mark.parametrize("K", [1, 2, 4, 6, 8])
@pytest.mark.parametrize("D,dtype,by_head", [(64, "bf16", False), (64, "bf16", True), (128, "bf16", False), (64, "f32", False),
                                             (128, "f32", False)])
def test_attend_split_keys_fix_bits_whatever_max_rows(K, D, dtype, by_head):
    """Nor on how many tokens another sequence of the batch may have."""
    rng = np.random.default_rng(42)
    c = Cache8(rng, [1000, 300, 50], K, D, 32, 16, by_head=by_head)
    q, q64 = values(rng, (3, 8 * K, D), dtype)
    announce(f"attend given split, max_rows {K} x {D} {dtype} by_head {by_head}")
    o, lse = F.focus_paged_attend(q, c.dev, split_keys=256)
    _check(c, q64, [1] * 3, (o, lse), dtype)
    for most in (2, 3, 5, 9, 33):
        o1, l1 = F.focus_paged_attend(q, c.dev, i32([0, 1, 2, 3]), max_rows=most, split_keys=256)
        assert torch.equal(o1, o) and torch.equal(l1, lse), most


@pytest.mark.parametrize("H,K,D,dtype,by_head", [
    (12, 2, 128, "bf16", False),     # two tiles of columns
    (10, 2, 64, "bf16", False),
    (12, 2, 64, "bf16", True),
    (80, 4, 128, "bf16", False),     # tiles of several workgroups
    (34, 2, 64, "bf16", False),
    (4, 2, 64, "bf16", False),       # two heads a wave
    (4, 2, 64, "f32", False),        # queries in three parts
    (3, 3, 128, "f32", False),
    (40, 2, 128, "f32", False),
    (40, 2, 64, "f32", False),
])
@pytest.mark.parametrize("split", [0, 128])
def test_attend_nan_only_where_it_is_seen_by_every_form(H, K, D, dtype, by_head, split):
    """NaN in the last rows' k and v: which elements of which tokens and heads become NaN is
    the oracle's, all others hold their tolerances."""
    rng = np.random.default_rng(H + K + D)
    announce(f"attend NaN {H}/{K} x {D} {dtype} by_head {by_head} split {split}")
    for lens in ([40, 31, 4], [300, 7, 1027]):
        c = Cache8(rng, lens, K, D, 16, 8, by_head=by_head)
        for b, n in enumerate(lens):
            for row, which, g, e in ((n - 1, "v", 0, [3, D - 1]), (n - 2, "v", K - 1, [D // 2, D // 2 + 7, 0]),
                                     (n - 3, "v", 0, [17]), (n - 1, "k", K - 1, [5])):
                p, r = c.table[b][row // 16], row % 16
                for x in e:
                    getattr(c.dev, which).view(torch.uint8)[p, r, g, x] = NAN if x % 2 else 0xff
        c.refresh()
        q, q64 = values(rng, (12, H, D), dtype)
        got = F.focus_paged_attend(q, c.dev, i32([0, 4, 8, 12]), max_rows=4, split_keys=split)
        bad = np.isnan(to64(got[0]))
        assert bad.any() and not bad[::4].any() and not bad.all(2).all()
        _check(c, q64, [4, 4, 4], got, dtype)


@pytest.mark.parametrize("H,K,D,dtype", [(4, 2, 64, "bf16"), (12, 2, 128, "bf16"), (4, 2, 64, "f32"), (3, 3, 128, "f32")])
@pytest.mark.parametrize("split", [0, 128])
def test_attend_values_over_the_whole_of_float32(H, K, D, dtype, split):
    """Values from the greatest numbers to the smallest: their weighted mean is a number that
    float32 has, whatever the sums of the weights are.  Compared with the scale taken off.

    For the least scales: a weight times the scale and a power of two, more than a quarter of one
    over the table's rows, enters in bf16 parts, whose least step is 2^-133: off by 2^-134, so o by
    that times 4 rows, 448 n and one over the weights' sum; an output below 2^-126 is rounded
    by half of 2^-133, or 2^-149, more."""
    announce(f"attend values {H}/{K} x {D} {dtype} split {split}")
    for p in (119, 118, 100, 64, 33, 32, 31, -31, -32, -33, -64, -90, -100, -110, -117, -126):
        rng = np.random.default_rng(41)
        c = Cache8(rng, [1500, 40, 3], K, D, 16, 8)
        c.dev.v_scale.fill_(2.0 ** p)
        if p == 119:
            c.dev.v.view(torch.uint8)[:] = c.dev.v.view(torch.uint8) & 0x7f       # all of one sign
        c.refresh()
        c.vs = np.ones_like(c.vs)
        q, q64 = values(rng, (5, H, D), dtype, 0.1)
        o, lse = F.focus_paged_attend(q, c.dev, i32([0, 2, 4, 5]), max_rows=2, split_keys=split)
        sc, at = D ** -0.5, 0
        for b, (n, m) in enumerate(zip(c.lens, (2, 2, 1))):
            k, v = c.rows(b, n, "k"), c.rows(b, n, "v")
            ro, rl = O.attend(q64[at:at + m], k, v, sc)
            to, tl = O.attend_tolerances(q64[at:at + m], k, v, sc, dtype, ro)
            least = 0.0
            if p < -80:
                group = H // K
                top = sc * np.stack([(q64[at:at + m, h] @ k[:, h // group].T).max(1) for h in range(H)], 1)
                least = 2.0 ** ((-134 if dtype == "bf16" else -150) - p)
                least = least + 2.0 ** (-134 - p) * 4 * c.max_pages * 16 * 448 * n / np.exp(rl - top)[..., None]
            within(to64(o)[at:at + m] * 2.0 ** -p, ro, to + least, f"2^{p} o[{b}]")
            within(to64(lse)[at:at + m], rl, tl, f"2^{p} lse[{b}]")
            at += m


@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (128, "bf16"), (64, "f32"), (128, "f32")])
@pytest.mark.parametrize("split", [0, 128])
def test_attend_values_that_grow_along_a_sequence(D, dtype, split):
    """Blocks of ever greater scales, over all that there are and over parts; of the greatest
    several, whose sum float32 does not have; and the same from the end on."""
    announce(f"attend growing values {D} {dtype} split {split}")
    for n, lo, hi in ((1500, -126, 119), (1500, -40, -20), (1500, 20, 40), (1500, -10, 10), (250, -126, 119), (30, -70, 70)):
        for back in (False, True):
            rng = np.random.default_rng(abs(n + lo))
            c = Cache8(rng, [n], 2, D, 16, 8)
            e = np.sort(rng.integers(lo, hi + 1, -(-n // 8)))
            e[-8:] = hi
            e = e[::-1] if back else e
            s = c.dev.v_scale
            for j, x in enumerate(e):
                s[int(c.table[0][j // 2]), :, j % 2] = 2.0 ** float(x)
            c.dev.v.view(torch.uint8)[:] = c.dev.v.view(torch.uint8) & 0x7f
            c.refresh()
            q, q64 = values(rng, (2, 4, D), dtype, 0.1)
            _check(c, q64, [2], F.focus_paged_attend(q, c.dev, i32([0, 2]), max_rows=2, split_keys=split), dtype)


@pytest.mark.parametrize("H,K,D,dtype", [(4, 2, 64, "bf16"), (12, 2, 128, "bf16"), (34, 2, 64, "bf16"), (4, 2, 64, "f32"),
                                         (3, 3, 128, "f32")])
@pytest.mark.parametrize("split", [0, 128])
def test_attend_great_values_reach_only_who_sees_them(H, K, D, dtype, split):
    """A last block of the greatest values, in one KV head and one sequence of three: tokens and
    heads that do not see it keep their bits, the others' outputs are theirs; NaN stay NaN."""
    rng = np.random.default_rng(43)
    announce(f"attend great values seen {H}/{K} x {D} {dtype} split {split}")
    for lens in ([41, 5, 16], [1025, 700, 9]):
        c = Cache8(rng, lens, K, D, 16, 8)
        q, q64 = values(rng, (6, H, D), dtype, 0.1)
        cu = i32([0, 2, 4, 6])
        before = F.focus_paged_attend(q, c.dev, cu, max_rows=2, split_keys=split)
        n = lens[0]
        p = int(c.table[0][(n - 1) // 16])
        c.dev.v_scale[p, K - 1, (n - 1) % 16 // 8] = 2.0 ** 119
        c.refresh()
        o, lse = F.focus_paged_attend(q, c.dev, cu, max_rows=2, split_keys=split)
        _check(c, q64, [2, 2, 2], (o, lse), dtype)
        same = torch.ones(6, H, dtype=torch.bool, device=DEV)
        same[1, H - H // K:] = False
        assert torch.equal(o[same], before[0][same]) and torch.equal(lse[same], before[1][same])
        c.dev.v.view(torch.uint8)[p, (n - 1) % 16, K - 1, 7] = NAN
        c.refresh()
        _check(c, q64, [2, 2, 2], F.focus_paged_attend(q, c.dev, cu, max_rows=2, split_keys=split), dtype)
