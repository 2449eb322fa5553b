"""focus_paged_decode on the GPU against the float64 oracle (tolerances:
paged_util.decode_tolerances)."""

import numpy as np
import pytest
import torch

import paper_2511_14694_amd as F
from gpu_util import DEV, announce, to64
from oracle import paged as P
from paged_util import HALF_STEP, Cache, decode_tolerances, values, within

pytestmark = pytest.mark.gpu


def _check(c, q64, got, dtype, scale=None, visible=None, weight=None, decay=None):
    """got (o, lse) and the cache's weights against the oracle, sequence by sequence."""
    o, lse = to64(got[0]), to64(got[1])
    w = None if weight is None else c.dev.weight.cpu().numpy().astype(np.float64)
    H, D = q64.shape[1:]
    K = c.dev.k.shape[2]
    sc = D ** -0.5 if scale is None else scale
    for b, n in enumerate(c.lens):
        seen = np.ones(n, bool) if visible is None else visible[b]
        ro, rl, rw = P.decode(q64[b], c.k[b], c.v[b], sc, seen)
        to, tl, rel = decode_tolerances(q64[b], c.k[b][seen], sc, dtype, c.v[b][seen], ro)
        within(o[b], ro, to, f"o[{b}]")
        within(lse[b], rl, tl, f"lse[{b}]")
        if w is not None:
            old = decay * weight[b].astype(np.float64) if decay else np.zeros_like(weight[b], np.float64)
            ref = old.copy()
            ref[:, :n] += rw
            ref[:, n:] = weight[b][:, n:]
            tol = np.zeros_like(ref)
            grow = rel.reshape(K, H // K).max(1)[:, None] + 2.0 ** -21 + (H // K) * 2.0 ** -24
            tol[:, :n] = rw * grow + np.abs(ref[:, :n]) * 2.0 ** -23 + 1e-30
            within(w[b], ref, tol, f"weight[{b}]")


@pytest.mark.parametrize("lens,H,K,D,page,dtype,by_head", [
    ([1], 1, 1, 64, 8, "f32", False),
    ([1], 32, 8, 128, 64, "bf16", False),
    ([137], 32, 8, 128, 64, "bf16", False),
    ([0, 5, 0], 4, 2, 64, 16, "bf16", False),
    ([31, 32, 33, 7, 8, 9], 6, 2, 128, 8, "bf16", False),
    ([15, 16, 17, 63, 65], 6, 6, 64, 16, "f32", True),
    ([300, 1, 2021], 6, 2, 64, 32, "f32", True),
    ([1000, 129, 127, 128], 8, 8, 128, 128, "bf16", True),
    ([513, 90], 16, 1, 128, 16, "bf16", False),      # a group of 16
    ([257], 40, 2, 64, 16, "bf16", False),           # groups of 20: more than one tile
    ([257, 70], 34, 2, 128, 16, "f32", False),       # groups of 17
    ([3000], 3, 3, 128, 1024, "bf16", False),
    ([5000, 10, 2500], 8, 2, 128, 64, "bf16", False),
    ([5000, 10, 2500], 4, 4, 128, 16, "f32", False),
])
@pytest.mark.parametrize("split", [0, 128, 640])
def test_decode_matches_oracle(lens, H, K, D, page, dtype, by_head, split):
    announce(f"paged decode {lens} {H}/{K} x {D} page {page} {dtype} by_head {by_head} split {split}")
    rng = np.random.default_rng(sum(lens) + H + D)
    c = Cache(rng, lens, K, D, page, dtype, by_head=by_head, padded=not by_head and D == 64, weight=True)
    q, q64 = values(rng, (len(lens), H, D), dtype, 1.5)
    got = F.focus_paged_decode(q, c.dev, split_keys=split)
    _check(c, q64, got, dtype)
    assert np.array_equal(c.dev.weight.cpu().numpy(), c.weight), "weights without weight_decay"
    again = F.focus_paged_decode(q, c.dev, split_keys=split, weight_decay=0.875)
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1]), "not deterministic"
    _check(c, q64, again, dtype, weight=c.weight, decay=0.875)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_table_far_larger_than_the_lengths(dtype):
    """Capacity of 65 536 rows a sequence, lengths from none to a few hundred."""
    rng = np.random.default_rng(31)
    lens = [0, 1, 700, 33]
    c = Cache(rng, lens, 2, 128, 64, dtype, max_pages=1024, weight=True)
    q, q64 = values(rng, (4, 8, 128), dtype)
    announce(f"paged decode wide table {dtype}")
    got = F.focus_paged_decode(q, c.dev, weight_decay=0.0)
    _check(c, q64, got, dtype, weight=c.weight, decay=0.0)


def test_decode_many_sequences():
    rng = np.random.default_rng(32)
    lens = [int(x) for x in rng.integers(0, 90, 300)]
    c = Cache(rng, lens, 1, 64, 16, "bf16", weight=True)
    q, q64 = values(rng, (300, 2, 64), "bf16")
    announce("paged decode 300 sequences")
    _check(c, q64, F.focus_paged_decode(q, c.dev, weight_decay=1.0), "bf16", weight=c.weight, decay=1.0)


@pytest.mark.parametrize("batch,top,H,K,dim,dtype,by_head", [
    (130, 700, 4, 4, 64, "bf16", False),     # more sequences than a wave has lanes
    (70, 1500, 2, 1, 128, "f32", False),
    (40, 1100, 8, 8, 128, "bf16", True),     # chunks that would not all be resident: larger ones
    (5, 4000, 34, 2, 64, "bf16", False),     # groups of 17, two KV heads together
    (3, 9000, 4, 4, 128, "bf16", False),
])
def test_decode_chunks_chosen(batch, top, H, K, dim, dtype, by_head):
    """Lengths from 0 to top in tables long enough to be split: every way a chunk's size
    is chosen, with weights and without."""
    announce(f"paged decode {batch} x {top} {H}/{K} x {dim} {dtype} by_head {by_head}")
    rng = np.random.default_rng(batch)
    lens = [top, 0, 1] + [int(x) for x in (rng.integers(top * 9 // 10, top, batch - 3) if by_head else
                                           np.exp(rng.uniform(0, np.log(top), batch - 3)))]
    c = Cache(rng, lens, K, dim, 64, dtype, by_head=by_head, weight=True)
    q, q64 = values(rng, (batch, H, dim), dtype)
    got = F.focus_paged_decode(q, c.dev)
    _check(c, q64, got, dtype)
    again = F.focus_paged_decode(q, c.dev, weight_decay=1.0)
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
    _check(c, q64, again, dtype, weight=c.weight, decay=1.0)


@pytest.mark.parametrize("batch,top,H,K,dim,dtype", [
    (128, 600, 4, 2, 64, "f32"),         # as many as one wave counts
    (129, 2000, 8, 1, 128, "bf16"),
    (1300, 700, 2, 2, 64, "bf16"),       # more than one workgroup's threads
])
@pytest.mark.parametrize("split", [0, 256])
def test_decode_chunks_of_many_sequences(batch, top, H, K, dim, dtype, split):
    """A few long sequences among many short or empty ones, the longest first and last."""
    announce(f"paged decode {batch} x {top} {H}/{K} x {dim} {dtype} split {split}")
    rng = np.random.default_rng(batch + split)
    lens = [int(x) for x in np.where(rng.random(batch) < 0.05, rng.integers(0, top, batch), rng.integers(0, 40, batch))]
    lens[0] = lens[-1] = top
    c = Cache(rng, lens, K, dim, 32, dtype, weight=True)
    q, q64 = values(rng, (batch, H, dim), dtype)
    got = F.focus_paged_decode(q, c.dev, split_keys=split)
    _check(c, q64, got, dtype)
    again = F.focus_paged_decode(q, c.dev, split_keys=split, weight_decay=0.5)
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
    _check(c, q64, again, dtype, weight=c.weight, decay=0.5)


@pytest.mark.parametrize("H,K,lens", [(260, 1, [900, 3]), (512, 1, [130]), (27, 3, [2000, 300, 0])])
def test_decode_large_groups(H, K, lens):
    """More heads of a KV head than one workgroup or one wave of the second launch has
    threads for, and groups that its steps do not divide; with weights."""
    announce(f"paged decode {H}/{K} {lens}")
    rng = np.random.default_rng(H)
    c = Cache(rng, lens, K, 64, 16, "bf16", weight=True)
    q, q64 = values(rng, (len(lens), H, 64), "bf16")
    got = F.focus_paged_decode(q, c.dev, split_keys=128)
    _check(c, q64, got, "bf16")
    again = F.focus_paged_decode(q, c.dev, split_keys=128, weight_decay=0.75)
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
    _check(c, q64, again, "bf16", weight=c.weight, decay=0.75)


@pytest.mark.parametrize("batch,top,H,K,dtype", [(140, 900, 20, 1, "bf16"), (5, 200, 99, 3, "f32"), (9, 3000, 36, 2, "f32")])
def test_decode_rows_shared_by_workgroups(batch, top, H, K, dtype):
    """Groups of more than 16 heads in tables that are split, not split, and divided by a
    launch of their own."""
    announce(f"paged decode shared rows {batch} x {top} {H}/{K} {dtype}")
    rng = np.random.default_rng(batch + H)
    lens = [top, 0] + [int(x) for x in rng.integers(0, top + 1, batch - 2)]
    c = Cache(rng, lens, K, 64, 32, dtype, weight=True)
    q, q64 = values(rng, (batch, H, 64), dtype)
    got = F.focus_paged_decode(q, c.dev)
    _check(c, q64, got, dtype)
    again = F.focus_paged_decode(q, c.dev, weight_decay=0.5)
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
    _check(c, q64, again, dtype, weight=c.weight, decay=0.5)


@pytest.mark.parametrize("rows", [50, 5000])
def test_decode_scores_far_below_zero(rows):
    """Scores of -1e31 and less are scores: the highest takes all the weight, alone in its
    chunk or not (each differs from the next by more than 1e30)."""
    rng = np.random.default_rng(41)
    c = Cache(rng, [rows], 1, 64, 64, "f32", weight=True)
    q = torch.full((1, 2, 64), 1e15, device=DEV)
    best = rows * 2 // 3
    order = np.arange(1, rows + 1) + np.where(np.arange(rows) == best, -rows, rows)
    for r in range(rows):
        c.k[0][r, 0] = -2e15 * max(int(order[r]), 1)
    k = torch.as_tensor(c.k[0][:, 0, 0].astype(np.float32)).to(DEV)
    where = torch.as_tensor(c.table[0][np.arange(rows) // 64].astype(np.int64)).to(DEV)
    c.dev.k[where, torch.arange(rows, device=DEV) % 64, 0] = k[:, None].expand(rows, 64)
    o, lse = F.focus_paged_decode(q, c.dev, weight_decay=0.0)
    assert np.array_equal(to64(o)[0], np.broadcast_to(c.v[0][best], (2, 64)))
    top = float(k[best]) * 1e15 * 8
    within(to64(lse)[0], np.full(2, top), abs(top) * 80 * 2.0 ** -24, "lse")
    w = c.dev.weight.cpu().numpy()[0, 0, :rows]
    assert w[best] == 2 and np.count_nonzero(w) == 1


def test_decode_split_keys_fix_a_sequences_bits():
    """With a given split a sequence's result does not depend on the rest of the batch."""
    rng = np.random.default_rng(40)
    c = Cache(rng, [3000, 900, 40], 2, 128, 32, "bf16")
    q, _ = values(rng, (3, 8, 128), "bf16")
    o, lse = F.focus_paged_decode(q, c.dev, split_keys=256)
    for b in range(3):
        one = F.PagedCache(c.dev.k, c.dev.v, c.dev.table[b:b + 1], c.dev.length[b:b + 1])
        o1, l1 = F.focus_paged_decode(q[b:b + 1], one, split_keys=256)
        assert torch.equal(o1[0], o[b]) and torch.equal(l1[0], lse[b])


def test_decode_sharp_scores_scale_and_views():
    """Scores of several hundred, a given scale, q as a view of a projection, outputs
    given; old weights that are not numbers count only where they are read."""
    rng = np.random.default_rng(33)
    c = Cache(rng, [400, 77], 2, 128, 32, "bf16", weight=True)
    qkv, x = values(rng, (2, 12, 128), "bf16", 6.0)
    q, q64 = qkv[:, 2:10], x[:, 2:10]
    c.dev.weight.fill_(float("nan"))
    o, lse = torch.empty(2, 8, 128, dtype=torch.bfloat16, device=DEV), torch.empty(2, 8, device=DEV)
    got = F.focus_paged_decode(q, c.dev, o=o, lse=lse, softmax_scale=0.5, weight_decay=0.0)
    assert got[0] is o and got[1] is lse
    nan = np.full_like(c.weight, np.nan)
    _check(c, q64, got, "bf16", scale=0.5, weight=nan, decay=0.0)
    o2, none = F.focus_paged_decode(q, c.dev, softmax_scale=0.5, want_lse=False)
    assert none is None and torch.equal(o2, o)


def test_decode_infinities_stay_in_their_column():
    """V of visible rows: an infinity or NaN reaches its column only; rows past the
    length and masked rows nothing (they hold NaN throughout these tests)."""
    rng = np.random.default_rng(34)
    for dtype in ("bf16", "f32"):
        c = Cache(rng, [45], 1, 64, 16, dtype)
        q, q64 = values(rng, (1, 4, 64), dtype)
        clean = F.focus_paged_decode(q, c.dev)[0]
        page, row = int(c.table[0, 2]), 7
        c.dev.v[page, row, 0, 5] = float("inf")
        c.dev.v[page, row, 0, 9] = float("nan")
        got = F.focus_paged_decode(q, c.dev)[0]
        assert torch.isposinf(got[..., 5]).all() and torch.isnan(got[..., 9]).all()
        got[..., 5], got[..., 9] = clean[..., 5], clean[..., 9]
        assert torch.equal(got, clean)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("accumulate", [False, True])
def test_decode_bad_pages_and_lengths(dtype, accumulate):
    """Rows of pages outside the pool are left out; a length past the table is clipped."""
    announce(f"paged decode bad pages {dtype} accumulate {accumulate}")
    rng = np.random.default_rng(35)
    page = 16
    lens = [100, 64, 20, 48]
    c = Cache(rng, lens, 2, 64, page, dtype, weight=True, max_pages=7)
    c.dev.table[0, 1] = -5
    c.dev.table[0, 6] = c.dev.k.shape[0]
    c.dev.table[2, 0] = 2 ** 31 - 1
    c.dev.table[2, 1] = -1
    seen = [np.ones(n, bool) for n in lens]
    seen[0][16:32] = seen[0][96:] = False
    seen[2][:] = False
    q, q64 = values(rng, (4, 4, 64), dtype)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = F.focus_paged_decode(q, c.dev, weight_decay=0.5 if accumulate else None, err=err)
    assert int(err.item()) == 2
    _check(c, q64, got, dtype, visible=seen, weight=c.weight if accumulate else None, decay=0.5)
    err.zero_()
    c.dev.length[3] = -3
    c.dev.length[1] = 64
    got = F.focus_paged_decode(q, c.dev, err=err)
    assert int(err.item()) == 3
    assert not got[0][3].any() and torch.isneginf(got[1][3]).all()
    # a length past the table: its rows, here of bad pages past the fourth
    err.zero_()
    c.dev.length[3] = 10_000
    got = F.focus_paged_decode(q, c.dev, err=err)
    assert int(err.item()) == 3
    ro, rl, _ = P.decode(q64[3], c.k[3], c.v[3])
    to, tl, _ = decode_tolerances(q64[3], c.k[3], 64 ** -0.5, dtype, c.v[3], ro)
    within(to64(got[0])[3], ro, to, "clipped o")
    within(to64(got[1])[3], rl, tl, "clipped lse")


def test_decode_shared_pages():
    """Two sequences that share their first pages (a common prefix), with weights."""
    rng = np.random.default_rng(36)
    page = 16
    c = Cache(rng, [64, 40], 2, 128, page, "bf16", weight=True)
    c.table[1, :2] = c.table[0, :2]
    c.dev.table.copy_(torch.as_tensor(c.table))
    for x in (c.k, c.v):
        x[1] = np.concatenate([x[0][:32], x[1][32:]])
    q, q64 = values(rng, (2, 4, 128), "bf16")
    _check(c, q64, F.focus_paged_decode(q, c.dev, weight_decay=1.0), "bf16", weight=c.weight, decay=1.0)


def test_decode_offsets_past_32_bits():
    """A pool of more than 2^32 bytes (2^31 elements), the sequence's rows at its end."""
    page, K, D = 64, 8, 128
    n_pages = (1 << 31) // (page * K * D) + 3
    announce(f"paged decode pool of {n_pages} pages")
    k = torch.empty(n_pages, page, K, D, dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    rng = np.random.default_rng(37)
    rows = {w: values(rng, (2 * page, K, D), "bf16") for w in "kv"}
    last = [n_pages - 1, n_pages - 2]
    for t, w in ((k, "k"), (v, "v")):
        for i, p in enumerate(last):
            t[p] = rows[w][0][i * page:(i + 1) * page]
    n = 2 * page - 5
    cache = F.PagedCache(k, v, torch.tensor([last], dtype=torch.int32, device=DEV),
                         torch.tensor([n], dtype=torch.int32, device=DEV))
    q, q64 = values(rng, (1, 16, D), "bf16")
    o, lse = F.focus_paged_decode(q, cache)
    ro, rl, _ = P.decode(q64[0], rows["k"][1][:n], rows["v"][1][:n])
    to, tl, _ = decode_tolerances(q64[0], rows["k"][1][:n], D ** -0.5, "bf16", rows["v"][1][:n], ro)
    within(to64(o)[0], ro, to, "o")
    within(to64(lse)[0], rl, tl, "lse")


def test_decode_other_stream_and_workspace():
    rng = np.random.default_rng(38)
    c = Cache(rng, [900, 4000], 2, 128, 64, "bf16", weight=True)
    q, q64 = values(rng, (2, 8, 128), "bf16")
    ref = F.focus_paged_decode(q, c.dev, weight_decay=0.0)
    w = c.dev.weight.clone()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    n = F.focus_paged_decode_workspace(q, c.dev, weight_decay=0.0)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    outs = []
    for workspace in (None, ws):
        c.dev.weight.fill_(3.0)
        torch.cuda.synchronize()
        outs.append(F.focus_paged_decode(q, c.dev, weight_decay=0.0, workspace=workspace, stream=s))
        s.synchronize()
        live = torch.as_tensor(np.arange(c.weight.shape[2])[None] < np.array(c.lens)[:, None]).to(DEV)[:, None]
        assert torch.equal(torch.where(live, c.dev.weight, w), w)
    for o, lse in outs:
        assert torch.equal(o, ref[0]) and torch.equal(lse, ref[1])


def test_decode_captured_and_replayed():
    """Lengths that grow between replays, eager work in between."""
    rng = np.random.default_rng(39)
    c = Cache(rng, [300, 20], 2, 128, 16, "bf16", weight=True)
    q, _ = values(rng, (2, 8, 128), "bf16")
    full = c.dev.length.clone()
    o, lse = torch.empty_like(q), torch.empty(2, 8, device=DEV)
    ws = torch.empty(max(16, F.focus_paged_decode_workspace(q, c.dev, weight_decay=1.0)), dtype=torch.uint8, device=DEV)
    call = lambda: F.focus_paged_decode(q, c.dev, o=o, lse=lse, weight_decay=1.0, workspace=ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for n0, n1 in ((1, 20), (130, 0), (300, 7)):
        c.dev.length.copy_(torch.tensor([n0, n1], dtype=torch.int32))
        q.copy_(values(rng, (2, 8, 128), "bf16")[0])
        w0 = c.dev.weight.clone()
        g.replay()
        torch.cuda.synchronize()
        got = o.clone(), lse.clone(), c.dev.weight.clone()
        c.dev.weight.copy_(w0)
        call()
        torch.cuda.synchronize()
        assert torch.equal(got[0], o) and torch.equal(got[1], lse) and torch.equal(got[2], c.dev.weight)
    c.dev.length.copy_(full)


@pytest.mark.parametrize("D,group", [(64, 1), (64, 20), (128, 1), (128, 5)])
def test_decode_weights_hold_the_bits_of_a_float32(D, group):
    """bf16 products with the softmax weights lose none of their 24 bits.  Three rows of
    weights 1, y and 1 before the division, whose v are y's first two bf16 parts and -1:
    what is left of the sum is the third part of y, up to 2^-18.

    Off by: the score's scale and product, 2 2^-24 of at most 0.6 log2 e; the exponential,
    one step, 2^-24; at most twelve additions in float32 of at most 1; together
    (1.8 + 1 + 12) 2^-24, over a sum of weights of at least 2.5, and half a step of o.
    The rows' y are chosen so that two parts alone would be off by twice that."""
    announce(f"paged decode bits of the weights {D} group {group}")
    K = 32
    bf = lambda x: to64(torch.as_tensor(x).to(torch.bfloat16))  # noqa: E731
    s = bf(np.linspace(0.07, 0.6, 20_000, dtype=np.float32))
    s = np.unique(s)
    y = np.exp(-s)
    hi = bf(y)
    mid = bf(y - hi)
    rest = np.abs(y - hi - mid) / (2 + y)
    best = np.argsort(-rest)[:K]
    s, y, hi, mid = s[best], y[best], hi[best], mid[best]
    ref = (hi + mid - y) / (2 + y)
    tol = (1.8 + 1 + 12) * 2.0 ** -24 / 2.5 + HALF_STEP["bf16"] * np.abs(ref)
    assert (np.abs(ref) > 2 * tol).all()
    k, v = (np.zeros((1, 8, K, D), np.float32) for _ in range(2))
    k[0, 1, :, 0] = -s
    v[0, 0], v[0, 1], v[0, 2] = hi[:, None], -1.0, mid[:, None]
    dev = lambda a: torch.as_tensor(a).to(torch.bfloat16).to(DEV)  # noqa: E731
    cache = F.PagedCache(dev(k), dev(v), torch.zeros(1, 1, dtype=torch.int32, device=DEV),
                         torch.tensor([3], dtype=torch.int32, device=DEV))
    q = torch.zeros(1, K * group, D, dtype=torch.bfloat16, device=DEV)
    q[..., 0] = 1.0
    o, _ = F.focus_paged_decode(q, cache, softmax_scale=1.0)
    within(to64(o)[0].reshape(K, group, D), np.broadcast_to(ref[:, None, None], (K, group, D)),
           np.broadcast_to(tol[:, None, None], (K, group, D)), "o")


@pytest.mark.parametrize("rows,page,split,H,K,dtype", [
    (20_011, 8, 16_384, 6, 3, "bf16"),         # chunks of two rounds of 1024 pages, and one
    (20_011, 8, 16_384, 3, 3, "f32"),
    (50_000, 8, 24_960, 17, 1, "bf16"),        # three and more, more than one tile of heads
    (532_813, 256, 266_368, 2, 1, "bf16"),     # the second chunk and its rounds begin inside a page
    (532_813, 256, 266_368, 1, 1, "f32"),
])
def test_decode_chunks_of_more_pages_than_are_held_at_a_time(rows, page, split, H, K, dtype):
    announce(f"paged decode {rows} rows on pages of {page} split {split} {H}/{K} {dtype}")
    rng = np.random.default_rng(rows + H)
    c = Cache(rng, [rows, 70], K, 64, page, dtype, weight=True)
    q, q64 = values(rng, (2, H, 64), dtype)
    got = F.focus_paged_decode(q, c.dev, split_keys=split)
    _check(c, q64, got, dtype)
    again = F.focus_paged_decode(q, c.dev, split_keys=split, weight_decay=0.5)
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
    _check(c, q64, again, dtype, weight=c.weight, decay=0.5)
    # an infinity and a NaN in V, in the second round and in the last rows: the sums are
    # taken again, page by page
    clean = got[0]
    for r, col, x in ((1024 * page + 3, 5, float("inf")), (rows - 1, 9, float("nan"))):
        c.dev.v[int(c.table[0, r // page]), r % page, 0, col] = x
    o = F.focus_paged_decode(q, c.dev, split_keys=split)[0]
    G = H // K
    assert not torch.isfinite(o[0, :G, 5]).any() and torch.isnan(o[0, :G, 9]).all()
    o[0, :G, 5], o[0, :G, 9] = clean[0, :G, 5], clean[0, :G, 9]
    assert torch.equal(o, clean)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_bad_pages_past_the_first_round(dtype):
    """Pages outside the pool in the second round of a chunk's pages, reported and left out."""
    announce(f"paged decode bad pages past the first round {dtype}")
    rng = np.random.default_rng(73)
    rows, page = 12_000, 8
    c = Cache(rng, [rows], 1, 64, page, dtype, weight=True)
    seen = np.ones(rows, bool)
    for j in (1023, 1024, 1300, rows // page - 1):
        c.dev.table[0, j] = -1 if j % 2 else c.dev.k.shape[0]
        seen[j * page:(j + 1) * page] = False
    q, q64 = values(rng, (1, 2, 64), dtype)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = F.focus_paged_decode(q, c.dev, split_keys=16_384, weight_decay=0.25, err=err)
    assert int(err.item()) == 2
    _check(c, q64, got, dtype, visible=[seen], weight=c.weight, decay=0.25)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,top", [(60, 4096), (60, -4096), (3000, 4096), (3000, 512)])
def test_decode_large_scores_keep_their_differences(rows, top, dtype):
    """Scores of thousands, exact in float32, that differ by up to 4: the weights follow from
    the differences.  Off by: the scale's roundings, 2^-24 + 2^-25 of at most 4 log2 e; the
    exponential, 2^-23; the sums, each of at most rows / 16 + 16 additions in float32; the
    division, 2^-23.  Together below rel; o by that and its own sums, lse by its logarithm's
    and product's roundings.  (Scores scaled and rounded first would be off by 2^-12.)"""
    announce(f"paged decode large scores {rows} around {top} {dtype}")
    rng = np.random.default_rng(abs(rows + top))
    c = Cache(rng, [rows], 1, 64, 64, dtype, weight=True)
    t = rng.integers(0, 64, rows) / 16.0
    k = np.zeros((rows, 64))
    k[:, 0], k[:, 1] = top / 64.0, t
    at = torch.as_tensor(c.table[0][np.arange(rows) // 64].astype(np.int64)).to(DEV), torch.arange(rows, device=DEV) % 64
    c.dev.k[at] = torch.as_tensor(k).to(c.dev.k.dtype).to(DEV)[:, None]
    assert np.array_equal(to64(c.dev.k[at])[:, 0], k)
    q64 = np.zeros((2, 64))
    q64[:, 0], q64[0, 1], q64[1, 1] = 64.0, 1.0, -1.0
    q = torch.as_tensor(q64).to(c.dev.k.dtype).to(DEV)[None]
    o, lse = F.focus_paged_decode(q, c.dev, softmax_scale=1.0, weight_decay=0.0)
    ro, rl, rw = P.decode(q64, k[:, None], c.v[0], 1.0)
    sums = (rows / 16 + 16) * 2.0 ** -24
    rel = 4 * 1.4427 * (2.0 ** -24 + 2.0 ** -25) + 2 * 2.0 ** -23 + sums
    vmax = np.abs(c.v[0]).max()
    within(to64(o)[0], ro, (2 * rel + sums) * vmax + HALF_STEP[dtype] * np.abs(ro), "o")
    within(to64(lse)[0], rl, rel + np.abs(rl) * 2.0 ** -22, "lse")
    w = c.dev.weight.cpu().numpy()[0, :, :rows].astype(np.float64)
    within(w, rw, rw * (2 * rel + 2.0 ** -22), "weight")


@pytest.mark.parametrize("pages,split", [(4, 0), (80, 0), (80, 128)])
def test_decode_batch_past_the_grids_second_dimension(pages, split):
    """33 000 sequences, of short tables and of longer ones whose chunks a launch of its own
    divides: parts of the batch as by themselves (a given split, or none, fixes the bits), and
    single sequences against the oracle."""
    batch, page, D = 33_000, 8, 64
    announce(f"paged decode {batch} sequences of {pages} pages split {split}")
    g = torch.Generator(device=DEV).manual_seed(pages)
    k = torch.randn(4000, page, 1, D, generator=g, device=DEV).to(torch.bfloat16)
    v = torch.randn(4000, page, 1, D, generator=g, device=DEV).to(torch.bfloat16)
    table = torch.randint(0, 4000, (batch, pages), generator=g, device=DEV, dtype=torch.int32)
    n = torch.randint(0, 40, (batch,), generator=g, device=DEV, dtype=torch.int32).clamp(max=pages * page)
    n[::5000] = pages * page
    w = torch.rand(batch, 1, pages * page, generator=g, device=DEV)
    q = torch.randn(batch, 2, D, generator=g, device=DEV).to(torch.bfloat16)
    for decay in (None, 0.5):
        old = w.clone()
        o, lse = F.focus_paged_decode(q, F.PagedCache(k, v, table, n, w), split_keys=split, weight_decay=decay)
        if decay is None:
            assert torch.equal(w, old)
        if split or pages * page <= 256:
            for b in (0, 4950, 16_300, 32_700, batch - 100):
                at = slice(b, b + 100)
                ow = old[at].clone()
                o1, l1 = F.focus_paged_decode(q[at], F.PagedCache(k, v, table[at], n[at].contiguous(), ow),
                                              split_keys=split, weight_decay=decay)
                assert torch.equal(o1, o[at]) and torch.equal(l1, lse[at]) and torch.equal(ow, w[at])
        for b in (0, 1, 5000, 20_000, 32_767, 32_768, 32_769, batch - 1):
            m = int(n[b])
            rows = table[b].long().cpu()[torch.arange(m) // page], torch.arange(m) % page
            kk, vv = to64(k[rows[0].to(DEV), rows[1].to(DEV)]), to64(v[rows[0].to(DEV), rows[1].to(DEV)])
            ro, rl, _ = P.decode(to64(q[b]), kk, vv)
            to, tl, _ = decode_tolerances(to64(q[b]), kk, D ** -0.5, "bf16", vv, ro)
            within(to64(o[b]), ro, to, f"o[{b}]")
            within(to64(lse[b]), rl, tl, f"lse[{b}]")


def test_decode_q_shared_by_the_batch():
    """One query for all sequences and heads (strides of 0)."""
    rng = np.random.default_rng(77)
    c = Cache(rng, [300, 41], 2, 64, 16, "bf16", weight=True)
    q, _ = values(rng, (1, 1, 64), "bf16")
    q = q.expand(2, 4, 64)
    _check(c, to64(q), F.focus_paged_decode(q, c.dev, weight_decay=1.0), "bf16", weight=c.weight, decay=1.0)
