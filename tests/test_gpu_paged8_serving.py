"""The 8-bit paged cache's calls as a serving loop makes them: slots taken, positions turned,
rows stored, the newest tokens attended, drafted ones given back -- against the oracle, which
follows the same loop -- and captured, on other streams and side by side."""

from types import SimpleNamespace

import numpy as np
import pytest
import torch

import paper_2511_14694_amd as F
from gpu_util import DEV, announce, to64
from oracle import paged as P
from oracle import paged8 as O
from paged8_util import E4M3, NAN, Cache8, i32, to_codes
from paged_util import HALF_STEP, values, within

pytestmark = pytest.mark.gpu


def _pool(pages, page, K, D, block):
    """A pool of NaN."""
    k, v = (torch.full((pages, page, K, D), NAN, dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2))
    ks, vs = (torch.full((pages, K, page // block), float("nan"), device=DEV) for _ in range(2))
    return k, v, ks, vs


@pytest.mark.parametrize("dtype,H,K,D,page,block,pages", [("bf16", 8, 2, 128, 16, 8, 10), ("f32", 4, 4, 64, 32, 32, 6)])
def test_serving_loop(dtype, H, K, D, page, block, pages):
    announce(f"8-bit serving loop {dtype} {H}/{K} x {D} page {page} block {block}")
    rng = np.random.default_rng(71)
    B, width, most = 4, 9, 5
    cache = F.PagedCache8(*_pool(pages, page, K, D, block), torch.full((B, width), -1, dtype=torch.int32, device=DEV),
                          torch.zeros(B, dtype=torch.int32, device=DEV))
    table, length, free = [[-1] * width for _ in range(B)], [0] * B, [int(x) for x in rng.permutation(pages)]
    d_free, d_count = i32(free), i32([pages])
    rows = [[np.zeros((0, D)) for _ in range(K)] for _ in range(2 * B)]      # of k and v, 8-bit numbers
    scales = [[np.full(width * page // block, np.nan) for _ in range(K)] for _ in range(2 * B)]
    turns = F.focus_rope_turns(D)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    unserved = 0

    def give_back(drop):
        F.focus_paged_extend(cache.table, cache.length, page, i32([-x for x in drop]), d_free, d_count, 0, err=err)
        O.extend(table, length, page, [-x for x in drop], free, 0)
        for b in range(B):
            for side in (b, B + b):
                rows[side] = [x[:length[b]] for x in rows[side]]

    for step in range(14):
        # prompts first, then one to five tokens of each sequence, some with none
        add = [40, 1, 0, 75] if step == 0 else [int(x) for x in rng.integers(0, most + 1, B)]
        if step == 9:
            give_back([1000, 0, 2, 1000])      # two sequences end: their slots start again
        n = sum(add) + 3                       # a batch padded to more rows than there are
        q, _ = values(rng, (n, H, D), dtype)
        k, _ = values(rng, (n, K, D), dtype, 2.0 ** rng.integers(-3, 4))
        v, _ = values(rng, (n, K, D), dtype)
        err.zero_()
        got = F.focus_paged_extend(cache.table, cache.length, page, i32(add), d_free, d_count, n, err=err)
        start, cu, *_, fine = O.extend(table, length, page, add, free, n)
        assert cache.table.tolist() == table and cache.length.tolist() == length and got.start.tolist() == start
        assert err.item() == (0 if fine else F.FOCUS_ERR_CAPACITY)
        qt, kt = F.focus_rope(got.row_pos, turns, q, k)
        F.focus_paged_append(kt, v, cache, got.start, got.cu_rows)
        o, lse = F.focus_paged_attend(qt, cache, got.cu_rows, max_rows=75 if step == 0 else most)
        assert cache.length.tolist() == length
        q64, k64, v64 = to64(qt), to64(kt), to64(v)
        o, lse = to64(o), to64(lse)
        for b in range(B):
            new = slice(cu[b], cu[b + 1])
            if start[b] < 0:
                unserved += 1
                continue
            kk, vv = [], []
            for side, x, to in ((b, k64, kk), (B + b, v64, vv)):
                for g in range(K):
                    if add[b]:
                        rows[side][g], scales[side][g] = O.append(rows[side][g], scales[side][g], block, start[b], x[new, g])
                    to.append(rows[side][g] * scales[side][g].repeat(block)[:length[b], None])
            kk, vv = np.stack(kk, 1), np.stack(vv, 1)
            ro, rl = O.attend(q64[new], kk, vv)
            to, tl = O.attend_tolerances(q64[new], kk, vv, D ** -0.5, dtype, ro)
            within(o[new], ro, to, f"step {step} o[{b}]")
            within(lse[new], rl, tl, f"step {step} lse[{b}]")
            # and of the rows as they were before they were held in 8 bits: off by 2^-4 of them
            # at most where a row's scale is its block's
            r = length[b] - 1
            if r >= 0 and add[b]:
                p, at = table[b][r // page], r % page
                got_k = to_codes(cache.k)[p, at] * cache.k_scale.cpu().double().numpy()[p, :, at // block][:, None]
                least = cache.k_scale.cpu().double().numpy()[p, :, at // block][:, None] * 2.0 ** -10
                within(got_k, k64[cu[b + 1] - 1], 2.0 ** -4 * np.abs(k64[cu[b + 1] - 1]) + least, "k")
        # drafted tokens that are not kept
        if step % 3 == 2:
            give_back([int(rng.integers(0, x + 1)) if s >= 0 else 0 for x, s in zip(add, start)])
    assert unserved, "the pool never ran out"


def test_turned_rows_are_stored_at_the_maps_of_a_bf16_cache_too():
    """focus_paged_extend's maps are what focus_rope stores by: a bf16 cache and an 8-bit one of
    the same tables, decoded alike but for the rounding."""
    rng = np.random.default_rng(72)
    announce("bf16 and 8-bit cache side by side")
    B, H, K, D, page, pages = 3, 4, 2, 64, 16, 12
    table = torch.full((B, 4), -1, dtype=torch.int32, device=DEV)
    length, free, count = i32([0] * B), i32(rng.permutation(pages)), i32([pages])
    add = [20, 33, 1]
    got = F.focus_paged_extend(table, length, page, i32(add), free, count, 60, first_pos=i32([5, 0, 900]))
    q, k, v = (values(rng, (60, h, D), "bf16")[0] for h in (H, K, K))
    wide = F.PagedCache(torch.zeros(pages, page, K, D, dtype=torch.bfloat16, device=DEV),
                        torch.zeros(pages, page, K, D, dtype=torch.bfloat16, device=DEV), table, length.clone())
    turns = F.focus_rope_turns(D)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    qt, kt = F.focus_rope(got.row_pos, turns, q, k, v, k_out=torch.empty_like(k), cache=wide, row_seq=got.row_seq,
                          row_slot=got.row_slot, err=err)
    assert err.item() == 0 and wide.length.tolist() == add
    small = F.PagedCache8(*_pool(pages, page, K, D, 8), table, length)
    F.focus_paged_append(kt, v, small, got.start, got.cu_rows)
    last = (got.cu_rows[1:] - 1).long()
    o1, l1 = F.focus_paged_decode(qt[last], wide)
    o2, l2 = F.focus_paged_attend(qt[last], small)
    # a score is off by 2^-4 of its terms' absolute sum (and a little for small elements), a
    # weight relatively by twice that, o by it and by 2^-4 of the largest |v|
    cu = [0, 20, 53, 54]
    for b in range(B):
        k64, v64, q64 = to64(kt)[cu[b]:cu[b + 1]], to64(v)[cu[b]:cu[b + 1]], to64(qt)[cu[b + 1] - 1]
        e = max(np.abs(k64[:, h // 2]).max(0) @ np.abs(q64[h]) for h in range(H)) * D ** -0.5 * (2.0 ** -4 + 2.0 ** -7)
        assert np.abs(to64(l1)[b] - to64(l2)[b]).max() <= e + 2.0 ** -10
        assert np.abs(to64(o1)[b] - to64(o2)[b]).max() <= (2 * e * np.exp(2 * e) + 2.0 ** -4 + 2.0 ** -6) * np.abs(v64).max()


@pytest.mark.parametrize("batch,rows,D", [(3, 300, 128), (2, 3000, 64), (150, 20, 64)])
def test_serving_steps_captured(batch, rows, D):
    """A whole step in one graph, its lengths and pages moving on by themselves; every replay
    against the eager calls, with eager work between."""
    announce(f"8-bit serving step captured {batch} x {rows} x {D}")
    rng = np.random.default_rng(73)
    H, K, page, block, new, steps = 4, 2, 16, 8, 2, 5
    need = -(-(rows + new * steps) // page) + 1
    lens = [rows - (b % 3) for b in range(batch)]
    turns = F.focus_rope_turns(D)

    def state():
        c = Cache8(np.random.default_rng(5), lens, K, D, page, block, max_pages=need + 20, spare=batch * 3)
        free = i32(c.free + [-1] * 4)
        return c.dev, free, i32([len(c.free)])

    n = batch * new
    q, k, v = (torch.zeros(n, h, D, dtype=torch.bfloat16, device=DEV) for h in (H, K, K))
    add = i32([new] * batch)
    inputs = [[values(rng, x.shape, "bf16")[0] for x in (q, k, v)] for _ in range(steps)]

    def step(cache, free, count):
        got = F.focus_paged_extend(cache.table, cache.length, page, add, free, count, n)
        qt, kt = F.focus_rope(got.row_pos, turns, q, k)
        F.focus_paged_append(kt, v, cache, got.start, got.cu_rows)
        return F.focus_paged_attend(qt, cache, got.cu_rows, max_rows=new)

    one, two = state(), state()
    eager = []
    for x in inputs:
        for to, y in zip((q, k, v), x):
            to.copy_(y)
        o, lse = step(*one)
        eager.append([t.clone() for t in (o, lse, one[0].k.view(torch.uint8), one[0].v_scale, one[0].table, one[0].length,
                                          one[1], one[2])])
    torch.cuda.synchronize()
    warm = state()
    step(*warm)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o, lse = step(*two)
    for x, want in zip(inputs, eager):
        for to, y in zip((q, k, v), x):
            to.copy_(y)
        g.replay()
        F.focus_paged_attend(q, warm[0], i32([new * b for b in range(batch + 1)]), max_rows=new)    # eager work between
        torch.cuda.synchronize()
        for a, b in zip((o, lse, two[0].k.view(torch.uint8), two[0].v_scale, two[0].table, two[0].length, two[1], two[2]), want):
            assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))
    assert two[0].length.tolist() == [x + new * steps for x in lens]


def test_calls_on_two_streams_at_once():
    announce("8-bit calls on two streams")
    rng = np.random.default_rng(74)
    work = []
    for n in (5000, 36_000):
        c = Cache8(rng, [n, 100], 2, 64, 64, 16, spare=8, max_pages=n // 64 + 4)
        q, k, v = (values(rng, (3, h, 64), "bf16")[0] for h in (8, 2, 2))
        work.append((c.dev, q, k, v, i32(c.free), i32([len(c.free)])))
    keep = [(c.length.clone(), c.table.clone(), c.k.view(torch.uint8).clone(), c.k_scale.clone(), free.clone(), count.clone())
            for c, *_, free, count in work]

    def call(c, q, k, v, free, count, stream=None):
        got = F.focus_paged_extend(c.table, c.length, 64, add, free, count, 3, stream=stream)
        F.focus_paged_append(k, v, c, got.start, got.cu_rows, stream=stream)
        o, lse = F.focus_paged_attend(q, c, got.cu_rows, max_rows=2, stream=stream)
        return o, lse, got.row_slot

    add = i32([2, 1])
    one = [call(*x) for x in work]
    after = [(c.k.view(torch.uint8).clone(), c.length.clone(), count.clone()) for c, *_, count in work]
    for (c, *_, free, count), (length, table, codes, scale, f, n) in zip(work, keep):
        c.length.copy_(length), c.table.copy_(table), c.k.view(torch.uint8).copy_(codes), c.k_scale.copy_(scale)
        free.copy_(f), count.copy_(n)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    two = [call(*x, stream=s) for x, s in zip(work, streams)]
    torch.cuda.synchronize()
    for a, b, (codes, length, n), (c, *_, count) in zip(one, two, after, work):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
        assert torch.equal(codes, c.k.view(torch.uint8)) and torch.equal(length, c.length) and torch.equal(n, count)


def test_a_call_on_another_stream_inside_a_capture_and_by_its_handle():
    announce("8-bit call captured on another stream")
    rng = np.random.default_rng(75)
    c = Cache8(rng, [3000, 100], 2, 64, 64, 16)
    q, _ = values(rng, (2, 8, 64), "bf16")
    want = F.focus_paged_attend(q, c.dev)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = F.focus_paged_attend(q, c.dev, stream=SimpleNamespace(cuda_stream=other.cuda_stream))
    other.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        other.wait_stream(torch.cuda.current_stream())
        o, lse = F.focus_paged_attend(q, c.dev, stream=other)
        torch.cuda.current_stream().wait_stream(other)
    for _ in range(3):
        q.copy_(values(rng, (2, 8, 64), "bf16")[0])
        g.replay()
        torch.cuda.synchronize()
        got = o.clone(), lse.clone()
        want = F.focus_paged_attend(q, c.dev)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_summary_rows_of_a_prefill_in_8_bits():
    """FOCUS's own retention: the summary rows of focus_qkv_project, sequence after sequence,
    appended at once; pages and scales as the oracle's."""
    rng = np.random.default_rng(76)
    announce("summary rows in 8 bits")
    seq, W, kk, H, K, D, dm = [2600, 900], 500, 50, 4, 2, 128, 128
    tot = F.focus_layout_plan(seq, W, None, kk)
    lay = F.focus_layout(tot, seq, W, None, kk, device=DEV)
    hid, _ = values(rng, (tot.n_tokens, dm), "bf16")
    w, _ = values(rng, (dm, (H + 2 * K) * D), "bf16", dm ** -0.5)
    q, k, v = F.focus_qkv_project(lay, hid, w, H, K)
    counts = [52, 18]
    rows = lay["sum_tok"]
    assert rows.numel() == sum(counts)
    page, block, pages = 16, 16, 8
    table, length = torch.full((2, 5), -1, dtype=torch.int32, device=DEV), i32([0, 0])
    free, count = i32(rng.permutation(pages)), i32([pages])
    got = F.focus_paged_extend(table, length, page, i32(counts), free, count, sum(counts))
    cache = F.PagedCache8(*_pool(pages, page, K, D, block), table, length)
    ks, vs = k[rows], v[rows]
    F.focus_paged_append(ks, vs, cache, got.start, got.cu_rows)
    codes, scale = to_codes(cache.k), cache.k_scale.cpu().double().numpy()
    t = table.cpu().numpy()
    k64 = to64(ks)
    for b, (n, r0) in enumerate(zip(counts, (0, 52))):
        r = np.arange(n)
        for g in range(K):
            ref, s = O.append(np.zeros((0, D)), np.zeros(5 * page // block), block, 0, k64[r0:r0 + n, g])
            assert np.array_equal(codes[t[b][r // page], r % page, g], ref)
            assert np.array_equal(scale[t[b][r // page], g, r % page // block], s[r // block])
    o, lse = F.focus_paged_attend(q[rows[torch.tensor([51, 69], device=DEV)]], cache)
    for b, n in enumerate(counts):
        p = t[b][np.arange(n) // page], np.arange(n) % page
        kk64, vv64 = (to_codes(x)[p] * y.cpu().double().numpy()[p[0], :, p[1] // block][:, :, None]
                      for x, y in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
        q64 = to64(q[rows[[51, 69][b]]])[None]
        ro, rl = O.attend(q64, kk64, vv64)
        to, tl = O.attend_tolerances(q64, kk64, vv64, D ** -0.5, "bf16", ro)
        within(to64(o)[b], ro[0], to[0], "o")
        within(to64(lse)[b], rl[0], tl[0], "lse")
