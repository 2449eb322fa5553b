"""The paged-cache calls as a serving loop makes them: rows stored, one token a step
attended with weights accumulated, the cache cut to a budget on the way, decoding
continued over what is left -- against the float64 oracle, which follows the same loop
on its own rows.  And FOCUS's own retention over pages: the summary rows of a prefill."""

from types import SimpleNamespace

import numpy as np
import pytest
import torch

import paper_2511_14694_amd as F
from gpu_util import DEV, announce, to64
from oracle import paged as P
from paged_util import HALF_STEP, Cache, decode_tolerances, paged_rows, values, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,H,K,D,page", [("bf16", 8, 2, 128, 16), ("f32", 4, 4, 64, 8)])
def test_serving_loop(dtype, H, K, D, page):
    announce(f"serving loop {dtype} {H}/{K} x {D} page {page}")
    rng = np.random.default_rng(61)
    B, budget, recent, max_pages = 3, 20, 6, 8
    prompt = [17, 1, 30]
    pool = 2 * B * max_pages
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    k, v = (torch.full((pool, page, K, D), float("nan"), dtype=dt, device=DEV) for _ in range(2))
    free = [int(x) for x in rng.permutation(pool)]
    table = lambda: torch.tensor([[free.pop() for _ in range(max_pages)] for _ in range(B)],  # noqa: E731
                                 dtype=torch.int32, device=DEV)
    weight = lambda: torch.full((B, K, max_pages * page), float("nan"), device=DEV)  # noqa: E731
    cache = F.PagedCache(k, v, table(), torch.zeros(B, dtype=torch.int32, device=DEV), weight())
    turns = F.focus_rope_turns(D, scaling=F.FOCUS_ROPE_BANDS, factor=4.0, context=4096)
    t64 = turns.cpu().numpy()
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    d = lambda a: torch.as_tensor(np.asarray(a, np.int32)).to(DEV)  # noqa: E731

    # the prompts, all sequences in one ragged call
    seq, slot = (np.concatenate(x) for x in zip(*[(np.full(n, b), np.arange(n)) for b, n in enumerate(prompt)]))
    pos = slot + 1000 * (seq + 1)
    kp, kp64 = values(rng, (len(seq), K, D), dtype)
    vp, vp64 = values(rng, (len(seq), K, D), dtype)
    F.focus_rope(d(pos), turns, None, kp, vp, layout=F.FOCUS_ROPE_HALF, cache=cache, row_seq=d(seq), row_slot=d(slot),
                 err=err)
    assert cache.length.tolist() == prompt
    # the oracle's rows are what the pages hold (checked against the rotation here), so
    # that its decode starts from the same numbers
    rows = {b: [[paged_rows(cache, b, n, w)[:, g] for g in range(K)] for w in "kv"] for b, n in enumerate(prompt)}
    ref = P.rope(kp64, pos, t64, "half")
    for b, n in enumerate(prompt):
        got = np.stack(rows[b][0], 1)
        within(got, ref[seq == b], HALF_STEP[dtype] * 1.01 * np.abs(ref[seq == b]) + 2.0 ** -19, "stored k")
        assert np.array_equal(np.stack(rows[b][1], 1), vp64[seq == b])
    w64 = {b: [np.zeros(n) for _ in range(K)] for b, n in enumerate(prompt)}
    slack = {b: 0.0 for b in range(B)}          # of the accumulated weights

    lens = list(prompt)
    for step in range(12):
        q, q64 = values(rng, (B, H, D), dtype)
        kn, _ = values(rng, (B, K, D), dtype)
        vn, vn64 = values(rng, (B, K, D), dtype)
        at = np.array([1000 * (b + 1) + prompt[b] + step for b in range(B)])
        qt, _ = F.focus_rope(d(at), turns, q, kn, vn, layout=F.FOCUS_ROPE_HALF, cache=cache, row_seq=d(range(B)),
                             row_slot=d(lens), err=err)
        o, lse = F.focus_paged_decode(qt, cache, weight_decay=0.5, err=err)
        q64 = to64(qt)
        for b in range(B):
            new = paged_rows(cache, b, lens[b] + 1)[-1]
            for g in range(K):
                rows[b][0][g] = np.vstack([rows[b][0][g], new[g]])
                rows[b][1][g] = np.vstack([rows[b][1][g], vn64[b, g]])
                w64[b][g] = np.append(w64[b][g], 0.0)
            lens[b] += 1
            kk, vv = np.stack(rows[b][0], 1), np.stack(rows[b][1], 1)
            ro, rl, rw = P.decode(q64[b], kk, vv)
            to, tl, rel = decode_tolerances(q64[b], kk, D ** -0.5, dtype, vv, ro)
            within(to64(o)[b], ro, to, f"step {step} o[{b}]")
            within(to64(lse)[b], rl, tl, f"step {step} lse[{b}]")
            slack[b] = 0.5 * slack[b] + H // K * (rel.max() + 2.0 ** -20)
            for g in range(K):
                w64[b][g] = 0.5 * w64[b][g] + rw[g]
                within(cache.weight[b, g, :lens[b]].cpu().numpy(), w64[b][g], slack[b], f"step {step} weight[{b}]")
        assert cache.length.tolist() == lens
        if step in (4, 9):
            out = F.PagedCache(k, v, table() if step == 4 else first, torch.zeros_like(cache.length), weight())
            first = cache.table
            keep = F.focus_paged_evict(cache, out, budget, recent=recent, err=err).cpu().numpy()
            # the choice is checked on the device's own weights: two that differ by less
            # than their rounding may change places
            dev_w = cache.weight.cpu().numpy()
            for b in range(B):
                m = min(lens[b], budget)
                for g in range(K):
                    kept = P.keep(dev_w[b, g, :lens[b]], budget, recent)
                    assert keep[b, g, :m].tolist() == kept and (keep[b, g, m:] == -1).all()
                    for w in (0, 1):
                        rows[b][w][g] = rows[b][w][g][kept]
                    w64[b][g] = w64[b][g][kept]
                lens[b] = m
            cache = out
            assert cache.length.tolist() == lens
    assert int(err.item()) == 0


def test_summary_rows_of_a_prefill_into_pages():
    """focus_qkv_project's turned rows of the summary tokens, stored at the layout's own
    cache rows: the pages hold what focus_compact_kv appends to a contiguous cache, and
    a token attends over them as focus_decode_step does."""
    rng = np.random.default_rng(62)
    announce("summary rows into pages")
    seq, W, kk, H, K, D, dm = [2600, 900], 500, 50, 4, 2, 128, 128
    tot = F.focus_layout_plan(seq, W, None, kk)
    lay = F.focus_layout(tot, seq, W, None, kk, device=DEV)
    hid, _ = values(rng, (tot.n_tokens, dm), "bf16")
    w, _ = values(rng, (dm, (H + 2 * K) * D), "bf16", dm ** -0.5)
    q, k, v = F.focus_qkv_project(lay, hid, w, H, K)
    cap = int(tot.max_cache_per_seq)
    ck = torch.zeros(2, cap + 1, K, D, dtype=torch.bfloat16, device=DEV)
    cv, clen = torch.zeros_like(ck), torch.zeros(2, dtype=torch.int32, device=DEV)
    F.focus_compact_kv(lay, k, v, ck, cv, clen)

    page, per = 16, -(-(cap + 1) // 16)
    pool = torch.zeros(2 * per, page, K, D, dtype=torch.bfloat16, device=DEV)
    table = torch.as_tensor(rng.permutation(2 * per).astype(np.int32).reshape(2, per)).to(DEV)
    cache = F.PagedCache(pool, torch.zeros_like(pool), table, torch.zeros(2, dtype=torch.int32, device=DEV))
    summary = lay["tok_kind"] == F.FOCUS_TOK_SUMMARY
    slot = torch.where(summary, lay["tok_kmer"], torch.full_like(lay["tok_kmer"], -1))
    F.focus_rope(lay["tok_pos"], None, None, k, v, cache=cache, row_seq=lay["win_seq"][lay["tok_win"].long()],
                 row_slot=slot)
    assert cache.length.tolist() == clen.tolist()
    for b, n in enumerate(clen.tolist()):
        assert np.array_equal(paged_rows(cache, b, n, "k"), to64(ck[b, :n]))
        assert np.array_equal(paged_rows(cache, b, n, "v"), to64(cv[b, :n]))
    # the next summary token, through both caches
    qn, kn, vn = (values(rng, (2, h, D), "bf16")[0] for h in (H, K, K))
    kind = torch.full((2,), F.FOCUS_STEP_SUMMARY, dtype=torch.uint8, device=DEV)
    win = torch.zeros(2, 1, K, D, dtype=torch.bfloat16, device=DEV)
    n0 = clen.clone()
    o1, l1 = F.focus_decode_step(qn, kn, vn, kind, ck, cv, clen, win, win.clone(), torch.zeros_like(clen))
    F.focus_rope(torch.zeros(2, dtype=torch.int32, device=DEV), None, None, kn, vn, cache=cache,
                 row_seq=torch.arange(2, dtype=torch.int32, device=DEV), row_slot=n0)
    o2, l2 = F.focus_paged_decode(qn, cache)
    for b, n in enumerate(clen.tolist()):
        k64, v64, q64 = to64(ck[b, :n]), to64(cv[b, :n]), to64(qn)[b]
        to, tl, _ = decode_tolerances(q64, k64, D ** -0.5, "bf16", v64, to64(o1)[b])
        within(to64(o2)[b], to64(o1)[b], 2 * to, "o")
        within(to64(l2)[b], to64(l1)[b], 2 * tl, "lse")


@pytest.mark.parametrize("batch,rows,K,G", [(3, 700, 2, 4), (140, 600, 1, 2)])
def test_serving_steps_captured(batch, rows, K, G):
    """Store, attend and weigh in one graph, cut in another (both with scratch of their
    own), replayed in turn with eager work between, against the same calls eagerly."""
    announce(f"captured serving of {batch} x {rows}")
    rng = np.random.default_rng(batch)
    D, page, steps, budget = 64, 16, 3, rows // 2
    lens = [int(x) for x in rng.integers(1, rows, batch)]
    lens[0] = rows
    per = -(-(rows + steps) // page)
    c = Cache(rng, lens, K, D, page, "bf16", max_pages=per, weight=True, spare=batch * (per + 2))
    free = c.free
    for b in range(batch):       # pages for the rows to come
        for j in range(per):
            if c.table[b, j] < 0:
                c.table[b, j] = free.pop()
    c.dev.table.copy_(torch.as_tensor(c.table))
    c.dev.weight.zero_()
    q, k, v = (values(rng, (batch, h, D), "bf16")[0] for h in (K * G, K, K))
    seq = torch.arange(batch, dtype=torch.int32, device=DEV)
    slot, pos = c.dev.length.clone(), c.dev.length.clone()
    turns = F.focus_rope_turns(D)
    opages = -(-budget // page)
    pool = torch.zeros(batch * opages, page, K, D, dtype=torch.bfloat16, device=DEV)
    out = F.PagedCache(pool, pool.clone(), torch.arange(batch * opages, dtype=torch.int32, device=DEV).view(batch, -1),
                       torch.zeros_like(slot), torch.zeros(batch, K, opages * page, device=DEV))
    keep = torch.empty(batch, K, budget, dtype=torch.int32, device=DEV)
    o, lse, qt = torch.empty_like(q), torch.empty(batch, K * G, device=DEV), torch.empty_like(q)
    src = c.dev

    def step():
        F.focus_rope(pos, turns, q, k, v, q_out=qt, cache=src, row_seq=seq, row_slot=slot)
        F.focus_paged_decode(qt, src, o=o, lse=lse, weight_decay=0.9)

    def cut():
        F.focus_paged_evict(src, out, budget, recent=8, keep=keep)

    state = [src.k, src.v, src.length, src.weight, o, lse, qt, out.k, out.v, out.length, out.weight, keep]
    first = [t.clone() for t in state]
    eager = []
    for i in range(steps):
        step(), cut()
        eager.append([t.clone() for t in state])
        slot += 1
        pos += 1
    torch.cuda.synchronize()
    for t, x in zip(state, first):
        t.copy_(x)
    slot -= steps
    pos -= steps
    torch.cuda.synchronize()
    graphs = []
    for call in (step, cut):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        graphs.append(g)
    for i in range(steps):
        for g in graphs:
            g.replay()
            F.focus_paged_decode(q, src)     # eager work in between
        torch.cuda.synchronize()
        for t, x in zip(state, eager[i]):
            assert torch.equal(t.view(torch.uint8), x.view(torch.uint8))
        slot += 1
        pos += 1


def test_calls_on_two_streams_at_once():
    """Each call has scratch of its own: decoding and cutting on two streams gives what one
    after another gives."""
    announce("two streams")
    rng = np.random.default_rng(63)
    work = []
    for n in (5000, 36_000):
        c = Cache(rng, [n, 100], 2, 64, 64, "bf16", weight=True, spare=2 * 20)
        q, _ = values(rng, (2, 8, 64), "bf16")
        out = c.other(rng, 1000)
        work.append((c, q, out))

    def call(c, q, out, stream=None):
        o, lse = F.focus_paged_decode(q, c.dev, weight_decay=0.5, stream=stream)
        keep = F.focus_paged_evict(c.dev, out, 1000, recent=10, stream=stream)
        return o, lse, keep, c.dev.weight.clone() if stream is None else None

    w0 = [c.dev.weight.clone() for c, _, _ in work]
    one = [call(*x) for x in work]
    for (c, _, _), w in zip(work, w0):
        c.dev.weight.copy_(w)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    two = [call(*x, stream=s) for x, s in zip(work, streams)]
    torch.cuda.synchronize()
    for a, b, (c, _, _) in zip(one, two, work):
        assert all(torch.equal(x, y) for x, y in zip(a[:3], b[:3]))
        assert torch.equal(a[3], c.dev.weight)


def test_outputs_do_not_take_blocks_that_the_callers_stream_still_writes():
    """Blocks of the outputs' sizes, freed on the caller's stream with a write to them still
    to come there: calls on another stream have outputs of their own."""
    announce("outputs on another stream")
    rng = np.random.default_rng(64)
    c = Cache(rng, [5000, 100], 2, 64, 64, "bf16", weight=True, spare=2 * 20)
    q, _ = values(rng, (2, 8, 64), "bf16")
    out = c.other(rng, 1000)
    pos = torch.tensor([7, 8], dtype=torch.int32, device=DEV)
    turns = F.focus_rope_turns(64)

    def call(stream=None):
        qt, _ = F.focus_rope(pos, turns, q, stream=stream)
        o, lse = F.focus_paged_decode(q, c.dev, stream=stream)
        keep = F.focus_paged_evict(c.dev, out, 1000, recent=10, stream=stream)
        return qt, o, lse, keep

    want = [t.clone() for t in call()]
    other = torch.cuda.Stream()
    warm = call(other)
    torch.cuda.synchronize()
    del warm
    a = torch.randn(4096, 4096, device=DEV)
    torch.cuda.synchronize()
    blocks = [torch.empty_like(t) for t in want]
    for _ in range(20):
        a = a @ a * 1e-3          # some milliseconds before the writes
    for t in blocks:
        t.fill_(77)
    del blocks, t
    got = call(other)
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g, w)
    # a result read on the caller's stream and freed there keeps its block until then
    a = torch.randn(4096, 4096, device=DEV)
    torch.cuda.synchronize()
    o, _ = F.focus_paged_decode(q, c.dev, stream=other)
    torch.cuda.current_stream().wait_stream(other)
    for _ in range(20):
        a = a @ a * 1e-3
    read = o.clone()
    del o
    for _ in range(3):
        F.focus_paged_decode(torch.zeros_like(q), c.dev, stream=other)
    torch.cuda.synchronize()
    assert torch.equal(read, want[1])


def test_a_call_on_another_stream_inside_a_capture():
    """A capture that forks to another stream for a call, outputs allocated in it, and joins."""
    announce("captured on another stream")
    rng = np.random.default_rng(65)
    c = Cache(rng, [3000, 100], 2, 64, 64, "bf16", weight=True)
    q, _ = values(rng, (2, 8, 64), "bf16")
    F.focus_paged_decode(q, c.dev)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        other.wait_stream(torch.cuda.current_stream())
        o, lse = F.focus_paged_decode(q, c.dev, stream=other)
        torch.cuda.current_stream().wait_stream(other)
    for seed in range(3):
        q.copy_(values(rng, (2, 8, 64), "bf16")[0])
        g.replay()
        torch.cuda.synchronize()
        got = o.clone(), lse.clone()
        want = F.focus_paged_decode(q, c.dev)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_stream_given_by_its_handle():
    """stream= takes any object with a handle in cuda_stream, also where a call allocates."""
    announce("a stream by its handle")
    rng = np.random.default_rng(66)
    c = Cache(rng, [3000, 100], 2, 64, 64, "bf16", weight=True)
    q, _ = values(rng, (2, 8, 64), "bf16")
    want = F.focus_paged_decode(q, c.dev)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    got = F.focus_paged_decode(q, c.dev, stream=SimpleNamespace(cuda_stream=other.cuda_stream))
    other.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
