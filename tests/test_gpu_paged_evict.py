"""focus_paged_evict on the GPU: the rows kept equal the oracle's, and rows, weights and
lengths are copied bit for bit."""

import numpy as np
import pytest
import torch

import paper_2511_14694_amd as F
from gpu_util import DEV, announce
from oracle import paged as P
from paged_util import Cache, paged_rows

pytestmark = pytest.mark.gpu


def _weights(rng, shape, kind):
    if kind == "ties":
        return rng.integers(0, 3, shape).astype(np.float32)
    if kind == "equal":
        return np.full(shape, 0.25, np.float32)
    if kind == "signs":
        return (rng.standard_normal(shape) * np.exp2(rng.integers(-40, 40, shape))).astype(np.float32)
    if kind == "special":
        return rng.choice(np.array([0.0, -0.0, np.nan, -np.nan, np.inf, -np.inf, 1e-45, -1e-45, 1.0], np.float32), shape)
    return (rng.random(shape) ** 8).astype(np.float32)


def _check(c, out, budgets, recent, keep, old):
    """out and keep after an eviction of the Cache c (its pools before: old)."""
    K = c.dev.k.shape[2]
    got, w, ow = keep.cpu().numpy(), c.dev.weight.cpu().numpy(), None if out.weight is None else out.weight.cpu().numpy()
    touched = [old[0].clone(), old[1].clone()]
    lens = []
    for b, n in enumerate(c.lens):
        m = min(n, max(budgets[b], 0), got.shape[2], out.table.shape[1] * out.k.shape[1])
        lens.append(m)
        for g in range(K):
            ref = P.keep(w[b, g, :n], m, recent)
            assert got[b, g, :m].tolist() == ref, (b, g)
            assert (got[b, g, m:] == -1).all()
            if ow is not None:
                assert np.array_equal(ow[b, g, :m], w[b, g, ref], equal_nan=True)
                assert (ow[b, g, m:] == -1.0).all(), "weights past the rows kept"
            for which, rows in (("k", c.k[b]), ("v", c.v[b])):
                assert np.array_equal(paged_rows(out, b, m, which)[:, g], rows[ref, g]), (b, g, which)
        if m:
            r = np.arange(m)
            pid = out.table[b][torch.as_tensor(r // out.k.shape[1]).to(DEV)].long()
            for t, now in zip(touched, (out.k, out.v)):
                t[pid, torch.as_tensor(r % out.k.shape[1]).to(DEV)] = now[pid, torch.as_tensor(r % out.k.shape[1]).to(DEV)]
    assert out.length.tolist() == lens
    for t, now in zip(touched, (out.k, out.v)):
        assert torch.equal(t.nan_to_num(7.0), now.nan_to_num(7.0)), "rows that are not kept were written"


@pytest.mark.parametrize("lens,K,D,page,dtype,budget,recent", [
    ([1], 1, 64, 8, "f32", 1, 0),
    ([5, 0, 9], 2, 64, 8, "bf16", 4, 2),
    ([40, 41, 8, 200], 3, 128, 16, "bf16", 40, 7),
    ([1210], 1, 64, 16, "f32", 200, 37),
    ([3000, 129], 2, 128, 64, "bf16", 1500, 0),
    ([3000, 129], 2, 96, 128, "bf16", 1, 1),
    ([700, 64], 8, 8, 32, "bf16", 300, 300),         # the latest rows only
    ([700, 64], 4, 256, 32, "f32", 0, 10),           # nothing
    ([9000], 2, 64, 16, "bf16", 8999, 100),
])
@pytest.mark.parametrize("kind", ["skewed", "ties", "equal", "signs", "special"])
def test_evict_matches_oracle(lens, K, D, page, dtype, budget, recent, kind):
    announce(f"evict {lens} x {K} x {D} page {page} {dtype} budget {budget} recent {recent} {kind}")
    rng = np.random.default_rng(sum(lens) + budget)
    rows = -(-budget // page) * page or page
    c = Cache(rng, lens, K, D, page, dtype, weight=True, spare=len(lens) * (rows // page), by_head=kind == "ties")
    c.dev.weight.copy_(torch.as_tensor(_weights(rng, c.weight.shape, kind)))
    out = c.other(rng, budget)
    old = c.dev.k.clone(), c.dev.v.clone()
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    keep = F.focus_paged_evict(c.dev, out, budget, recent=recent, err=err)
    assert keep.shape == (len(lens), K, budget) and int(err.item()) == 0
    _check(c, out, [budget] * len(lens), recent, keep, old)


@pytest.mark.parametrize("n,budget", [(70_001, 20_000), (131_072, 131_000)])
def test_evict_long(n, budget):
    """Rows beyond what one pass of a workgroup holds; most of the weights equal."""
    announce(f"evict long {n} -> {budget}")
    rng = np.random.default_rng(n)
    c = Cache(rng, [n, 300], 1, 64, 128, "bf16", weight=True, spare=2 * (budget // 128 + 1))
    w = np.where(rng.random(c.weight.shape) < 0.5, 0.0, c.weight).astype(np.float32)
    c.dev.weight.copy_(torch.as_tensor(w))
    out = c.other(rng, budget)
    old = c.dev.k.clone(), c.dev.v.clone()
    keep = F.focus_paged_evict(c.dev, out, budget, recent=1000)
    _check(c, out, [budget] * 2, 1000, keep, old)


def test_evict_budgets_other_pool_and_errors():
    """Budgets of their own (a negative one counts as 0), rows of another pool with other
    pages, too little room, pages outside the pool, lengths outside the table."""
    rng = np.random.default_rng(51)
    lens = [100, 50, 20]
    c = Cache(rng, lens, 2, 64, 16, "bf16", weight=True, max_pages=7)
    budgets = [30, 60, -4]
    k = torch.full((12, 2, 8, 64), 9.0, dtype=torch.bfloat16, device=DEV).transpose(1, 2)
    out = F.PagedCache(k, k.clone(memory_format=torch.preserve_format),
                       torch.tensor([[7, 0, 11, 3], [2, 9, 4, 5], [1, 6, 8, 10]], dtype=torch.int32, device=DEV),
                       torch.full((3,), -1, dtype=torch.int32, device=DEV))
    old = out.k.clone(), out.v.clone()
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    announce("evict budgets")
    keep = F.focus_paged_evict(c.dev, out, torch.tensor(budgets, dtype=torch.int32, device=DEV), recent=5, err=err)
    assert int(err.item()) == 3 and keep.shape == (3, 2, 32)      # 50 rows do not fit in four pages of 8
    _check(c, out, budgets, 5, keep, old)
    # a caller's keep of fewer rows than the budget
    err.zero_()
    out.k.fill_(9.0)
    out.v.fill_(9.0)
    keep = torch.full((3, 2, 17), 5, dtype=torch.int32, device=DEV)
    assert F.focus_paged_evict(c.dev, out, 20, recent=5, keep=keep, err=err) is keep
    assert int(err.item()) == 1
    _check(c, out, [20] * 3, 5, keep, old)
    # a source page and a destination page outside the pool: those rows stay as they were
    announce("evict bad pages")
    err.zero_()
    out.k.fill_(9.0)
    c.dev.table[0, 0] = -1
    out.table[1, 1] = 12
    keep = F.focus_paged_evict(c.dev, out, 20, recent=20, err=err)
    assert int(err.item()) == 2
    assert keep[0, 0].tolist() == list(range(80, 100))
    keep = F.focus_paged_evict(c.dev, out, 100, recent=0, err=err)
    assert out.length.tolist() == [32, 32, 20]
    # lengths outside the table are clipped
    err.zero_()
    c.dev.length[1] = -1
    F.focus_paged_evict(c.dev, out, 20, err=err)
    assert int(err.item()) & 1 and out.length.tolist() == [20, 0, 20]


def test_evict_length_in_place_and_empty():
    rng = np.random.default_rng(52)
    c = Cache(rng, [33, 12], 2, 64, 8, "f32", weight=True, spare=8)
    out = c.other(rng, 16)
    out.length = c.dev.length
    old = c.dev.k.clone(), c.dev.v.clone()
    keep = F.focus_paged_evict(c.dev, out, 16, recent=3)
    _check(c, out, [16, 16], 3, keep, old)
    none = F.PagedCache(c.dev.k, c.dev.v, c.dev.table[:0], c.dev.length[:0], c.dev.weight[:0])
    assert F.focus_paged_evict(none, none, 4).shape == (0, 2, 4)


def test_evict_shared_pages_stay():
    """Two sequences that share a prefix's pages: each is cut on its own, the shared
    pages keep their rows."""
    rng = np.random.default_rng(53)
    c = Cache(rng, [64, 40], 2, 64, 16, "bf16", weight=True, spare=4)
    c.table[1, :2] = c.table[0, :2]
    c.dev.table.copy_(torch.as_tensor(c.table))
    for x in (c.k, c.v):
        x[1] = np.concatenate([x[0][:32], x[1][32:]])
    out = c.other(rng, 24)
    old = c.dev.k.clone(), c.dev.v.clone()
    keep = F.focus_paged_evict(c.dev, out, 24, recent=4)
    _check(c, out, [24, 24], 4, keep, old)


def test_evict_captured_and_replayed():
    rng = np.random.default_rng(54)
    c = Cache(rng, [600, 90], 2, 64, 16, "bf16", weight=True, spare=20)
    out = c.other(rng, 64)
    old = c.dev.k.clone(), c.dev.v.clone()
    keep = torch.empty(2, 2, 64, dtype=torch.int32, device=DEV)
    n = F.focus_paged_evict_workspace(c.dev, out, 64, 8, keep)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)
    call = lambda: F.focus_paged_evict(c.dev, out, 64, recent=8, keep=keep, workspace=ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in range(3):
        c.dev.weight.copy_(torch.as_tensor(_weights(rng, c.weight.shape, ("ties", "skewed", "special")[i])))
        out.k.copy_(old[0])
        out.v.copy_(old[1])
        out.weight.fill_(-1.0)
        g.replay()
        torch.cuda.synchronize()
        _check(c, out, [64, 64], 8, keep, old)


@pytest.mark.parametrize("n,budget", [(300, 40), (9000, 5000), (40_000, 700)])
def test_evict_lengths_in_the_place_of_budgets(n, budget):
    """out.length is the tensor that holds the budgets, of as many sequences as there are
    heads to run beside each other."""
    announce(f"evict lengths over budgets {n} -> {budget}")
    rng = np.random.default_rng(n)
    lens = [n, 0, n // 2, budget, 7, n]
    c = Cache(rng, lens, 4, 64, 64, "bf16", weight=True, spare=len(lens) * (budget // 64 + 1))
    out = c.other(rng, budget)
    old = c.dev.k.clone(), c.dev.v.clone()
    budgets = [budget, 3, budget // 2, budget, 0, 1]
    out.length.copy_(torch.tensor(budgets, dtype=torch.int32))
    keep = F.focus_paged_evict(c.dev, out, out.length, recent=9)
    _check(c, out, budgets, 9, keep, old)


@pytest.mark.parametrize("batch,top,K,D,budget", [(40, 1000, 8, 64, 100), (70, 130, 4, 128, 130), (300, 60, 1, 64, 7),
                                                  (75, 4000, 4, 64, 600)])
@pytest.mark.parametrize("kind", ["skewed", "ties", "equal", "special"])
def test_evict_many_heads(batch, top, K, D, budget, kind):
    """More heads than the device has compute units, of every length up to top."""
    announce(f"evict {batch} x {top} x {K} x {D} budget {budget} {kind}")
    rng = np.random.default_rng(batch)
    lens = [top, 0, 1] + [int(x) for x in rng.integers(0, top + 1, batch - 3)]
    c = Cache(rng, lens, K, D, 64, "bf16", weight=True, spare=batch * -(-budget // 64))
    c.dev.weight.copy_(torch.as_tensor(_weights(rng, c.weight.shape, kind)))
    out = c.other(rng, budget)
    old = c.dev.k.clone(), c.dev.v.clone()
    keep = F.focus_paged_evict(c.dev, out, budget, recent=5)
    _check(c, out, [budget] * batch, 5, keep, old)


@pytest.mark.parametrize("kind", ["skewed", "ties", "special"])
def test_evict_long_tables_of_many_heads(kind):
    """Tables past what a workgroup holds, heads enough for half of the device: lengths of
    none to all, on and beside the rounds of 16 384 rows."""
    announce(f"evict long tables of many heads {kind}")
    rng = np.random.default_rng(71)
    lens = [0, 1, 33_000, 16_384, 16_385, 32_768, 20_000, 700] + [int(x) for x in rng.integers(0, 900, 24)]
    c = Cache(rng, lens, 4, 64, 1024, "bf16", weight=True, spare=32)
    c.dev.weight.copy_(torch.as_tensor(_weights(rng, c.weight.shape, kind)))
    out = c.other(rng, 500)
    old = c.dev.k.clone(), c.dev.v.clone()
    keep = F.focus_paged_evict(c.dev, out, 500, recent=20)
    _check(c, out, [500] * 32, 20, keep, old)


@pytest.mark.parametrize("dtype,K", [("f32", 4), ("f32", 3), ("bf16", 6)])
def test_evict_widest_rows(dtype, K):
    """Heads of 256 elements, copied by a launch of their own and by the selecting workgroup."""
    announce(f"evict widest rows {dtype} {K}")
    rng = np.random.default_rng(72)
    for budget in (9, 400):
        c = Cache(rng, [900, 31], K, 256, 16, dtype, weight=True, spare=2 * 25)
        out = c.other(rng, budget)
        old = c.dev.k.clone(), c.dev.v.clone()
        keep = F.focus_paged_evict(c.dev, out, budget, recent=4)
        _check(c, out, [budget] * 2, 4, keep, old)


@pytest.mark.parametrize("batch,K,cap", [(30, 4, 40_960), (100, 1, 66_560), (3, 1, 1 << 20)])
@pytest.mark.parametrize("kind", ["skewed", "ties"])
def test_evict_long_tables_in_larger_parts(batch, K, cap, kind):
    """Long tables of many rows in all, whose workgroups take more rows each; lengths on and
    beside the parts' ends, most sequences short."""
    announce(f"evict larger parts {batch} x {K} x {cap} {kind}")
    rng = np.random.default_rng(cap + batch)
    lens = [0, 32_769, 16_384] + [int(x) for x in rng.integers(0, 500, batch - 3)]
    lens[-1] = min(cap, 40_000)
    c = Cache(rng, lens, K, 64, 1024, "bf16", weight=True, max_pages=cap // 1024, spare=batch)
    c.dev.weight.copy_(torch.as_tensor(_weights(rng, c.weight.shape, kind)))
    out = c.other(rng, 700)
    old = c.dev.k.clone(), c.dev.v.clone()
    keep = F.focus_paged_evict(c.dev, out, 700, recent=33)
    _check(c, out, [700] * batch, 33, keep, old)


@pytest.mark.parametrize("lowest", [-np.inf, -3e38, -2.0 ** 127, -1.7e38])
@pytest.mark.parametrize("cap,recent", [(1024, 0), (2048, 0), (2048, 37), (4096, 5)])
def test_evict_keeps_all_rows_of_lowest_weights(cap, recent, lowest):
    """More heads than the device has compute units, and sequences that stay whole: in one
    head all weights are the lowest, in others one is, among sequences of every weight and
    some that are cut.  Lengths that fill a workgroup's registers, and one less or more."""
    announce(f"evict lowest weights {lowest} cap {cap} recent {recent}")
    rng = np.random.default_rng(cap + recent)
    lens = [cap, cap, 256 + recent, 1024, 512 + recent, 1024 - recent, 255, 257, cap - 1] + [3] * 58
    K = 4
    c = Cache(rng, lens, K, 8, 256, "bf16", weight=True, spare=len(lens) * (cap // 256))
    w = c.weight.copy()
    w[0, 0] = lowest
    for b, n in enumerate(lens):
        w[b, 1, n // 2] = lowest
        w[b, 2, :n:3] = lowest
    c.dev.weight.copy_(torch.as_tensor(w))
    out = c.other(rng, cap)
    budgets = [cap] * len(lens)
    budgets[1], budgets[6] = cap - 1, 254
    old = c.dev.k.clone(), c.dev.v.clone()
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    keep = F.focus_paged_evict(c.dev, out, torch.tensor(budgets, dtype=torch.int32, device=DEV), recent=recent, err=err)
    assert int(err.item()) == 0
    _check(c, out, budgets, recent, keep, old)


@pytest.mark.parametrize("budget", [12, 100])
@pytest.mark.parametrize("side", ["source", "destination"])
def test_evict_rows_of_bad_pages_are_not_copied(side, budget):
    """Kept rows whose own page, or the page they go to, lies outside the pool: reported,
    that place of out as it was, everything else copied."""
    announce(f"evict bad {side} page, budget {budget}")
    rng = np.random.default_rng(74)
    page, K = 8, 2
    c = Cache(rng, [120, 40], K, 64, page, "bf16", weight=True, max_pages=15)
    k = torch.full((30, page, K, 64), 9.0, dtype=torch.bfloat16, device=DEV)
    ids = rng.permutation(30)[:26].reshape(2, 13).astype(np.int32)
    out = F.PagedCache(k, k.clone(), torch.as_tensor(ids).to(DEV), torch.full((2,), -1, dtype=torch.int32, device=DEV),
                       torch.full((2, K, 104), -1.0, device=DEV))
    # rows 40 .. 47 of the first sequence stay, whatever else does
    c.weight[0, :, 40:48] = 5.0
    c.dev.weight.copy_(torch.as_tensor(c.weight))
    if side == "source":
        c.dev.table[0, 5] = 2 ** 31 - 1
    else:
        out.table[0, 0] = 30
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    keep = F.focus_paged_evict(c.dev, out, budget, recent=2, err=err).cpu().numpy()
    assert int(err.item()) == 2
    want = [np.full((30, page, K, 64), 9.0) for _ in range(2)]
    for b, n in enumerate(c.lens):
        for g in range(K):
            ref = P.keep(c.weight[b, g, :n], budget, 2)
            assert keep[b, g, :len(ref)].tolist() == ref
            missed = 0
            for j, r in enumerate(ref):
                if b == 0 and (40 <= r < 48 if side == "source" else j < page):
                    missed += 1
                    continue
                for w, rows in zip(want, (c.k[b], c.v[b])):
                    w[ids[b, j // page], j % page, g] = rows[r, g]
            assert b or missed == 8
    for w, now in zip(want, (out.k, out.v)):
        assert np.array_equal(now.double().cpu().numpy(), w)
    assert out.length.tolist() == [min(n, budget) for n in c.lens]


def test_evict_to_the_same_pages_of_another_pool():
    """One table for two pools: every page goes to the page of its number."""
    announce("evict one table, two pools")
    rng = np.random.default_rng(75)
    c = Cache(rng, [300, 77], 2, 64, 16, "bf16", weight=True)
    out = F.PagedCache(torch.full_like(c.dev.k, 9.0), torch.full_like(c.dev.v, 9.0), c.dev.table,
                       torch.full((2,), -1, dtype=torch.int32, device=DEV))
    old = out.k.clone(), out.v.clone()
    keep = F.focus_paged_evict(c.dev, out, 100, recent=7)
    _check(c, out, [100, 100], 7, keep, old)


@pytest.mark.parametrize("batch,K,cap", [(2, 1, 40_960), (33, 4, 36_864)])
@pytest.mark.parametrize("lowest", [-np.inf, -3e38])
def test_evict_long_tables_kept_whole(batch, K, cap, lowest):
    """Tables of more rows than a workgroup holds, whose sequences stay whole, the lowest
    weights among them; one of each is cut by a row."""
    announce(f"evict long tables kept whole {batch} x {K} x {cap} {lowest}")
    rng = np.random.default_rng(cap + batch)
    lens = [cap, cap - 1] + [int(x) for x in rng.choice([0, 1, 1024, 8192], batch - 2, p=[.3, .3, .39, .01])]
    c = Cache(rng, lens, K, 8, 1024, "bf16", weight=True, spare=batch * (cap // 1024))
    w = c.weight.copy()
    w[:, :, ::3] = lowest
    w[1, 0] = lowest
    c.dev.weight.copy_(torch.as_tensor(w))
    out = c.other(rng, cap)
    for recent, last in ((0, cap), (100, cap - 2)):
        budgets = [cap] * batch
        budgets[1] = last
        out.k.copy_(c.dev.k)
        out.weight.fill_(-1.0)
        old = c.dev.k.clone(), c.dev.v.clone()
        keep = F.focus_paged_evict(c.dev, out, torch.tensor(budgets, dtype=torch.int32, device=DEV), recent=recent)
        _check(c, out, budgets, recent, keep, old)


def test_evict_and_stored_rows_past_32_bits():
    """A pool of more than 2^32 bytes (2^31 elements): rows stored in its last pages, and cut
    to others of its last."""
    page, K, D = 64, 8, 128
    n_pages = (1 << 31) // (page * K * D) + 5
    announce(f"store and evict in a pool of {n_pages} pages")
    rng = np.random.default_rng(76)
    k = torch.empty(n_pages, page, K, D, dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    n = 2 * page - 3
    table = torch.tensor([[n_pages - 1, n_pages - 4]], dtype=torch.int32, device=DEV)
    cache = F.PagedCache(k, v, table, torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros(1, K, 2 * page, device=DEV))
    kn, vn = (torch.as_tensor(rng.standard_normal((n, K, D)).astype(np.float32)).to(torch.bfloat16).to(DEV) for _ in range(2))
    rows = torch.arange(n, dtype=torch.int32, device=DEV)
    F.focus_rope(rows, None, None, kn, vn, cache=cache, row_seq=torch.zeros_like(rows), row_slot=rows)
    assert cache.length.tolist() == [n]
    at = table[0].long()[rows.long() // page], rows.long() % page
    assert torch.equal(k[at], kn) and torch.equal(v[at], vn)
    w = rng.random((K, 2 * page)).astype(np.float32)
    cache.weight.copy_(torch.as_tensor(w)[None])
    out = F.PagedCache(k, v, torch.tensor([[n_pages - 2]], dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV))
    keep = F.focus_paged_evict(cache, out, 50, recent=5)
    for g in range(K):
        ref = P.keep(w[g, :n], 50, 5)
        assert keep[0, g].tolist() == ref
        for pool, new in ((k, kn), (v, vn)):
            assert torch.equal(pool[n_pages - 2, :50, g], new[torch.as_tensor(ref).to(DEV), g])


def test_evict_batch_past_the_grids_second_dimension():
    """33 000 short sequences."""
    announce("evict 33 000 sequences")
    batch, page = 33_000, 8
    g = torch.Generator(device=DEV).manual_seed(7)
    k = torch.randn(2 * batch, page, 1, 8, generator=g, device=DEV)
    ids = torch.randperm(2 * batch, generator=g, device=DEV).to(torch.int32).view(2, batch, 1)
    n = torch.randint(0, page + 1, (batch,), generator=g, device=DEV, dtype=torch.int32)
    w = torch.rand(batch, 1, page, generator=g, device=DEV)
    cache = F.PagedCache(k, k.clone(), ids[0].contiguous(), n, w)
    out = F.PagedCache(k, cache.v, ids[1].contiguous(), torch.zeros_like(n), torch.zeros_like(w))
    before = k.clone()
    keep = F.focus_paged_evict(cache, out, 5, recent=1).cpu().numpy()
    assert torch.equal(out.length, n.clamp(max=5))
    for b in range(0, batch, 97):
        ref = P.keep(w[b, 0, :int(n[b])].cpu().numpy(), 5, 1)
        assert keep[b, 0, :len(ref)].tolist() == ref and (keep[b, 0, len(ref):] == -1).all()
    rows = torch.as_tensor(keep[:, 0]).to(DEV).long()
    live = rows >= 0
    src, dst = before[ids[0, :, 0].long()], k[ids[1, :, 0].long()]
    got, want = dst[:, :5, 0], src[:, :, 0].gather(1, rows.clamp(min=0)[..., None].expand(-1, -1, 8))
    assert torch.equal(got[live], want[live])
    assert torch.equal(k[ids[0, :, 0].long()], src)
