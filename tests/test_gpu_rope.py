"""focus_rope on the GPU against the float64 oracle.

Tolerance: the angle's fraction is exact up to float64; what is rounded to float32 is
at most 1/8 turn (angle off by 0.8 x 2^-24), its sine and cosine (2 ulp), their product
with the amplitude, and the two products and the sum of each output: together below
2^-21 amplitude (|x| + |y|); bf16 outputs add half a step.  Elements that do not turn
are copied."""

import numpy as np
import pytest
import torch

import paper_2511_14694_amd as F
from gpu_util import DEV, announce, to64, torch_dtype
from oracle import paged as P
from paged_util import HALF_STEP, Cache, paged_rows, values, within

pytestmark = pytest.mark.gpu

PAIRS = {"interleaved": F.FOCUS_ROPE_INTERLEAVED, "half": F.FOCUS_ROPE_HALF}


def _tol(x, ref, rot, pairs, amplitude, dtype):
    re, im = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if pairs == "interleaved" else \
        (np.arange(rot // 2), np.arange(rot // 2, rot))
    tol = np.zeros_like(ref)
    both = abs(amplitude) * (np.abs(x[..., re]) + np.abs(x[..., im])) * 2.0 ** -21
    tol[..., re] = tol[..., im] = both
    tol[..., :rot] += HALF_STEP[dtype] * np.abs(ref[..., :rot]) * (1 + 2.0 ** -6) + 1e-38
    return tol


def _check(got, x, pos, turns, pairs, inverse, amplitude, dtype, what):
    ref = P.rope(x, pos, turns, pairs, inverse, amplitude)
    within(to64(got), ref, _tol(x, ref, 2 * len(turns), pairs, amplitude, dtype), what)


@pytest.mark.parametrize("rows,heads,kv,dim,rot,pairs,dtype", [
    (1, 32, 8, 128, 128, "half", "bf16"),
    (1, 1, 1, 64, 64, "interleaved", "f32"),
    (7, 3, 1, 64, 64, "half", "f32"),
    (33, 32, 8, 128, 128, "interleaved", "bf16"),
    (130, 12, 4, 96, 32, "half", "bf16"),
    (61, 5, 5, 80, 24, "half", "bf16"),        # half the turned part is 12 elements
    (61, 5, 5, 80, 20, "half", "f32"),
    (17, 2, 1, 8, 2, "half", "bf16"),
    (17, 2, 1, 8, 6, "interleaved", "bf16"),
    (9, 2, 2, 256, 256, "half", "f32"),
    (9, 4, 2, 256, 254, "interleaved", "bf16"),
    (300, 1, 1, 4, 4, "half", "f32"),
    (1025, 8, 2, 64, 64, "half", "bf16"),
])
@pytest.mark.parametrize("inverse", [False, True])
def test_rope_matches_oracle(rows, heads, kv, dim, rot, pairs, dtype, inverse):
    announce(f"rope {rows} x {heads}/{kv} x {dim} rot {rot} {pairs} {dtype} inverse {inverse}")
    rng = np.random.default_rng(rows + dim + rot)
    q, q64 = values(rng, (rows, heads, dim), dtype)
    k, k64 = values(rng, (rows, kv, dim), dtype)
    pos = rng.integers(-50, 3_000_000, rows).astype(np.int32)
    pos[0] = 2 ** 31 - 1
    pos[-1] = 0 if rows > 1 else 1_000_003
    turns = F.focus_rope_turns(rot, theta=10000.0)
    t64 = turns.cpu().numpy()
    qo, ko = F.focus_rope(torch.as_tensor(pos).to(DEV), turns, q, k, layout=PAIRS[pairs], inverse=inverse,
                          amplitude=1.125)
    _check(qo, q64, pos, t64, pairs, inverse, 1.125, dtype, "q")
    _check(ko, k64, pos, t64, pairs, inverse, 1.125, dtype, "k")
    assert np.array_equal(to64(q), q64) and np.array_equal(to64(k), k64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs", sorted(PAIRS))
def test_rope_views_in_place_and_one_input(pairs, dtype):
    """Views of one projection, outputs over the inputs, by-head outputs, q or k alone."""
    announce(f"rope views {pairs} {dtype}")
    rng = np.random.default_rng(11)
    n, H, K, D, rot = 37, 6, 2, 64, 32
    qkv, x = values(rng, (n, H + 2 * K, D), dtype)
    pos = rng.integers(0, 100_000, n).astype(np.int32)
    p = torch.as_tensor(pos).to(DEV)
    turns = F.focus_rope_turns(rot)
    t64 = turns.cpu().numpy()
    q, k = qkv[:, :H], qkv[:, H:H + K]
    by_head = torch.full((H, n, D), float("nan"), dtype=qkv.dtype, device=DEV)
    qo, ko = F.focus_rope(p, turns, q, k, layout=PAIRS[pairs], q_out=by_head.transpose(0, 1))
    _check(qo, x[:, :H], pos, t64, pairs, False, 1.0, dtype, "by head")
    assert qo.data_ptr() == by_head.data_ptr() and not torch.isnan(by_head.float()).any()
    alone, none = F.focus_rope(p, turns, q, layout=PAIRS[pairs])
    assert none is None and torch.equal(alone, qo)
    none, alone = F.focus_rope(p, turns, k=k, layout=PAIRS[pairs])
    assert none is None and torch.equal(alone, ko)
    F.focus_rope(p, turns, q, k, layout=PAIRS[pairs], q_out=q, k_out=k)
    assert torch.equal(q, qo) and torch.equal(k, ko)
    assert np.array_equal(to64(qkv[:, H + K:]), x[:, H + K:])
    same, _ = F.focus_rope(p, None, q)
    assert torch.equal(same, q)
    empty, _ = F.focus_rope(p[:0], turns, q[:0])
    assert empty.shape == (0, H, D)


def test_rope_values_that_are_not_finite_stay_in_their_pair():
    rng = np.random.default_rng(12)
    q, q64 = values(rng, (3, 2, 16), "f32")
    q[1, 0, 3] = float("nan")
    q[2, 1, 15] = float("inf")
    pos = torch.tensor([1, 2, 3], dtype=torch.int32, device=DEV)
    turns = F.focus_rope_turns(16)
    clean, _ = F.focus_rope(pos, turns, torch.as_tensor(q64).float().to(DEV))
    got, _ = F.focus_rope(pos, turns, q)
    hit = torch.zeros_like(got, dtype=torch.bool)
    hit[1, 0, 2:4] = True
    hit[2, 1, 14:] = True
    assert torch.equal(got[~hit], clean[~hit]) and not torch.isfinite(got[hit]).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs", ["half", "interleaved"])
@pytest.mark.parametrize("rot", [0, 2, 12, 20, 24, 32, 40])
def test_rope_elements_that_do_not_turn_keep_their_bits(rot, pairs, dtype):
    """Any bits at all, NaN with payloads among them; every width of piece."""
    announce(f"rope bits {rot} {pairs} {dtype}")
    rng = np.random.default_rng(rot)
    kind = np.uint16 if dtype == "bf16" else np.uint32
    bits = rng.integers(0, 1 << 8 * np.dtype(kind).itemsize, (77, 3, 64)).astype(kind)
    q = torch.as_tensor(bits.view(np.int16 if dtype == "bf16" else np.int32)).to(DEV).view(torch_dtype(dtype))
    pos = torch.arange(77, dtype=torch.int32, device=DEV)
    turns = F.focus_rope_turns(rot) if rot else None
    got, _ = F.focus_rope(pos, turns, q, layout=PAIRS[pairs])
    got = got.view(torch.int16 if dtype == "bf16" else torch.int32).cpu().numpy().view(kind)
    assert np.array_equal(got[..., rot:], bits[..., rot:])


def test_rope_gradient_against_differences():
    """The inverse call is the gradient of sum(g * rope(x)): against the formula's own
    differences in float64 (the map is linear, so a difference of any width is exact)."""
    rng = np.random.default_rng(13)
    n, H, D = 5, 2, 32
    x, x64 = values(rng, (n, H, D), "f32")
    g, g64 = values(rng, (n, H, D), "f32")
    pos = rng.integers(0, 1 << 20, n).astype(np.int32)
    turns = F.focus_rope_turns(24, scaling=F.FOCUS_ROPE_LINEAR, factor=4.0)
    t64 = turns.cpu().numpy()
    for pairs in PAIRS:
        dx, _ = F.focus_rope(torch.as_tensor(pos).to(DEV), turns, g, layout=PAIRS[pairs], inverse=True, amplitude=1.5)
        dx = to64(dx)
        loss = lambda y: (g64 * P.rope(y, pos, t64, pairs, amplitude=1.5)).sum()  # noqa: E731
        for idx in [(0, 0, 0), (1, 1, 13), (4, 0, 23), (2, 1, 24), (3, 0, 31)]:
            d = np.zeros_like(x64)
            d[idx] = 1.0
            ref = (loss(x64 + d) - loss(x64 - d)) / 2
            assert abs(dx[idx] - ref) <= 1.5 * 2 * np.abs(g64).max() * 2.0 ** -21 + 1e-12, (pairs, idx)


@pytest.mark.parametrize("dtype,page,by_head,padded", [("bf16", 16, False, False), ("f32", 8, True, False),
                                                       ("bf16", 64, False, True)])
@pytest.mark.parametrize("dim,rot", [(128, 128), (96, 40), (64, 0)])
def test_rope_stores_rows_in_pages(dtype, page, by_head, padded, dim, rot):
    announce(f"rope store {dtype} page {page} by_head {by_head} padded {padded} dim {dim} rot {rot}")
    rng = np.random.default_rng(page + dim)
    H, K = 4, 2
    lens = [5, 0, 3 * page - 1]
    c = Cache(rng, lens, K, dim, page, dtype, weight=True, by_head=by_head, padded=padded, max_pages=4)
    table = c.table.copy()
    table[1, 0] = c.free[0]              # room for the appended rows
    c.dev.table.copy_(torch.as_tensor(table))
    before_k, before_v = c.dev.k.clone(), c.dev.v.clone()
    # rows appended out of order to each sequence, one to none, two sequences interleaved
    seq = np.array([2, 0, 1, 0, 0, 2], np.int32)
    slot = np.array([3 * page - 1, 5, 0, 6, -1, 1], np.int32)
    n = len(seq)
    q, q64 = values(rng, (n, H, dim), dtype)
    k, k64 = values(rng, (n, K, dim), dtype)
    v, v64 = values(rng, (n, K, dim), dtype)
    pos = rng.integers(0, 50_000, n).astype(np.int32)
    turns = F.focus_rope_turns(rot) if rot else None
    t64 = turns.cpu().numpy() if rot else np.zeros(0)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    d = lambda a: torch.as_tensor(a).to(DEV)  # noqa: E731
    qo, ko = F.focus_rope(d(pos), turns, q, k, v, layout=PAIRS["half"], cache=c.dev, row_seq=d(seq), row_slot=d(slot),
                          err=err)
    assert ko is None and int(err.item()) == 0
    _check(qo, q64, pos, t64, "half", False, 1.0, dtype, "q")
    at = slot >= 0
    pid = torch.as_tensor(table[seq[at], slot[at] // page].astype(np.int64)).to(DEV)
    row = torch.as_tensor((slot[at] % page).astype(np.int64)).to(DEV)
    _check(c.dev.k[pid, row], k64[at], pos[at], t64, "half", False, 1.0, dtype, "k")
    assert np.array_equal(to64(c.dev.v[pid, row]), v64[at])
    # everything else as it was
    for now, was in ((c.dev.k, before_k), (c.dev.v, before_v)):
        now = now.clone()
        now[pid, row] = was[pid, row]
        assert torch.equal(now.nan_to_num(7.0), was.nan_to_num(7.0))
    assert c.dev.length.tolist() == [7, 1, 3 * page]
    w = c.weight.copy()
    w[seq[at], :, slot[at]] = 0.0
    assert np.array_equal(c.dev.weight.cpu().numpy(), w)
    # with k_out too: the same rows
    _, ko = F.focus_rope(d(pos), turns, None, k, v, layout=PAIRS["half"], k_out=torch.empty_like(k), cache=c.dev,
                         row_seq=d(seq), row_slot=d(slot))
    assert torch.equal(ko[torch.as_tensor(at)], c.dev.k[pid, row])


def test_rope_bad_rows_are_not_stored():
    rng = np.random.default_rng(21)
    page, K, D = 8, 2, 64
    c = Cache(rng, [3, 4], K, D, page, "bf16", max_pages=2, weight=True)
    c.dev.table[1, 1] = c.dev.k.shape[0]          # outside the pool
    k0, v0, w0 = c.dev.k.clone(), c.dev.v.clone(), c.dev.weight.clone()
    d = lambda a: torch.as_tensor(np.asarray(a, np.int32)).to(DEV)  # noqa: E731
    for seq, slot, bit in ((2, 0, 2), (-1, 0, 2), (0, 16, 1), (1, 9, 2), (0, 9, 2), (0, 2 ** 31 - 1, 1)):
        announce(f"rope bad row seq {seq} slot {slot}")
        err = torch.zeros(1, dtype=torch.int32, device=DEV)
        q, q64 = values(rng, (1, 2, D), "bf16")
        k, _ = values(rng, (1, K, D), "bf16")
        qo, ko = F.focus_rope(d([7]), F.focus_rope_turns(D), q, k, k, k_out=torch.empty_like(k), cache=c.dev,
                              row_seq=d([seq]), row_slot=d([slot]), err=err)
        assert int(err.item()) == bit
        _check(qo, q64, [7], F.focus_rope_turns(D).cpu().numpy(), "interleaved", False, 1.0, "bf16", "q")
        assert torch.equal(c.dev.k.nan_to_num(7.0), k0.nan_to_num(7.0))
        assert torch.equal(c.dev.v.nan_to_num(7.0), v0.nan_to_num(7.0))
        assert c.dev.length.tolist() == [3, 4] and torch.equal(c.dev.weight, w0)


def test_rope_agrees_with_the_fused_projection():
    """The rotation focus_qkv_project fuses into its store: the same pairs and angles
    (both round the same float32 products, from sums of different order)."""
    rng = np.random.default_rng(22)
    seq, W, kk, H, K, D, dm = [700], 500, 100, 2, 1, 128, 128
    tot = F.focus_layout_plan(seq, W, None, kk)
    lay = F.focus_layout(tot, seq, W, None, kk, device=DEV)
    hid, _ = values(rng, (tot.n_tokens, dm), "bf16")
    w, _ = values(rng, (dm, (H + 2 * K) * D), "bf16", dm ** -0.5)
    plain = F.focus_qkv_project(lay, hid, w, H, K, rope_theta=0.0)
    turned = F.focus_qkv_project(lay, hid, w, H, K)
    q, k = F.focus_rope(lay["tok_pos"], F.focus_rope_turns(D), plain[0], plain[1])
    for got, ref, raw in ((q, turned[0], plain[0]), (k, turned[1], plain[1])):
        # inputs rounded to bf16 before the rotation here: half a step of each of the
        # pair, and half a step of either output; the hardware sine there adds 2^-17
        x = to64(raw)
        pair = np.repeat(np.abs(x[..., 0::2]) + np.abs(x[..., 1::2]), 2, axis=-1)
        within(to64(got), to64(ref), pair * (2.0 ** -8 + 2.0 ** -16) + np.abs(to64(ref)) * 2.0 ** -7, "projection")


def test_rope_captured_and_replayed():
    rng = np.random.default_rng(23)
    n, H, K, D, page = 3, 4, 2, 64, 16
    c = Cache(rng, [4, 4, 4], K, D, page, "bf16", weight=True, max_pages=1)
    q, k, v = (values(rng, (n, h, D), "bf16")[0] for h in (H, K, K))
    d = lambda a: torch.as_tensor(np.asarray(a, np.int32)).to(DEV)  # noqa: E731
    pos, seq, slot, turns = d([9, 8, 7]), d([0, 1, 2]), d([4, 4, 4]), F.focus_rope_turns(D)
    qo = torch.empty_like(q)
    call = lambda: F.focus_rope(pos, turns, q, k, v, q_out=qo, cache=c.dev, row_seq=seq, row_slot=slot)  # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for step in range(3):
        q.copy_(values(rng, (n, H, D), "bf16")[0])
        slot.fill_(5 + step)
        g.replay()
        torch.cuda.synchronize()
        got = qo.clone()
        assert c.dev.length.tolist() == [6 + step] * 3
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, qo)


@pytest.mark.parametrize("rows,heads,kv,dim,rot,pairs,dtype", [
    (4_097, 1, 1, 64, 64, "half", "bf16"),             # two rows a workgroup, one in the last
    (17_003, 2, 1, 64, 32, "interleaved", "bf16"),     # eight, many of them in one step
    (17_001, 20, 3, 64, 64, "interleaved", "f32"),     # 16 heads a step: two steps a row
    (16_385, 37, 5, 64, 48, "half", "bf16"),           # 32 heads a step
    (9_001, 5, 2, 80, 40, "half", "bf16"),             # pieces of 8 bytes
    (8_195, 9, 1, 64, 20, "half", "bf16"),             # single elements, 4 heads a step
    (6_200, 3, 2, 64, 20, "half", "f32"),
    (12_300, 7, 7, 32, 6, "interleaved", "bf16"),      # pieces of two elements
    (6_147, 2, 2, 256, 256, "half", "f32"),
])
def test_rope_several_rows_a_workgroup(rows, heads, kv, dim, rot, pairs, dtype):
    """More rows than eight for each of 256 compute units: a workgroup takes several, the
    last one fewer."""
    announce(f"rope {rows} x {heads}/{kv} x {dim} rot {rot} {pairs} {dtype}")
    rng = np.random.default_rng(rows + dim + rot)
    q, q64 = values(rng, (rows, heads, dim), dtype)
    k, k64 = values(rng, (rows, kv, dim), dtype)
    pos = rng.integers(-50, 3_000_000, rows).astype(np.int32)
    turns = F.focus_rope_turns(rot)
    t64 = turns.cpu().numpy()
    p = torch.as_tensor(pos).to(DEV)
    qo, ko = F.focus_rope(p, turns, q, k, layout=PAIRS[pairs], amplitude=0.75)
    _check(qo, q64, pos, t64, pairs, False, 0.75, dtype, "q")
    _check(ko, k64, pos, t64, pairs, False, 0.75, dtype, "k")
    back, _ = F.focus_rope(p, turns, q, None, layout=PAIRS[pairs], inverse=True)
    _check(back, q64, pos, t64, pairs, True, 1.0, dtype, "inverse")
    F.focus_rope(p, turns, q, k, layout=PAIRS[pairs], amplitude=0.75, q_out=q, k_out=k)
    assert torch.equal(q, qo) and torch.equal(k, ko)


@pytest.mark.parametrize("page,K,dtype,by_head", [(16, 3, "bf16", False), (64, 1, "f32", True), (8, 8, "bf16", True)])
def test_rope_stores_many_ragged_rows(page, K, dtype, by_head):
    """A ragged batch of some thousand rows, several rows a workgroup: runs that cross
    workgroups and sequences, rows not stored and rows that cannot be among them, single
    rows out of order, one sequence of them alone."""
    announce(f"rope ragged store page {page} K {K} {dtype} by_head {by_head}")
    rng = np.random.default_rng(page + K)
    H, dim, rot = 4, 64, 32
    lens = [0, 5, 3000, 1, 4100, 17, 0, 1900]
    cap = 4200
    c = Cache(rng, [0] * len(lens), K, dim, page, dtype, weight=True, by_head=by_head, max_pages=-(-cap // page),
              spare=sum(-(-n // page) for n in lens) + 2)
    table = c.table.copy()
    for b, n in enumerate(lens):
        for j in range(-(-n // page)):
            table[b, j] = c.free.pop()
    table[2, 20] = -1                                  # pages outside the pool
    table[7, 3] = c.dev.k.shape[0]
    c.dev.table.copy_(torch.as_tensor(table))
    seq = np.concatenate([np.full(n, b) for b, n in enumerate(lens)])
    slot = np.concatenate([np.arange(n) for n in lens])
    n = len(seq)
    assert n > 8192
    tail = rng.permutation(np.flatnonzero(seq == 7))   # the last sequence out of order
    slot[seq == 7] = slot[tail]
    skip = rng.random(n) < 0.02
    skip[np.flatnonzero(seq == 4)[-3:]] = True         # a length that ends before the run does
    slot = np.where(skip, -1 - rng.integers(0, 5, n), slot)
    bad_seq = (rng.random(n) < 0.01) & ~skip
    seq = np.where(bad_seq, rng.choice([-1, len(lens), 2 ** 31 - 1], n), seq)
    past = (rng.random(n) < 0.01) & ~skip & ~bad_seq
    slot = np.where(past, table.shape[1] * page + rng.integers(0, 9, n), slot)
    seq, slot = seq.astype(np.int32), slot.astype(np.int32)
    ok = ~skip & ~bad_seq & ~past
    pid = np.full(n, -1)
    pid[ok] = table[seq[ok], slot[ok] // page]
    stored = ok & (pid >= 0) & (pid < c.dev.k.shape[0])
    assert (ok & ~stored).any()
    q, q64 = values(rng, (n, H, dim), dtype)
    k, k64 = values(rng, (n, K, dim), dtype)
    v, v64 = values(rng, (n, K, dim), dtype)
    pos = rng.integers(0, 1_000_000, n).astype(np.int32)
    turns = F.focus_rope_turns(rot)
    t64 = turns.cpu().numpy()
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    before = c.dev.k.clone(), c.dev.v.clone()
    d = lambda a: torch.as_tensor(a).to(DEV)  # noqa: E731
    qo, ko = F.focus_rope(d(pos), turns, q, k, v, k_out=torch.empty_like(k), cache=c.dev, row_seq=d(seq),
                          row_slot=d(slot), err=err)
    assert int(err.item()) == 3
    _check(qo, q64, pos, t64, "interleaved", False, 1.0, dtype, "q")
    _check(ko, k64, pos, t64, "interleaved", False, 1.0, dtype, "k")
    at = d(pid[stored].astype(np.int64)), d((slot[stored] % page).astype(np.int64))
    assert torch.equal(c.dev.k[at], ko[d(stored)])
    assert np.array_equal(to64(c.dev.v[at]), v64[stored])
    for now, was in zip((c.dev.k, c.dev.v), before):
        now = now.clone()
        now[at] = was[at]
        assert torch.equal(now.nan_to_num(7.0), was.nan_to_num(7.0)), "other rows were written"
    ends = [int(slot[stored & (seq == b)].max(initial=-1)) + 1 for b in range(len(lens))]
    assert c.dev.length.tolist() == ends
    w = c.weight.copy()
    w[seq[stored], :, slot[stored]] = 0.0
    assert np.array_equal(c.dev.weight.cpu().numpy(), w)


def test_rope_offsets_past_32_bits():
    """q of more than 2^31 elements, in place: its last rows as by themselves."""
    n, H, D = 66_000, 256, 128
    announce(f"rope {n} x {H} x {D} in place")
    q = torch.empty(n, H, D, dtype=torch.bfloat16, device=DEV)
    assert q.numel() > 1 << 31
    g = torch.Generator(device=DEV).manual_seed(5)
    ends = [slice(0, 9), slice(65_530, 65_540), slice(n - 9, n)]
    for at in ends:
        q[at] = torch.randn(q[at].shape, generator=g, device=DEV).to(torch.bfloat16)
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    turns = F.focus_rope_turns(D)
    want = [F.focus_rope(pos[at], turns, q[at].clone())[0] for at in ends]
    F.focus_rope(pos, turns, q, q_out=q)
    for at, x in zip(ends, want):
        assert torch.equal(q[at], x)
