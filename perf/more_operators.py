"""Performance cases of the 8-bit paged cache's operators on one GPU.

    extend   slots for new rows of a batch of sequences taken from a list of free pages,
             those of dropped rows given back: page tables, lengths and slot maps
    append   new rows of k and v stored in a paged cache in 8 bits (e4m3), with one scale,
             a power of two, for each block of rows and head
    attend   attention of the newest tokens of every sequence (one, or a few drafted ones
             at once) over such a cache

run() computes an operator in elementary torch operations (float32) or, with `own`,
through the package's public functions, on the buffers that a serving program keeps
between calls (pages, scales, page tables, lengths, free pages).
"""

from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
E4M3 = torch.float8_e4m3fn
MOST = 448.0    # the largest e4m3 number


def _extend(name, batch, rows, add, page=16):
    """batch sequences of 0 to rows cached rows; in the first call the even ones take slots
    for 1 to add rows (spread over the logarithm) and the odd ones drop as many, in the
    second the other way round."""
    c = dict(kind="extend", batch=batch, rows=rows, add=add, page=page)
    return dict(c, name=name) if name else c


def _append(name, batch, rows, add, kv_heads, dim=128, page=64, block=16, dtype="bf16", fused=False, by_head=False):
    """add rows (spread over the logarithm where more than one) behind 0 to rows cached ones
    of batch sequences, a scale for every block rows; fused: k and v are views of one
    projection; by_head: pages laid out [H_kv, page, D] instead of [page, H_kv, D]."""
    c = dict(kind="append", batch=batch, rows=rows, add=add, kv_heads=kv_heads, dim=dim, page=page, block=block,
             dtype=dtype, fused=fused, by_head=by_head)
    return dict(c, name=name) if name else c


def _attend(name, batch, rows, heads, kv_heads, dim=128, page=64, block=16, dtype="bf16", new=1, ragged=False,
            by_head=False):
    """The newest `new` tokens of batch sequences of rows cached rows each (ragged: new to
    rows, spread over the logarithm, and 1 to new tokens); dtype of q and o."""
    c = dict(kind="attend", batch=batch, rows=rows, heads=heads, kv_heads=kv_heads, dim=dim, page=page, block=block,
             dtype=dtype, new=new, ragged=ragged, by_head=by_head)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a decode step of a serving batch: a few drafted tokens taken, a few rejected ones dropped
        _extend("extend_step_b64", 64, 8_192, 4),
        # a round of admissions: a long ragged batch of prompts comes, finished sequences go
        _extend("extend_admit_b500", 500, 1_000, 4_095, page=64),
        # the new token of each of 64 sequences, into blocks that hold rows already
        _append("append_step_b64", 64, 8_192, 1, 8, fused=True),
        # all rows of a 100 kb prefill of 32 heads
        _append("append_prefill_100kb", 1, 0, 101_000, 32, page=64, block=32),
        # float32 heads of 96, odd lengths, pages laid out by head, a scale for eight rows
        _append("append_part_f32", 7, 1_021, 1_023, 3, dim=96, page=32, block=8, dtype="f32", by_head=True),
        # interactive decode early in a text: one sequence, a few pages
        _attend("attend_b1_137", 1, 137, 32, 8),
        # a batch of 16 behind 10 000 retained rows (about 1 Mb), a key head per query head
        _attend("attend_b16_1mb", 16, 10_000, 32, 32, block=32),
        # a serving batch of uneven lengths on small pages
        _attend("attend_b64_ragged", 64, 8_192, 32, 8, page=16, ragged=True),
        # one long cache: all parallelism comes from splitting its length
        _attend("attend_b1_262k", 1, 262_144, 32, 8, page=128, block=64),
        # up to five drafted tokens of 32 sequences looked at together
        _attend("attend_draft_b32", 32, 16_384, 32, 8, new=5, ragged=True),
        # float32 heads of 64, an odd batch, odd lengths, pages laid out by head
        _attend("attend_b3_f32", 3, 2_021, 6, 2, dim=64, page=32, block=8, dtype="f32", new=2, ragged=True, by_head=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    kind = rng.choice(["extend", "append", "append", "attend", "attend", "attend"])
    page = rng.choice([16, 16, 32, 64, 128, 256])
    if kind == "extend":
        batch = _log_int(rng, 1, 1_500)
        return _extend("", batch, _log_int(rng, 1, 20_000), _log_int(rng, 1, min(8_000, 1_600_000 // batch)), page)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    es = 2 if dtype == "bf16" else 4
    kv = rng.choice([1, 2, 3, 4, 8, 8, 16, 32])
    block = rng.choice([b for b in (8, 16, 16, 32, 64, 256) if b <= page])
    batch = _log_int(rng, 1, 128)
    by_head = rng.random() < 0.3
    if kind == "append":
        dim = rng.choice([64, 96, 128, 128, 256])
        most = int(4.0e8 // (kv * dim * es * batch))
        add = 1 if rng.random() < 0.3 else _log_int(rng, 1, max(1, min(100_000, most)))
        return _append("", batch, _log_int(rng, 1, max(1, min(4_000, most))), add, kv, dim, page, block, dtype,
                       rng.random() < 0.5, by_head)
    dim = rng.choice([64, 128, 128])
    heads = kv * rng.choice([g for g in (1, 2, 3, 4, 6, 8, 16) if g * kv <= 128])
    new = rng.choice([1, 1, 1, 2, 3, 4, 5, 8])
    # (a matrix product takes 16 columns: more query heads of a key head cost more)
    most = int(1.2e9 / (2 * kv * dim * batch) / max(1.0, new * heads / kv / 16))
    rows = _log_int(rng, new, max(new, min(262_144, most)))
    return _attend("", batch, rows, heads, kv, dim, page, block, dtype, new, rng.random() < 0.6, by_head)


# ------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 6151 + 443)
    return g


def _randn(g, shape, dtype, scale=1.0):
    return (torch.randn(tuple(shape), generator=g, dtype=torch.float32, device=DEV) * scale).to(dtype)


def _spread(n, lo, hi):
    """n sizes from hi down to about lo, spread over the logarithm: a plain formula, so that
    every seed of a case does the same work."""
    return [max(lo, int(round(hi * (lo / hi) ** (i / max(1, n))))) for i in range(n)]


def _before(case):
    """Cached rows before the call: multiples of nothing in particular, 0 to rows."""
    n, rows = case["batch"], case["rows"]
    return [(rows * (2 * b + 1) // (2 * n) + 5 * b) % (rows + 1) for b in range(n)]


def _added(case):
    return [case["add"]] * case["batch"] if case["add"] == 1 else _spread(case["batch"], 1, case["add"])


def _attended(case):
    """Rows and new tokens of each sequence."""
    n, rows, new = case["batch"], case["rows"], case["new"]
    if not case["ragged"]:
        return [rows] * n, [new] * n
    return _spread(n, new, rows), [1 + (3 * b + new - 1) % new for b in range(n)]


def _tables(g, need, width, spare):
    """Pages in random order: a table [batch, width] (-1 past a sequence's last page) and
    the pages that are left."""
    total = sum(need)
    order = torch.randperm(total + spare, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(need), width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    return table, order[at:].clone()


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _offsets(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _pool(g, pages, case):
    """A pool's k or v with its scales: normal values, each block and head at a magnitude of
    its own within two binades, the largest of a block near the end of the 8-bit range."""
    kv, D, page, block = case["kv_heads"], case["dim"], case["page"], case["block"]
    scale = torch.exp2(torch.randint(-8, -5, (pages, kv, page // block), generator=g, device=DEV).float())
    x = torch.empty((pages, kv, page, D) if case["by_head"] else (pages, page, kv, D), dtype=E4M3, device=DEV)
    for p in range(0, pages, 512):
        part = x[p:p + 512]
        x[p:p + 512] = (torch.randn(part.shape, generator=g, device=DEV) * 90.0).clamp(-MOST, MOST).to(E4M3)
    return (x.transpose(1, 2) if case["by_head"] else x), scale


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    page = case["page"]
    if case["kind"] == "extend":
        before, add = _before(case), _spread(case["batch"], 1, case["add"])
        # an odd sequence's rows to drop are cached, an even one's to take are not
        s["length"] = _int32([n + (a if b % 2 else 0) for b, (n, a) in enumerate(zip(before, add))])
        s["add"] = [_int32([-a if (b + call) % 2 else a for b, a in enumerate(add)]) for call in range(2)]
        s["rows"] = [sum(a for b, a in enumerate(add) if b % 2 == call) for call in range(2)]
        width = max(-(-(n + a) // page) for n, a in zip(before, add)) + 1
        need = [-(-n // page) for n in s["length"].tolist()]
        extra = sum(-(-(n + a) // page) for n, a in zip(before, add)) + 3
        s["table"], free = _tables(g, need, width, extra)
        s["free_pages"] = torch.cat((free, torch.full((sum(need),), -1, dtype=torch.int32, device=DEV)))
        s["free_count"] = _int32([free.numel()])
        s["first_pos"] = torch.randint(0, 1_000_000, (case["batch"],), generator=g, device=DEV).to(torch.int32)
        return s
    dt, D, kv = DTYPES[case["dtype"]], case["dim"], case["kv_heads"]
    if case["kind"] == "append":
        before, add = _before(case), _added(case)
        lens, counts = [n + a for n, a in zip(before, add)], add
        n = sum(add)
        # elements of a row and head at a magnitude of their own
        if case["fused"]:
            both = _randn(g, (n, 2 * kv, D), dt)
            both *= torch.exp2(torch.randint(-3, 3, (n, 2 * kv, 1), generator=g, device=DEV).float()).to(dt)
            s["k"], s["v"] = both[:, :kv], both[:, kv:]
        else:
            for name in ("k", "v"):
                s[name] = _randn(g, (n, kv, D), dt)
                s[name] *= torch.exp2(torch.randint(-3, 3, (n, kv, 1), generator=g, device=DEV).float()).to(dt)
        s["start"] = _int32(before)
    else:
        lens, counts = _attended(case)
        s["q"] = _randn(g, (sum(counts), case["heads"], D), dt, 1.5)
    need = [-(-n // page) for n in lens]
    s["table"], _ = _tables(g, need, max(need), 1)
    pages = sum(need) + 1
    s["pk"], s["k_scale"] = _pool(g, pages, case)
    s["pv"], s["v_scale"] = _pool(g, pages, case)
    s["length"] = _int32(lens)
    s["cu_rows"] = _int32(_offsets(counts))
    return s


# ------------------------------------------------------- the operators' calls

def _own_run(s):
    import paper_2511_14694_amd as F
    c = s["case"]
    if c["kind"] == "extend":
        took = [F.focus_paged_extend(s["table"], s["length"], c["page"], s["add"][call], s["free_pages"], s["free_count"],
                                     s["rows"][call], first_pos=s["first_pos"]) for call in range(2)]
        return {"first": [took[0].start, took[0].cu_rows, took[0].row_seq, took[0].row_slot, took[0].row_pos],
                "second": [took[1].start, took[1].cu_rows, took[1].row_seq, took[1].row_slot, took[1].row_pos],
                "table": s["table"], "length": s["length"], "free_pages": s["free_pages"], "free_count": s["free_count"]}
    cache = F.PagedCache8(s["pk"], s["pv"], s["k_scale"], s["v_scale"], s["table"], s["length"])
    if c["kind"] == "append":
        F.focus_paged_append(s["k"], s["v"], cache, s["start"], cu_rows=s["cu_rows"])
        return {"pages_k": s["pk"], "pages_v": s["pv"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    o, lse = F.focus_paged_attend(s["q"], cache, cu_rows=s["cu_rows"], max_rows=c["new"])
    return {"o": o, "lse": lse}


# ----------------------------------------------------------- the plain forms

def _up(a, b):
    return torch.div(a + (b - 1), b, rounding_mode="floor")


def _plain_extend_call(s, add, n_rows):
    table, length, free, page = s["table"], s["length"].long(), s["free_pages"], s["case"]["page"]
    width, slots = table.shape[1], free.numel()
    add = add.long()
    j = torch.arange(width, device=DEV)
    have = _up(length, page)
    # pages of dropped rows go behind the free ones
    left = (length + add).clamp(min=0)
    keep = torch.where(add < 0, _up(left, page), have)
    back = have - keep
    count = s["free_count"].long()
    gone = (j >= keep[:, None]) & (j < have[:, None])
    to = count + (torch.cumsum(back, 0) - back)[:, None] + (j - keep[:, None])
    to = torch.where(gone, to, torch.full_like(to, slots)).clamp(max=slots)
    spare = torch.cat((free, free.new_zeros(1)))
    spare.scatter_(0, to.flatten(), table.flatten())
    free.copy_(spare[:slots])
    table.copy_(torch.where(gone, torch.full_like(table, -1), table))
    count = (count + back.sum()).clamp(max=slots)
    # pages for new rows come from the end
    rows = add.clamp(min=0)
    cu = torch.cat((rows.new_zeros(1), torch.cumsum(rows, 0)))
    fits = (rows > 0) & (length + rows <= width * page) & (cu[1:] <= n_rows)
    need = torch.where(fits, _up(length + rows, page) - have, torch.zeros_like(have))
    upto = torch.cumsum(need, 0)
    served = fits & ((need == 0) | (upto <= count))
    first = count - 1 - (upto - need)
    new = served[:, None] & (j >= have[:, None]) & (j < (have + need)[:, None])
    at = (first[:, None] - (j - have[:, None])).clamp(0, max(slots - 1, 0))
    table.copy_(torch.where(new, free[at], table))
    took = torch.where(served & (need > 0), upto, torch.zeros_like(upto)).amax()
    s["free_count"].copy_((count - took).to(torch.int32))
    start = torch.where(rows > 0, torch.where(served, length, torch.full_like(length, -1)), left)
    s["length"].copy_(torch.where(rows > 0, torch.where(served, length + rows, length), left).to(torch.int32))
    t = torch.arange(n_rows, device=DEV)
    seq = torch.searchsorted(cu[1:].contiguous(), t, right=True).clamp(max=len(rows) - 1)
    i = t - cu[seq]
    slot = torch.where(served[seq], start[seq] + i, torch.full_like(i, -1))
    return [x.to(torch.int32) for x in (start, cu, seq, slot, s["first_pos"].long()[seq] + i)]


def _plain_extend(s):
    first, second = (_plain_extend_call(s, s["add"][call], s["rows"][call]) for call in range(2))
    return {"first": first, "second": second, "table": s["table"], "length": s["length"], "free_pages": s["free_pages"],
            "free_count": s["free_count"]}


def _power_of_two(most):
    """The least 2^e, e >= -126, with most <= 448 2^e (448 = 0.875 2^9)."""
    m, e = torch.frexp(most)
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(min=-126)
    return torch.ldexp(torch.ones_like(most), e)


def _plain_append(s):
    c = s["case"]
    page, block, kv = c["page"], c["block"], c["kv_heads"]
    per = page // block
    start, cu = s["start"].long(), s["cu_rows"].long()
    t = torch.arange(s["k"].shape[0], device=DEV)
    seq = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    slot = start[seq] + t - cu[seq]
    at, x = s["table"][seq, slot // page].long(), slot % page
    blk = at * per + x // block
    # blocks that hold rows before the first new one: their scale does not shrink
    tail = (start % block > 0) & (cu[1:] > cu[:-1])
    tail_page = s["table"].gather(1, (start // page)[:, None].clamp(max=s["table"].shape[1] - 1))[:, 0].long().clamp(min=0)
    tail_blk = tail_page * per + start % page // block
    r = torch.arange(block, device=DEV)
    old = (tail[:, None] & (r < (start % block)[:, None]))[..., None, None]    # rows before the first new one
    old_at = tail_page[:, None], (start % page // block * block)[:, None] + r
    out = {}
    for name, pool, scales, rows in (("k", s["pk"], s["k_scale"], s["k"]), ("v", s["pv"], s["v_scale"], s["v"])):
        flat = scales.transpose(1, 2).reshape(-1, kv)                     # [blocks, H_kv], a copy
        most = torch.zeros_like(flat)
        row_most = rows.float().abs().amax(-1)
        most.scatter_reduce_(0, blk[:, None].expand(-1, kv), row_most, "amax")
        new = _power_of_two(most)
        kept = torch.zeros_like(flat)
        kept[tail_blk] = torch.where(tail[:, None], flat[tail_blk], torch.zeros_like(flat[tail_blk]))
        new = torch.maximum(new, kept)
        was = pool[old_at].float()                                        # [batch, block, H_kv, D]
        ratio = (flat[tail_blk] / new[tail_blk])[:, None, :, None]
        pool[old_at] = torch.where(old, was * ratio, was).to(E4M3)
        pool[at, x] = (rows.float() / new[blk][..., None]).to(E4M3)
        touched = torch.zeros(flat.shape[0], dtype=torch.bool, device=DEV)
        touched[blk] = True
        flat = torch.where(touched[:, None], new, flat)
        scales.copy_(flat.reshape(-1, per, kv).transpose(1, 2))
        out["pages_" + name], out[name + "_scale"] = pool, scales
    return out


def _plain_attend(s):
    c = s["case"]
    H, kv, D, page, block, new = c["heads"], c["kv_heads"], c["dim"], c["page"], c["block"], c["new"]
    G, B = H // kv, c["batch"]
    cu = s["cu_rows"].long()
    count = cu[1:] - cu[:-1]
    i = torch.arange(new, device=DEV)
    there = i < count[:, None]                                           # [B, new]
    row = (cu[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)
    q = s["q"].float()[row].view(B, new, kv, G, D)
    pages = s["table"].clamp(min=0).long()
    cap = pages.shape[1] * page
    seen = torch.arange(cap, device=DEV) < (s["length"].long()[:, None] - (count[:, None] - 1 - i))[..., None]
    o = torch.zeros_like(s["q"])
    lse = torch.zeros(s["q"].shape[:2], device=DEV)
    # a few sequences at a time: their rows in float32
    for b0 in range(0, B, max(1, int(3.0e8 // (cap * kv * D)))):
        b1 = min(B, b0 + max(1, int(3.0e8 // (cap * kv * D))))
        part = []
        for pool, scales in ((s["pk"], s["k_scale"]), (s["pv"], s["v_scale"])):
            x = pool[pages[b0:b1]].float()                               # [b, pages, page, H_kv, D]
            f = scales[pages[b0:b1]].repeat_interleave(block, -1).transpose(-1, -2)
            part.append((x * f[..., None]).reshape(b1 - b0, cap, kv, D))
            del x
        k = part[0].permute(0, 2, 3, 1).contiguous()
        x = torch.matmul(q[b0:b1].permute(0, 2, 1, 3, 4).reshape(b1 - b0, kv, new * G, D), k) * (D ** -0.5)
        x = x.view(b1 - b0, kv, new, G, cap)
        look = seen[b0:b1][:, None, :, None]
        x = torch.where(look, x, torch.full_like(x, -math.inf))
        top = x.amax(-1, keepdim=True)
        e = torch.where(look, torch.exp(x - top), torch.zeros_like(x))
        total = e.sum(-1, keepdim=True)
        y = torch.matmul((e / total).view(b1 - b0, kv, new * G, cap), part[1].transpose(1, 2).contiguous())
        y = y.view(b1 - b0, kv, new, G, D).transpose(1, 2).reshape(b1 - b0, new, H, D)
        z = (top + torch.log(total)).view(b1 - b0, kv, new, G).transpose(1, 2).reshape(b1 - b0, new, H)
        for n in range(new):
            at = torch.where(there[b0:b1, n], row[b0:b1, n], row[b0:b1, 0])
            m = n if new > 1 else 0
            o[at] = torch.where(there[b0:b1, n, None, None], y[:, m].to(o.dtype), o[at])
            lse[at] = torch.where(there[b0:b1, n, None], z[:, m], lse[at])
    return {"o": o, "lse": lse}


def run(s):
    if own:
        return _own_run(s)
    return {"extend": _plain_extend, "append": _plain_append, "attend": _plain_attend}[s["case"]["kind"]](s)


# ------------------------------------------------------------------- bounds

def work(case):
    page = case["page"]
    if case["kind"] == "extend":
        before, add = _before(case), _spread(case["batch"], 1, case["add"])
        pages = sum(-(-(n + a) // page) - -(-n // page) for n, a in zip(before, add))
        # both calls: three maps of the rows taken, pages out of the list and into a table
        # and back, the lengths, counts and offsets of the sequences
        return {"bytes": 12 * sum(add) + 16 * pages + 2 * 24 * case["batch"], "flops": 0}
    D, kv, es = case["dim"], case["kv_heads"], 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "append":
        add = _added(case)
        blocks = sum(-(-(n + a) // case["block"]) - n // case["block"] for n, a in zip(_before(case), add))
        return {"bytes": 2 * kv * (sum(add) * D * (es + 1) + 4 * blocks), "flops": 0}
    lens, new = _attended(case)
    H = case["heads"]
    pairs = sum(n * m - m * (m - 1) // 2 for n, m in zip(lens, new))
    blocks = sum(-(-n // case["block"]) for n in lens)
    return {"bytes": 2 * kv * (sum(lens) * D + 4 * blocks) + sum(new) * H * (2 * D * es + 4), "flops": 4 * pairs * H * D}


# --------------------------------------------------- the definition, 64 bits

def _exact_extend(s):
    page = s["case"]["page"]
    table, length = s["table"].tolist(), s["length"].tolist()
    free, count = s["free_pages"].tolist(), int(s["free_count"].item())
    pos = s["first_pos"].tolist()
    outs = []
    for add in (s["add"][0].tolist(), s["add"][1].tolist()):
        start = [0] * len(add)
        for b, a in enumerate(add):                      # dropped rows first
            if a <= 0:
                n = max(length[b] + a, 0)
                for j in range(-(-n // page), -(-length[b] // page)):
                    free[count] = table[b][j]
                    table[b][j] = -1
                    count += 1
                length[b] = start[b] = n
        cu, seq, slot, at = [0], [], [], []
        dry = False                                      # a sequence did not get its pages
        for b, a in enumerate(add):
            a = max(a, 0)
            cu.append(cu[-1] + a)
            if a == 0:
                continue
            have, want = -(-length[b] // page), -(-(length[b] + a) // page)
            ok = want <= len(table[b])
            if ok and want > have:
                dry = dry or want - have > count
                ok = not dry
            for j in range(have, want if ok else have):
                count -= 1
                table[b][j] = free[count]
            start[b] = length[b] if ok else -1
            seq += [b] * a
            slot += [start[b] + i if ok else -1 for i in range(a)]
            at += [pos[b] + i for i in range(a)]
            length[b] += a if ok else 0
        outs.append([_int32(x) for x in (start, cu, seq, slot, at)])
    return {"first": outs[0], "second": outs[1], "table": _int32(table), "length": _int32(length),
            "free_pages": _int32(free), "free_count": _int32([count])}


def _nearest(x):
    """The nearest e4m3 number, ties to the even one: steps of 2^-9 below 2^-6, above them
    of an eighth of the power of two below the number."""
    low = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(low - 3.0)
    return torch.round(x / step) * step


def _exact_append(s):
    c = s["case"]
    page, block = c["page"], c["block"]
    out = {}
    for name, pool, scales, rows in (("k", s["pk"], s["k_scale"], s["k"]), ("v", s["pv"], s["v_scale"], s["v"])):
        p8, sc = pool.double(), scales.double()
        cu, before, table = s["cu_rows"].tolist(), s["start"].tolist(), s["table"].tolist()
        for b in range(c["batch"]):
            n0, n1 = before[b], before[b] + cu[b + 1] - cu[b]
            # the sequence's blocks that get rows, whole: [blocks, block, H_kv, D]
            first, last = n0 // block, -(-n1 // block)
            x = torch.zeros((last - first) * block, *rows.shape[1:], dtype=torch.float64, device=DEV)
            x[n0 - first * block:n1 - first * block] = rows[cu[b]:cu[b + 1]].double()
            x = x.view(last - first, block, *rows.shape[1:])
            most = x.abs().amax((1, 3))
            e = torch.ceil(torch.log2((most / MOST).clamp(min=2.0 ** -126)))
            new = torch.exp2(e)
            blocks = torch.arange(first, last, device=DEV)
            at = torch.tensor(table[b], device=DEV)[blocks * block // page], blocks * block % page // block
            old = n0 % block
            if old:
                was = sc[at[0][0], :, at[1][0]]
                new[0] = torch.maximum(new[0], was)
                r = at[1][0] * block + torch.arange(old, device=DEV)
                x[0, :old] = p8[at[0][0], r] * was[:, None]
            y = _nearest(x / new[:, None, :, None]).flatten(0, 1)
            r = torch.arange(first * block, n1, device=DEV)
            p8[torch.tensor(table[b], device=DEV)[r // page], r % page] = y[:len(r)]
            sc[at[0], :, at[1]] = new
        out["pages_" + name], out[name + "_scale"] = p8, sc
    return out


def _exact_attend(s):
    c = s["case"]
    H, kv, D, page, block = c["heads"], c["kv_heads"], c["dim"], c["page"], c["block"]
    G = H // kv
    cu = s["cu_rows"].tolist()
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    for b, n in enumerate(s["length"].tolist()):
        r = torch.arange(n, device=DEV)
        at = s["table"][b].long()[r // page], r % page
        new = cu[b + 1] - cu[b]
        for g in range(kv):
            k, v = (pool[at[0], at[1], g].double() * scales[at[0], g, at[1] // block].double()[:, None]
                    for pool, scales in ((s["pk"], s["k_scale"]), (s["pv"], s["v_scale"])))
            for i in range(new):
                m = n - (new - 1 - i)
                hs = slice(g * G, (g + 1) * G)
                q = s["q"][cu[b] + i, hs].double()
                x = torch.mm(k[:m], q.t().contiguous()) / math.sqrt(D)       # [m, G]
                z = torch.logsumexp(x, 0)
                lse[cu[b] + i, hs] = z
                o[cu[b] + i, hs] = torch.mm(torch.exp(x - z).t().contiguous(), v[:m])
    return {"o": o, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    return {"extend": _exact_extend, "append": _exact_append, "attend": _exact_attend}[case["kind"]](s)
