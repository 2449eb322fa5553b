"""CPU checks of the 8-bit paged cache's calls: host validation refuses bad descriptors before
any launch (no GPU is touched), the binding refuses tensors that do not fit, fills every field
of its descriptors, and allocates on the call's stream and device."""

import contextlib
import ctypes as C
import math
from types import SimpleNamespace

import pytest
import torch

import paper_2511_14694_amd as F
from paper_2511_14694_amd import _abi
from test_paged_abi import (E_ARG, E_DTYPE, E_NULL, E_SHAPE, E_UNSUPPORTED, E_WORKSPACE, FAKE, PAGED_BAD, _call, _paged,
                            _set)
from test_streams import Watch

i32 = torch.int32


def _cache8():
    c = _abi.PagedKv8(_paged(), 8, 0, FAKE, FAKE)
    c.kv.dtype, c.kv.weight, c.kv.weight_rows = 2, None, 0
    return c


CACHE8_BAD = [("kv." + f, v, st) for f, v, st in PAGED_BAD if f not in ("weight", "weight_rows", "dtype")] + [
    ("kv.dtype", 0, E_DTYPE), ("kv.dtype", 1, E_DTYPE), ("kv.dtype", 3, E_DTYPE), ("kv.weight", FAKE, E_SHAPE),
    ("scale_rows", 0, E_UNSUPPORTED), ("scale_rows", 4, E_UNSUPPORTED), ("scale_rows", 12, E_UNSUPPORTED),
    ("scale_rows", 32, E_UNSUPPORTED), ("scale_rows", -8, E_UNSUPPORTED),
    ("k_scale", None, E_NULL), ("v_scale", None, E_NULL), ("k_scale", FAKE + 2, E_ARG), ("v_scale", FAKE + 1, E_ARG),
]


def _extend_ok():
    d = _abi.PagedExtendDesc()
    d.page_rows, d.batch, d.max_pages, d.free_cap, d.n_rows = 16, 3, 7, 20, 9
    for f in ("table", "length", "add", "free_pages", "free_count", "first_pos", "start", "cu_rows", "row_seq", "row_slot",
              "row_pos"):
        setattr(d, f, FAKE)
    return d


@pytest.mark.parametrize("field,value,status", [
    ("batch", -1, E_ARG), ("max_pages", -1, E_ARG), ("free_cap", -1, E_ARG), ("n_rows", -1, E_ARG),
    ("page_rows", 0, E_UNSUPPORTED), ("page_rows", 4, E_UNSUPPORTED), ("page_rows", 24, E_UNSUPPORTED),
    ("page_rows", 2048, E_UNSUPPORTED), ("page_rows", -16, E_UNSUPPORTED),
    ("max_pages", 1 << 27, E_SHAPE), ("n_rows", 2 ** 31 - 1, E_SHAPE), ("n_rows", 1 << 40, E_SHAPE),
    ("batch", 2 ** 31 - 1, E_SHAPE), ("batch", 1 << 29, E_SHAPE),
] + [(f, None, E_NULL) for f in ("table", "length", "add", "free_pages", "free_count", "start", "cu_rows")]
  + [(f, FAKE + k, E_ARG) for k, f in enumerate(("table", "length", "add", "free_pages", "free_count", "first_pos",
                                                 "start", "cu_rows", "row_seq", "row_slot", "row_pos", "err"), 1) if k % 4])
def test_extend_refusals(field, value, status):
    d = _extend_ok()
    _set(field, value)(d)
    assert _call("focus_paged_extend", d) == status
    assert _abi.lib().focus_paged_extend(None, None) == E_NULL


def _append_ok():
    d = _abi.PagedAppendDesc()
    d.cache, d.dtype, d.n_rows = _cache8(), 0, 9
    for f in ("cu_rows", "start", "k", "v"):
        setattr(d, f, 2 * FAKE)
    d.k_row = d.v_row = 4 * 128
    d.k_head = d.v_head = 128
    return d


@pytest.mark.parametrize("field,value,status", [("cache." + f, v, st) for f, v, st in CACHE8_BAD] + [
    ("dtype", 2, E_DTYPE), ("dtype", -1, E_DTYPE), ("n_rows", -1, E_ARG), ("n_rows", 1 << 31, E_SHAPE),
    ("cu_rows", None, E_SHAPE),                      # one row a sequence, but nine rows
    ("start", None, E_NULL), ("k", None, E_NULL), ("v", None, E_NULL), ("start", FAKE, E_ARG),   # cache.length itself
    ("k", FAKE + 8, E_ARG), ("v", FAKE + 2, E_ARG), ("start", FAKE + 2, E_ARG), ("cu_rows", FAKE + 1, E_ARG),
    ("err", FAKE + 2, E_ARG), ("k_row", -512, E_ARG), ("k_head", 132, E_ARG), ("v_row", 516, E_ARG), ("v_head", -8, E_ARG),
])
def test_append_refusals(field, value, status):
    d = _append_ok()
    _set(field, value)(d)
    assert _call("focus_paged_append", d) == status


def test_append_of_nothing():
    d = _append_ok()
    d.n_rows = 0
    d.k = d.v = d.start = None
    assert _call("focus_paged_append", d) == 0
    d = _append_ok()
    d.cache.kv.batch = 0
    assert _call("focus_paged_append", d) == 0
    assert _abi.lib().focus_paged_append(None, None) == E_NULL


def _attend_ok():
    d = _abi.PagedAttendDesc()
    d.cache, d.dtype, d.n_heads, d.max_rows, d.n_rows = _cache8(), 0, 8, 3, 5
    d.q = d.o = d.cu_rows = d.lse = FAKE
    d.q_row, d.q_head = 8 * 128, 128
    return d


@pytest.mark.parametrize("field,value,status", [("cache." + f, v, st) for f, v, st in CACHE8_BAD] + [
    ("cache.kv.head_dim", 96, E_UNSUPPORTED), ("dtype", 2, E_DTYPE), ("dtype", -1, E_DTYPE), ("n_heads", 0, E_ARG),
    ("n_heads", 6, E_SHAPE), ("max_rows", 0, E_ARG), ("max_rows", -1, E_ARG), ("max_rows", 257, E_SHAPE),
    ("n_heads", 4 * 171, E_SHAPE), ("n_rows", -1, E_ARG), ("n_rows", 1 << 31, E_SHAPE), ("cu_rows", None, E_SHAPE),
    ("split_keys", -128, E_ARG), ("split_keys", 64, E_ARG), ("softmax_scale", math.nan, E_ARG),
    ("q_row", -8, E_ARG), ("q_head", 132, E_ARG), ("q", None, E_NULL), ("o", None, E_NULL), ("q", FAKE + 8, E_ARG),
    ("o", FAKE + 4, E_ARG), ("lse", FAKE + 2, E_ARG), ("cu_rows", FAKE + 2, E_ARG), ("err", FAKE + 1, E_ARG),
    ("cache.kv.batch", 1 << 24, E_SHAPE), ("cache.kv.page_stride", 1 << 33, E_SHAPE),
])
def test_attend_refusals(field, value, status):
    d = _attend_ok()
    _set(field, value)(d)
    assert _call("focus_paged_attend", d) == status
    if status not in (E_NULL,) and field not in ("q", "o", "lse", "cu_rows", "err"):
        assert _abi.lib().focus_paged_attend_workspace(C.byref(d)) == 0


def test_attend_workspace():
    query = _abi.lib().focus_paged_attend_workspace
    d = _attend_ok()
    assert query(C.byref(d)) == 0                        # 80 rows a table: not split
    d.split_keys = 128
    need = query(C.byref(d))
    assert need > 0
    assert _call("focus_paged_attend", d) == E_WORKSPACE
    d.workspace, d.workspace_bytes = FAKE, need - 1
    assert _call("focus_paged_attend", d) == E_WORKSPACE
    d.workspace, d.workspace_bytes = FAKE + 8, need
    assert _call("focus_paged_attend", d) == E_ARG
    # it grows with the tokens, the sequences and the tables, and holds every partial
    d = _attend_ok()
    d.cache.kv.max_pages = 5000
    sizes = []
    for batch, rows in ((2, 1), (2, 3), (2, 40), (500, 3)):
        d.cache.kv.batch, d.max_rows = batch, rows
        sizes.append(query(C.byref(d)))
        assert sizes[-1] >= 4 * 8 * rows * 128 * 2
    assert sizes[0] < sizes[1] < sizes[2] and sizes[1] < sizes[3] + 1
    d.split_keys = 128
    assert query(C.byref(d)) >= 500 * (5000 * 16 // 128) * 8 * 3 * 132 * 4
    d = _attend_ok()
    d.cache.kv.batch = 0
    assert query(C.byref(d)) == 0 and _call("focus_paged_attend", d) == 0
    d = _attend_ok()
    d.n_rows = 0
    assert _call("focus_paged_attend", d) == 0
    assert query(None) == 0 and _abi.lib().focus_paged_attend(None, None) == E_NULL


def test_attend_workspace_of_nothing():
    """No sequences or no rows: none, for any sizes, as many workgroups as they would be."""
    query = _abi.lib().focus_paged_attend_workspace
    d = _attend_ok()
    kv = d.cache.kv
    kv.max_pages, d.n_rows = 5000, 0
    assert query(C.byref(d)) == 0 and _call("focus_paged_attend", d) == 0
    # as many tiles of columns times sets of heads as 32 bits count
    kv.batch, kv.n_pages, kv.head_dim, kv.page_rows, kv.max_pages = 0, 1, 64, 16, 100
    kv.page_stride, kv.row_stride, kv.head_stride, d.cache.scale_rows = 64, 64, 1024, 16
    kv.n_kv_heads = d.n_heads = 1 << 29
    d.dtype, d.max_rows, d.q_row, d.q_head = 1, 512, 64, 64
    assert _call("focus_paged_attend", d) == 0 and query(C.byref(d)) == 0


@pytest.mark.parametrize("dtype,dim,heads,by_head", [(0, 128, 8, True), (0, 64, 8, True), (1, 128, 8, True), (0, 128, 9, False),
                                                      (0, 128, 40, False)])
def test_attend_call_and_query_agree_on_the_most_workgroups(dtype, dim, heads, by_head):
    """More workgroups than a launch holds: refused before a workspace is asked for, and the
    query, which a caller allocates by, says 0."""
    query = _abi.lib().focus_paged_attend_workspace
    d = _attend_ok()
    kv, page = d.cache.kv, 1024
    d.dtype, d.max_rows, d.split_keys, d.n_rows = dtype, 4, 128, 1
    kv.head_dim, kv.page_rows, kv.n_kv_heads, d.n_heads = dim, page, heads, heads
    kv.row_stride, kv.head_stride = (dim, page * dim) if by_head else (heads * dim, dim)
    kv.page_stride, d.q_row, d.q_head = page * heads * dim, heads * dim, dim
    kv.max_pages = 256
    seen = set()
    for batch in range(100, 4000, 50):
        kv.batch = batch
        st, need = _call("focus_paged_attend", d), query(C.byref(d))
        assert (st, need > 0) in ((E_WORKSPACE, True), (E_SHAPE, False)), batch
        seen.add(st)
        if st == E_SHAPE:
            d.workspace, d.workspace_bytes = FAKE, 1 << 60
            assert _call("focus_paged_attend", d) == E_SHAPE
            d.workspace, d.workspace_bytes = None, 0
    assert seen == {E_WORKSPACE, E_SHAPE}


# ------------------------------------------------------------------- the binding

def _cache(B=2, K=2, D=64, page=16, block=8, pages=4, width=3):
    t = torch.zeros
    k, v = (t(pages, page, K, D, dtype=torch.uint8).view(torch.float8_e4m3fn) for _ in range(2))
    return F.PagedCache8(k, v, t(pages, K, page // block), t(pages, K, page // block), t(B, width, dtype=i32), t(B, dtype=i32))


def _with(c, **kw):
    return F.PagedCache8(**{**c.__dict__, **kw})


def test_binding_refuses_what_does_not_fit():
    t = torch.zeros
    c = _cache()
    bad = [_with(c, k=c.k.view(torch.uint8)), _with(c, v=c.v[:3]), _with(c, k=c.k.transpose(1, 2)),
           _with(c, k=c.k[..., ::2], v=c.v[..., ::2]), _with(c, k_scale=t(4, 2, 3)), _with(c, k_scale=t(4, 1, 2)),
           _with(c, v_scale=t(4, 2, 1)), _with(c, k_scale=c.k_scale.double()), _with(c, k_scale=t(4, 2, 4)[..., ::2]),
           _with(c, k_scale=t(())), _with(c, k_scale=t(4, 2, 0), v_scale=t(4, 2, 0)), _with(c, table=c.table.long()),
           _with(c, table=c.table[0]), _with(c, length=t(3, dtype=i32)), _with(c, length=t(2)),
           _with(c, k=c.k[0], v=c.v[0])]
    q, k, start = t(2, 4, 64, dtype=torch.bfloat16), t(2, 2, 64, dtype=torch.bfloat16), t(2, dtype=i32)
    for b in bad:
        with pytest.raises((ValueError, RuntimeError)):
            b.desc()
    cu = t(3, dtype=i32)
    for call in (lambda: F.focus_paged_append(k[0], k, c, start), lambda: F.focus_paged_append(k.half(), k.half(), c, start),
                 lambda: F.focus_paged_append(k, k.float(), c, start), lambda: F.focus_paged_append(k, k[:1], c, start),
                 lambda: F.focus_paged_append(k[:, :1], k[:, :1], c, start), lambda: F.focus_paged_append(k, k, c, start[:1]),
                 lambda: F.focus_paged_append(k, k, c, start.long()), lambda: F.focus_paged_append(k, k, c, start, cu[:2]),
                 lambda: F.focus_paged_append(k[..., ::2], k[..., ::2], c, start),
                 lambda: F.focus_paged_attend(q[0], c), lambda: F.focus_paged_attend(q.half(), c),
                 lambda: F.focus_paged_attend(q[..., :32], c), lambda: F.focus_paged_attend(q, c, cu.long()),
                 lambda: F.focus_paged_attend(q, c, cu[:2]), lambda: F.focus_paged_attend(q, c, o=q.float()),
                 lambda: F.focus_paged_attend(q, c, lse=t(2, 3)), lambda: F.focus_paged_attend(q, c, o=q[:1]),
                 lambda: F.focus_paged_attend(q, c, max_rows=1 << 32), lambda: F.focus_paged_attend(q, c, split_keys=1 << 33),
                 lambda: F.focus_paged_attend(q, c), lambda: F.focus_paged_append(k, k, c, start)):   # not on a GPU
        with pytest.raises(ValueError):
            call()
    tab, length, add, free, count = t(2, 3, dtype=i32), t(2, dtype=i32), t(2, dtype=i32), t(9, dtype=i32), t(1, dtype=i32)

    def extend(table=tab, length=length, page=16, add=add, free=free, count=count, n=5, **kw):
        F.focus_paged_extend(table, length, page, add, free, count, n, **kw)
    rows = F.PagedRows(*(t(n, dtype=i32) for n in (2, 3, 5, 5, 5)))
    for kw in (dict(table=tab[0]), dict(table=tab.long()), dict(length=t(3, dtype=i32)), dict(add=t(2)), dict(free=free.float()),
               dict(count=t(2, dtype=i32)), dict(first_pos=t(3, dtype=i32)), dict(table=t(3, 2, dtype=i32).t()),
               dict(n=1 << 32), dict(out=rows, n=4), dict(out=F.PagedRows(rows.cu_rows, rows.cu_rows, rows.row_seq, rows.row_slot, rows.row_pos)),
               dict(err=t(0, dtype=i32)), dict()):
        with pytest.raises(ValueError):
            extend(**kw)


def test_descriptors_are_filled(monkeypatch):
    calls = {}

    def launch(name, d, dev, stream, accept=0):
        calls[name] = d
        return 0
    monkeypatch.setattr(F, "_launch", launch)
    t = torch.zeros
    B, K, D, H = 2, 3, 64, 6
    codes = t(4, K, 16, D, dtype=torch.uint8).view(torch.float8_e4m3fn)
    c = F.PagedCache8(codes.transpose(1, 2), codes.clone().transpose(1, 2), t(4, K, 2), t(4, K, 2), t(B, 7, dtype=i32),
                      t(B, dtype=i32))
    p = lambda x: x.data_ptr() if torch.is_tensor(x) else x  # noqa: E731

    def fields(d, want):
        assert set(want) == {f for f, *_ in d._fields_}
        for name, x in want.items():
            got = getattr(d, name)
            if isinstance(x, dict):
                fields(got, x)
            else:
                assert got == p(x), name
    cache = dict(kv=dict(dtype=2, n_kv_heads=K, head_dim=D, page_rows=16, n_pages=4, k=c.k, v=c.v, page_stride=K * 16 * D,
                         row_stride=D, head_stride=16 * D, batch=B, max_pages=7, table=c.table, length=c.length, weight=None,
                         weight_rows=0), scale_rows=8, reserved=0, k_scale=c.k_scale, v_scale=c.v_scale)
    fields(c.desc(), cache)
    n = 5
    qkv = t(n, H + 2 * K, D, dtype=torch.float32)
    q, k, v = qkv[:, :H], qkv[:, H:H + K], qkv[:, H + K:].transpose(0, 1).contiguous().transpose(0, 1)
    cu, start, err, ws = t(B + 1, dtype=i32), t(B, dtype=i32), t(1, dtype=i32), t(8)
    row = (H + 2 * K) * D
    F.focus_paged_append(k, v, c, start, cu_rows=cu, err=err)
    fields(calls["focus_paged_append"], dict(cache=cache, dtype=1, reserved=0, n_rows=n, cu_rows=cu, start=start, k=k, k_row=row,
                                              k_head=D, v=v, v_row=D, v_head=n * D, err=err))
    F.focus_paged_append(k[:2], v[:2], c, start)
    d = calls["focus_paged_append"]
    assert d.cu_rows is None and d.n_rows == 2 and d.err is None
    o, lse = t(n, H, D), t(n, H)
    F.focus_paged_attend(q, c, cu, 3, o=o, lse=lse, workspace=ws, split_keys=256, softmax_scale=0.5, err=err)
    fields(calls["focus_paged_attend"], dict(
        cache=cache, dtype=1, n_heads=H, max_rows=3, split_keys=256, softmax_scale=0.5, reserved=0, n_rows=n, cu_rows=cu, q=q,
        q_row=row, q_head=D, o=o, lse=lse, workspace=ws, workspace_bytes=32, err=err))
    got = F.focus_paged_attend(q, c, cu, 3, want_lse=False)
    d = calls["focus_paged_attend"]
    assert d.o == got[0].data_ptr() and d.lse is None and got[1] is None and got[0].is_contiguous()
    got = F.focus_paged_attend(q, c, cu, 3)
    assert calls["focus_paged_attend"].lse == got[1].data_ptr() and got[1].shape == (n, H) and got[1].dtype == torch.float32

    tab, add, free, count, first = t(B, 7, dtype=i32), t(B, dtype=i32), t(9, dtype=i32), t(1, dtype=i32), t(B, dtype=i32)
    for out in (None, F.PagedRows(*(t(m, dtype=i32) for m in (B, B + 1, n, n, n)))):
        r = F.focus_paged_extend(tab, c.length, 32, add, free, count, n, first_pos=first, out=out, err=err)
        assert out is None or r is out
        assert [x.shape[0] for x in r.__dict__.values()] == [B, B + 1, n, n, n]
        fields(calls["focus_paged_extend"], dict(
            page_rows=32, batch=B, max_pages=7, free_cap=9, table=tab, length=c.length, add=add, free_pages=free,
            free_count=count, first_pos=first, start=r.start, cu_rows=r.cu_rows, n_rows=n, row_seq=r.row_seq,
            row_slot=r.row_slot, row_pos=r.row_pos, err=err))


def _calls():
    t = torch.zeros
    c, free = _cache(), t(9, dtype=i32)
    q = t(2, 4, 64, dtype=torch.bfloat16)
    return {"extend": (lambda s: F.focus_paged_extend(c.table, c.length, 16, t(2, dtype=i32), free, free[:1], 5, stream=s), 1, 1),
            "attend": (lambda s: F.focus_paged_attend(q, c, stream=s), 3, 2)}


@pytest.mark.parametrize("name", sorted(_calls()))
def test_what_a_call_makes_belongs_to_its_stream(name, monkeypatch):
    class Lib:
        def __getattr__(self, what):
            return lambda *a: 48
    current, told = ["the caller's"], []

    @contextlib.contextmanager
    def stream(s):
        current.append(s)
        yield
        current.pop()
    monkeypatch.setattr(F, "lib", Lib)
    monkeypatch.setattr(F, "_launch", lambda *a: a[4] if len(a) > 4 else 0)     # a workspace is needed
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: f"stream {handle}")
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current[-1])
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: told.append(s), raising=False)
    call, count, outputs = _calls()[name]
    for s, where in ((SimpleNamespace(cuda_stream=5), "stream 5"), (None, "the caller's")):
        with Watch(current) as w:
            call(s)
        assert [x for _, x in w.made] == [where] * count, w.made
        assert told == (["the caller's"] * outputs if s else [])     # all but the scratch
        told.clear()


def test_workspace_is_asked_of_the_tensors_device(monkeypatch):
    """Tensors on device 1, current device 0."""
    asked, at = [], [0]

    class Lib:
        def __getattr__(self, name):
            return lambda *a: asked.append((name, at[-1])) or 16

    class Device:
        def __init__(self, n):
            self.n = n

        def __enter__(self):
            at.append(self.n)

        def __exit__(self, *a):
            at.pop()
    monkeypatch.setattr(F, "lib", Lib)
    monkeypatch.setattr(F, "_device", lambda: at[-1])
    monkeypatch.setattr(F, "_launch", lambda *a: a[4] if len(a) > 4 else 0)
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 1)
    c, q = _cache(), torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    F.focus_paged_attend_workspace(q, c)
    F.focus_paged_attend(q, c)
    assert [d for _, d in asked] == [1, 1] and at == [0], asked


def test_a_refused_call_is_an_error_whatever_status_another_may_have(monkeypatch):
    """Only the status that asks for a workspace is taken as an answer."""
    class Lib:
        def __getattr__(self, name):
            return {"focus_paged_attend": lambda d, s: 5, "focus_status_str": lambda s: b"unsupported"}[name]
    monkeypatch.setattr(F, "lib", Lib)
    monkeypatch.setattr(_abi, "lib", Lib)
    monkeypatch.setattr(F, "_raw_stream", lambda dev: 0)
    monkeypatch.setattr(F, "_device", lambda: 0)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    with pytest.raises(F.FocusError):
        F.focus_paged_attend(torch.zeros(2, 4, 64, dtype=torch.bfloat16), _cache())
