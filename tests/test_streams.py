"""CPU checks of the stream= argument: what a call allocates or copies by itself is
made on that stream, and the caller's own stream is told of it (no GPU is touched:
streams are stand-ins, the library answers every call with success)."""

import contextlib
from types import SimpleNamespace

import numpy as np
import pytest
import torch
from torch.overrides import TorchFunctionMode

import paper_2511_14694_amd as F

MAKES = {torch.empty, torch.empty_like, torch.Tensor.new_empty, torch.as_tensor}


class Watch(TorchFunctionMode):
    """The calls that make tensors, with the stream that is current."""

    def __init__(self, current):
        super().__init__()
        self.current, self.made = current, []

    def __torch_function__(self, func, types, args=(), kwargs=None):
        if func in MAKES:
            self.made.append((func.__name__, self.current[-1]))
        return func(*args, **(kwargs or {}))


def _calls():
    t, i32, bf = torch.zeros, torch.int32, torch.bfloat16
    H, K, D, B = 4, 2, 64, 2
    pool = t(6, 16, K, D, dtype=bf)
    cache = F.PagedCache(pool, pool.clone(), t(B, 3, dtype=i32), t(B, dtype=i32), t(B, K, 48))
    q, k, pos, turns = t(3, H, D, dtype=bf), t(3, K, D, dtype=bf), t(3, dtype=i32), t(32, dtype=torch.float64)
    lay = F.Layout(F.LayoutTotals(), B, 100, {n: t(9, dtype=torch.int64) for n in
                                              F.WINDOW_FIELDS + F.TOKEN_FIELDS + ("sum_tok",)}, None, 7)
    rows = {"win_k": t(B, 8, K, D, dtype=bf), "win_v": t(B, 8, K, D, dtype=bf), "win_len": t(B, dtype=i32),
            "cache_k": t(B, 8, K, D, dtype=bf), "cache_v": t(B, 8, K, D, dtype=bf), "cache_len": t(B, dtype=i32)}
    logits = t(5, 8)
    hidden, w = t(3, 32, dtype=bf), t(32, (H + 2 * K) * D, dtype=bf)
    sched = F.DecodeSchedule(B, 100, device="cpu")
    return {
        "rope": (lambda s: F.focus_rope(pos, turns, q, k, stream=s), 2),
        "paged decode": (lambda s: F.focus_paged_decode(t(B, H, D, dtype=bf), cache, stream=s), 3),
        "paged evict": (lambda s: F.focus_paged_evict(cache, cache, 9, stream=s), 2),
        "window attention": (lambda s: F.focus_window_attn(lay, q, k, k, stream=s), 3),
        "decode step": (lambda s: F.focus_decode_step(t(B, H, D, dtype=bf), t(B, K, D, dtype=bf), t(B, K, D, dtype=bf),
                                                      t(B, dtype=torch.uint8), stream=s, **rows), 3),
        "schedule": (lambda s: sched.start([1, 2], stream=s), 1),
        "fidelity": (lambda s: F.focus_fidelity(logits, logits, cu_pos=[0, 2, 5], stream=s), 4),
        "gemm": (lambda s: F.focus_gemm(hidden, w, a_rows=[1, 2], stream=s), 2),
        "adapter attention": (lambda s: F.focus_adapter_attn(lay, q, k, k, stream=s), 2),
        "adapter layer": (lambda s: F.focus_adapter_layer(lay, t(0, 32, dtype=bf), t(32, H * D, dtype=bf), t(32, K * D, dtype=bf),
                                                          t(32, K * D, dtype=bf), t(H * D, 32, dtype=bf), H, K, stream=s), 2),
        "projection": (lambda s: F.focus_qkv_project(lay, hidden, w, H, K, stream=s), 3),
        "layout": (lambda s: F.focus_layout(F.LayoutTotals(), np.array([3, 4]), 100, np.array([1]), device="cpu", stream=s),
                   2 + 4 + len(F.WINDOW_FIELDS) + len(F.TOKEN_FIELDS)),
    }


@pytest.mark.parametrize("name", sorted(_calls()))
def test_what_a_call_makes_belongs_to_its_stream(name, monkeypatch):
    class Lib:
        def __getattr__(self, what):
            return lambda *a: 48 if "workspace" in what else 0
    current, told = ["the caller's"], []

    @contextlib.contextmanager
    def stream(s):
        current.append(s)
        yield
        current.pop()
    monkeypatch.setattr(F, "lib", Lib)
    monkeypatch.setattr(F, "_launch", lambda *a: None)
    monkeypatch.setattr(F, "_stream", lambda *a: 0)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: f"stream {handle}")
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current[-1])
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: told.append(s), raising=False)
    call, count = _calls()[name]
    for s, name in ((SimpleNamespace(cuda_stream=5), "stream 5"), (None, "the caller's")):
        with Watch(current) as w:
            call(s)
        assert len(w.made) == count, w.made
        assert {x for _, x in w.made} == {name}, w.made
        # all but the scratch, which nobody but the kernels reads
        if s:
            assert set(told) == {"the caller's"} and count - 1 <= len(told) <= count
            told.clear()
    assert not told
