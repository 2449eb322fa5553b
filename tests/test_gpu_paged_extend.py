"""focus_paged_extend on the GPU against the oracle, number for number."""

import numpy as np
import pytest
import torch

import paper_2511_14694_amd as F
from gpu_util import DEV, announce
from oracle import paged8 as O
from paged8_util import i32

pytestmark = pytest.mark.gpu


class Pool:
    """Sequences of `lens` rows and a stack of free pages, on the device and as lists."""

    def __init__(self, rng, lens, page, width, spare, room=None):
        need = [-(-n // page) for n in lens]
        order = [int(x) for x in rng.permutation(sum(need) + spare)]
        self.page, self.table = page, [[-1] * width for _ in lens]
        for b, m in enumerate(need):
            self.table[b][:m] = [order.pop() for _ in range(m)]
        self.length, self.free = list(lens), order
        self.room = sum(need) + spare if room is None else room
        self.d_table = i32(self.table).reshape(len(lens), width)
        self.d_length = i32(lens).reshape(-1)
        self.d_free = torch.full((self.room,), -7, dtype=torch.int32, device=DEV)
        self.d_free[:len(order)] = i32(order)
        self.d_count = i32([len(order)])
        self.err = torch.zeros(1, dtype=torch.int32, device=DEV)

    def step(self, add, n_rows, first_pos=None):
        self.err.zero_()
        got = F.focus_paged_extend(self.d_table, self.d_length, self.page, i32(add).reshape(-1), self.d_free, self.d_count,
                                   n_rows, first_pos=None if first_pos is None else i32(first_pos), err=self.err)
        *ref, fine = O.extend(self.table, self.length, self.page, add, self.free, n_rows, first_pos)
        for x, y, name in zip((got.start, got.cu_rows, got.row_seq, got.row_slot, got.row_pos), ref,
                              ("start", "cu", "seq", "slot", "pos")):
            assert x.tolist() == y, name
        assert self.d_table.tolist() == self.table and self.d_length.tolist() == self.length
        assert self.d_count.item() == len(self.free)
        assert self.d_free[:len(self.free)].tolist() == self.free
        assert self.err.item() == (0 if fine else F.FOCUS_ERR_CAPACITY)
        return fine


@pytest.mark.parametrize("batch,page,width,spare,most", [
    (1, 8, 4, 3, 12), (3, 16, 9, 20, 50), (64, 16, 12, 60, 30), (65, 8, 20, 300, 40), (1023, 8, 6, 700, 12),
    (1024, 16, 4, 800, 10), (2500, 8, 5, 2000, 9), (5, 1024, 3, 4, 1500),
])
def test_extend_matches_oracle(batch, page, width, spare, most):
    """Steps of rows that come and go, until pages run out and past that."""
    announce(f"extend {batch} sequences, pages of {page}, {width} each, {spare} spare")
    rng = np.random.default_rng(batch + page)
    p = Pool(rng, [int(x) for x in rng.integers(0, 2 * page, batch)], page, width, spare)
    for step in range(9):
        p.step([int(x) for x in np.where(rng.random(batch) < 0.3, 0, rng.integers(-most // 2 + step % 3, most, batch))],
               batch * most, first_pos=None if step % 2 else [int(x) for x in rng.integers(0, 1000, batch)])
    p.step([page * width - max(p.length) + (b % 2) for b in range(batch)], batch * page * width)
    assert not p.step([page * width + 1] * batch, batch * page * width)
    p.step([-10 ** 6] * batch, 0)
    assert p.length == [0] * batch and len(p.free) == p.room
    p.step([0] * batch, 5)


def test_extend_long_prompts():
    """Many pages of one sequence, rows past 65 536, and their return."""
    rng = np.random.default_rng(3)
    announce("extend long prompts")
    p = Pool(rng, [3, 0, 40], 8, 20_000, 30_000)
    assert p.step([100_001, 7, 70_000], 170_008, first_pos=[5, 2 ** 31 - 8, 0])
    assert p.step([-100_000, -7, 1], 1)
    assert p.length == [4, 0, 70_041]


@pytest.mark.parametrize("batch,rows,more", [(64, 41, 0), (64, 41, 700), (128, 67, 3), (300, 30, 9000), (1100, 5, 100), (2, 9000, 1)])
def test_extend_maps_of_many_rows(batch, rows, more):
    """More rows than the first launch maps: sequences without rows between, rows past the last."""
    rng = np.random.default_rng(batch)
    announce(f"extend maps {batch} x {rows} + {more}")
    add = [int(x) if y else 0 for x, y in zip(rng.integers(rows // 2, rows * 2, batch), rng.random(batch) < 0.8)]
    add[-1] = 0
    n = max(sum(add) + more, 9000 if batch > 256 else 2100)
    p = Pool(rng, [int(x) for x in rng.integers(0, 9, batch)], 16, (2 * rows + 32) // 16 + 1, batch * (rows // 8 + 3))
    assert p.step(add, n, first_pos=[int(x) for x in rng.integers(-50, 50, batch)])


def test_extend_out_of_pages_and_slots():
    rng = np.random.default_rng(4)
    announce("extend out of pages")
    p = Pool(rng, [8, 8, 5, 8], 8, 3, 3)
    # 2 pages, 2 (one is left: not served, nor those after that need one), none, 1
    assert not p.step([16, 9, 3, 8], 36) and p.length == [24, 8, 8, 8]
    assert not p.step([8, 0, 0, 1], 9) and p.length == [24, 8, 8, 9]        # the table is too short; takes nothing
    assert p.step([-24, 0, 0, 0], 0) and p.length == [0, 8, 8, 9]
    assert not p.step([0, 5, 5, 5], 7) and p.length == [0, 13, 8, 9]        # the maps end in the second's rows
    assert len(p.free) == 2
    assert p.step([0, -13, 9, 15], 24) and p.length == [0, 0, 17, 24]       # pages given back are taken at once
    p.step([2 ** 31 - 1, 2 ** 31 - 1, 3, 1], 4)


def test_extend_without_pages_or_sequences():
    announce("extend nothing")
    e = torch.empty(0, dtype=torch.int32, device=DEV)
    got = F.focus_paged_extend(torch.empty(0, 3, dtype=torch.int32, device=DEV), e, 8, e, e, i32([0]), 3)
    assert got.cu_rows.tolist() == [0] and got.row_seq.tolist() == [-1] * 3 == got.row_slot.tolist()
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    length = i32([0, 0])
    got = F.focus_paged_extend(torch.empty(2, 0, dtype=torch.int32, device=DEV), length, 8, i32([1, 0]), e, i32([0]), 1,
                               err=err)
    assert got.start.tolist() == [-1, 0] and err.item() == F.FOCUS_ERR_CAPACITY and length.tolist() == [0, 0]


def test_extend_clips_bad_state():
    announce("extend bad state")
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    table = i32([[4, 5], [6, 7], [-1, -1]])
    length = i32([-3, 99, 0])
    free, count = i32([1, 2, 3, -1]), i32([3])
    got = F.focus_paged_extend(table, length, 8, i32([8, -9, 3]), free, count, 11, err=err)
    # 0 rows of the first, 16 of the second: one page comes back, 7 rows stay, in 4 entries
    assert err.item() == F.FOCUS_ERR_BOUNDS
    assert length.tolist() == [8, 7, 3] and table.tolist() == [[7, 5], [6, -1], [3, -1]]
    assert count.item() == 2 and free.tolist()[:2] == [1, 2] and got.start.tolist() == [0, 7, 0]
    err.zero_()
    for bad, n in ((-5, 0), (2 ** 31 - 1, 4)):
        count.fill_(bad)
        F.focus_paged_extend(table, length, 8, i32([0, 0, 0]), free, count, 0, err=err)
        assert count.item() == n and err.item() == F.FOCUS_ERR_BOUNDS
    # no room on the stack: pages are lost, and that is said
    err.zero_()
    count.fill_(3)
    F.focus_paged_extend(table, length, 8, i32([-8, -7, 0]), free, count, 0, err=err)
    assert count.item() == 4 and free[3].item() == 7 and err.item() == F.FOCUS_ERR_CAPACITY
    assert table.tolist() == [[-1, 5], [-1, -1], [3, -1]]


def test_extend_writes_into_given_rows_on_another_stream():
    announce("extend out and stream")
    table, length, free, count = i32([[-1, -1]]), i32([0]), i32([5, 9]), i32([2])
    out = F.PagedRows(*(torch.full((n,), -9, dtype=torch.int32, device=DEV) for n in (1, 2, 10, 10, 10)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert F.focus_paged_extend(table, length, 8, i32([9]), free, count, 10, out=out, stream=side) is out
    side.synchronize()
    assert out.row_slot.tolist() == list(range(9)) + [-1] and out.cu_rows.tolist() == [0, 9]
    assert table.tolist() == [[9, 5]]
    add = i32([-9])
    side.wait_stream(torch.cuda.current_stream())
    got = F.focus_paged_extend(table, length, 8, add, free, count, 0, stream=side)
    side.synchronize()
    assert got.start.tolist() == [0] and count.item() == 2 and free.tolist() == [9, 5]
