"""Pins of the 8-bit paged cache's oracle: facts that the type and the definitions fix."""

import math

import numpy as np
import pytest
import torch

from oracle import paged as P
from oracle import paged8 as O


def test_e4m3_numbers_are_torchs():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(codes[:0x7f], O.E4M3) and np.array_equal(codes[0x80:0xff], -O.E4M3)
    assert np.isnan(codes[[0x7f, 0xff]]).all() and O.E4M3[-1] == 448.0 and O.E4M3[1] == 2.0 ** -9


def test_nearest_is_torchs_rounding():
    """Over all bf16 numbers up to 448 and the middles between neighbouring e4m3 numbers."""
    x = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).double()
    x = x[x.abs() <= 448].numpy()
    mid = (O.E4M3[1:] + O.E4M3[:-1]) / 2
    x = np.concatenate([x, mid, -mid, np.nextafter(mid, 0.0), np.nextafter(mid, 1e3)])
    x = x[np.float32(x) == x]
    assert np.array_equal(O.nearest(x), torch.as_tensor(x, dtype=torch.float32).to(torch.float8_e4m3fn).double().numpy())
    assert np.isnan(O.nearest(np.array([np.inf, -np.inf, np.nan]))).all()


@pytest.mark.parametrize("most,e", [(0.0, -126), (448.0, 0), (np.nextafter(448.0, 500.0), 1), (1.0, -8), (1.75, -8),
                                    (1.7500001, -7), (2.0 ** -149, -126), (3.4e38, 120), (448.0 * 2.0 ** -126, -126)])
def test_scale_is_the_least_that_fits(most, e):
    assert O.scale_of(np.array([[most, -most / 3, np.nan, np.inf]])) == 2.0 ** e


def test_append_in_steps_is_append_at_once_but_for_small_elements():
    """Row by row, a block's scale grows to what it is at once; requantised rows are the same
    where nothing falls below the smallest normal number."""
    rng = np.random.default_rng(0)
    new = rng.choice([-1.0, 1.0], (37, 5)) * rng.uniform(1.0, 16.0, (37, 5))
    once, s1 = O.append(np.zeros((0, 5)), np.zeros(3), 16, 0, new)
    rows, s2 = np.zeros((0, 5)), np.zeros(3)
    for r in range(37):
        rows, s2 = O.append(rows, s2, 16, r, new[r:r + 1])
    assert np.array_equal(s1, s2) and np.array_equal(once, rows)
    got = once * np.repeat(s1, 16)[:37, None]
    assert (np.abs(got - new) <= 2.0 ** -4 * np.abs(new)).all()


def test_append_forgets_rows_from_start_on():
    rows, scales = np.full((20, 4), 400.0), np.array([8.0, 8.0, 8.0])
    out, s = O.append(rows, scales, 8, 16, np.ones((2, 4)))
    assert np.array_equal(out[:16], rows[:16]) and s.tolist() == [8.0, 8.0, 2.0 ** -8]
    out, s = O.append(rows, scales, 8, 17, np.ones((2, 4)))     # row 16 stays, and its scale
    assert s[2] == 8.0 and out.shape == (19, 4) and out[17, 0] == 0.125


def test_attend_of_one_token_is_decode_and_earlier_tokens_see_less():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((3, 4, 8)), rng.standard_normal((9, 2, 8)), rng.standard_normal((9, 2, 8))
    o, lse = O.attend(q, k, v)
    for i, n in enumerate((7, 8, 9)):
        ro, rl, _ = P.decode(q[i], k[:n], v[:n])
        assert np.array_equal(o[i], ro) and np.array_equal(lse[i], rl)
    o, lse = O.attend(q, k[:1], v[:1])
    assert (o[:2] == 0).all() and (lse[:2] == -math.inf).all() and np.allclose(o[2], v[0].repeat(2, 0))


def test_extend_keeps_every_page_once():
    rng = np.random.default_rng(2)
    page, width, batch, pool = 8, 6, 7, 30
    table, length = [[-1] * width for _ in range(batch)], [0] * batch
    free = list(range(pool))
    unserved = 0
    for _ in range(300):
        add = [int(x) for x in rng.integers(-20, 20, batch)]
        before = list(length)
        start, cu, seq, slot, pos, fine = O.extend(table, length, page, add, free, 60)
        held = [p for b in range(batch) for p in table[b][:-(-length[b] // page)]]
        assert sorted(held + free) == list(range(pool))
        assert all(p == -1 for b in range(batch) for p in table[b][-(-length[b] // page):])
        for b, a in enumerate(add):
            if a > 0:
                assert (start[b], length[b]) in ((before[b], before[b] + a), (-1, before[b]))
                unserved += start[b] < 0
                for i in range(a):
                    if cu[b] + i < 60:
                        assert (seq[cu[b] + i], slot[cu[b] + i]) == (b, start[b] + i if start[b] >= 0 else -1)
            else:
                assert length[b] == start[b] == max(before[b] + a, 0)
        assert fine == all(s >= 0 for s in start)
    assert unserved > 50
