"""Pins of oracle/paged.py: facts that mathematics or the cited definitions fix,
checked without a GPU, and the host half of focus_rope_turns against them."""

import itertools
import math

import numpy as np
import pytest

import paper_2511_14694_amd as F
from oracle import paged as P
from oracle import projection
from oracle.attention import dense_causal

KINDS = {"none": F.FOCUS_ROPE_NONE, "linear": F.FOCUS_ROPE_LINEAR, "base": F.FOCUS_ROPE_BASE,
         "bands": F.FOCUS_ROPE_BANDS}


def test_rope_is_the_projection_oracles_rotation():
    rng = np.random.default_rng(0)
    x, pos = rng.normal(size=(7, 3, 16)), rng.integers(0, 1_000, 7)
    assert np.allclose(P.rope(x, pos, P.turns(16)), projection.rope(x, pos, 10000.0), atol=1e-10)


@pytest.mark.parametrize("pairs", ["interleaved", "half"])
@pytest.mark.parametrize("rot", [0, 2, 10, 16])
def test_rope_keeps_lengths_and_scores_depend_on_distance(pairs, rot):
    rng = np.random.default_rng(rot)
    t = P.turns(rot)
    q, k = rng.normal(size=(2, 1, 1, 16))
    a = P.rope(q, [12], t, pairs), P.rope(k, [5], t, pairs)
    b = P.rope(q, [1012], t, pairs), P.rope(k, [1005], t, pairs)
    assert np.isclose(np.linalg.norm(a[0]), np.linalg.norm(q))
    assert np.isclose((a[0] * a[1]).sum(), (b[0] * b[1]).sum())
    assert np.array_equal(a[0][..., rot:], q[..., rot:])
    assert np.allclose(P.rope(a[0], [12], t, pairs, inverse=True), q)


def test_rope_pairings_differ_by_a_permutation():
    rng = np.random.default_rng(3)
    x, pos, t = rng.normal(size=(4, 2, 12)), [0, 3, 9, -7], P.turns(12)
    order = np.concatenate([np.arange(0, 12, 2), np.arange(1, 12, 2)])
    assert np.allclose(P.rope(x, pos, t)[..., order], P.rope(x[..., order], pos, t, "half"))


@pytest.mark.parametrize("pairs", ["interleaved", "half"])
def test_rope_inverse_is_the_transpose(pairs):
    """<g, R x> = <R^T g, x>, the gradient of a linear map; and by differences."""
    rng = np.random.default_rng(4)
    x, g, t = rng.normal(size=(3, 2, 8)), rng.normal(size=(3, 2, 8)), P.turns(6)
    pos = [1, 50, 1 << 20]
    back = P.rope(g, pos, t, pairs, inverse=True, amplitude=1.25)
    assert np.isclose((g * P.rope(x, pos, t, pairs, amplitude=1.25)).sum(), (back * x).sum())
    for idx in [(0, 0, 1), (1, 1, 4), (2, 0, 7)]:
        d = np.zeros_like(x)
        d[idx] = 1e-6
        f = lambda y: (g * P.rope(y, pos, t, pairs, amplitude=1.25)).sum()  # noqa: E731
        assert np.isclose((f(x + d) - f(x - d)) / 2e-6, back[idx], atol=1e-6)


@pytest.mark.parametrize("scaling", sorted(KINDS))
@pytest.mark.parametrize("rot", [4, 32, 128])
def test_turns_of_the_library(scaling, rot):
    kw = dict(theta=50_000.0, factor=1.0 if scaling == "none" else 8.0, context=4096.0, low=1.0, high=32.0)
    got = F.focus_rope_turns(rot, scaling=KINDS[scaling], device="cpu", **kw).numpy()
    assert np.allclose(got, P.turns(rot, scaling=scaling, **kw), rtol=1e-14, atol=0)


def test_turns_limits():
    plain = P.turns(64)
    assert np.isclose(plain[0], 1 / (2 * math.pi))
    base = P.turns(64, scaling="base", factor=8.0)
    assert np.isclose(base[0], plain[0]) and np.isclose(base[-1], plain[-1] / 8.0)
    bands = P.turns(64, scaling="bands", factor=8.0, context=8192, low=1.0, high=32.0)
    r = plain * 8192
    assert np.array_equal(bands[r >= 32], plain[r >= 32])
    assert np.allclose(bands[r <= 1], plain[r <= 1] / 8)
    assert (np.diff(bands) < 0).all()


@pytest.mark.parametrize("kw", [dict(rot_dim=3), dict(rot_dim=0), dict(rot_dim=258), dict(theta=1.0),
                                dict(theta=math.nan), dict(theta=math.inf), dict(scaling=4), dict(scaling=-1),
                                dict(scaling=1, factor=0.5), dict(scaling=2, rot_dim=2), dict(scaling=3),
                                dict(scaling=3, context=100, low=2.0, high=2.0),
                                dict(scaling=3, context=100, low=-1.0), dict(scaling=1, factor=math.nan)])
def test_turns_refusals(kw):
    with pytest.raises(F.FocusError) as e:
        F.focus_rope_turns(**{"rot_dim": 8, "device": "cpu", **kw})
    assert e.value.status == 2


def test_decode_is_the_last_row_of_causal_attention():
    rng = np.random.default_rng(5)
    n, H, K, D = 9, 4, 2, 8
    q, k, v = rng.normal(size=(n, H, D)), rng.normal(size=(n, K, D)), rng.normal(size=(n, K, D))
    o, lse = dense_causal(q, k, v)
    o1, lse1, w = P.decode(q[-1], k, v)
    assert np.allclose(o1, o[-1]) and np.allclose(lse1, lse[-1])
    assert np.allclose(w.sum(1), H // K) and (w > 0).all()
    o0, lse0, w0 = P.decode(q[-1], k[:0], v[:0])
    assert not o0.any() and (lse0 == -np.inf).all() and w0.shape == (K, 0)


def test_decode_hidden_rows_are_as_if_absent():
    rng = np.random.default_rng(6)
    q, k, v = rng.normal(size=(2, 4)), rng.normal(size=(6, 1, 4)), rng.normal(size=(6, 1, 4))
    seen = np.array([1, 0, 1, 1, 0, 0], bool)
    a, b = P.decode(q, k, v, visible=seen), P.decode(q, k[seen], v[seen])
    assert np.allclose(a[0], b[0]) and np.allclose(a[1], b[1]) and np.allclose(a[2][:, seen], b[2])


def test_rows_walk_the_table():
    pool = np.arange(5 * 4).reshape(5, 4)
    assert list(P.rows(pool, [3, 0, 4], 9)) == [12, 13, 14, 15, 0, 1, 2, 3, 16]
    assert P.rows(pool, [], 0).shape == (0,)


def test_keep_against_every_subset():
    """Of all subsets of m rows that hold the recent ones, the kept one has the greatest
    weight, and the lowest rows where several do."""
    rng = np.random.default_rng(7)
    for _ in range(60):
        n = int(rng.integers(1, 8))
        w = rng.integers(0, 4, n).astype(float)
        budget, recent = int(rng.integers(0, n + 2)), int(rng.integers(0, n + 1))
        got = P.keep(w, budget, recent)
        m = min(n, budget)
        must = set(range(n - min(recent, m), n))
        best = max((s for s in itertools.combinations(range(n), m) if must <= set(s)),
                   key=lambda s: (w[list(s)].sum(), [-r for r in s]))
        assert tuple(got) == best, (w, budget, recent)


def test_keep_orders_nan_infinities_and_zeros():
    w = [0.0, -0.0, math.nan, math.inf, -math.inf, 1.0]
    assert P.keep(w, 1, 0) == [2]
    assert P.keep(w, 2, 0) == [2, 3]
    assert P.keep(w, 4, 0) == [0, 2, 3, 5]
    assert P.keep(w, 5, 0) == [0, 1, 2, 3, 5]
    assert P.keep(w, 2, 5) == [4, 5]
