"""CPU pins of the oracle for the bounded key/value cache."""
import itertools

import numpy as np
import pytest

from oracle import cache_oracle as co
from oracle import decode_oracle as do


def _rows(rng, *shape):
    return rng.standard_normal(shape)


@pytest.mark.parametrize("interleaved", [False, True])
def test_a_turn_by_nothing_and_by_a_quarter(interleaved):
    x = _rows(np.random.default_rng(0), 1, 2, 3, 6)
    still = co.rotary(x, np.zeros((1, 3, 1), int), np.ones(2), (2,), interleaved=interleaved)
    assert np.array_equal(still, x)
    quarter = co.rotary(x, np.ones((1, 3, 1), int), np.full(2, np.pi / 2), (2,), interleaved=interleaved)
    a, b = ([0, 2], [1, 3]) if interleaved else ([0, 1], [2, 3])
    assert np.allclose(quarter[..., a], -x[..., b]) and np.allclose(quarter[..., b], x[..., a])
    assert np.array_equal(quarter[..., 4:], x[..., 4:])


def test_scores_depend_on_the_difference_of_positions_alone():
    rng = np.random.default_rng(1)
    q, k = _rows(rng, 1, 1, 1, 8), _rows(rng, 1, 1, 1, 8)
    freq = np.array([1.0, 0.3, 0.1, 0.03])
    at = lambda x, p: co.rotary(x, np.array([[p]]), freq, (1, 2, 1))[0, 0, 0]
    for d in ((1, 2, 3), (-5, 0, 7)):
        s = [at(q, (10, 20, 30)) @ at(k, (10 + d[0], 20 + d[1], 30 + d[2])), at(q, (0, 0, 0)) @ at(k, d)]
        assert np.isclose(*s)


def test_the_inverse_is_the_transpose_and_undoes_the_turn():
    rng = np.random.default_rng(2)
    x, y, pos = _rows(rng, 2, 3, 4, 10), _rows(rng, 2, 3, 4, 10), rng.integers(0, 50, (2, 4, 2))
    how = dict(sections=(1, 3), interleaved=True)
    freq = np.array([1.0, 0.5, 0.2, 0.1])
    assert np.allclose(co.rotary(co.rotary(x, pos, freq, **how), pos, freq, inverse=True, **how), x)
    assert np.isclose((co.rotary(x, pos, freq, **how) * y).sum(), (x * co.rotary(y, pos, freq, inverse=True, **how)).sum())


@pytest.mark.parametrize("kw", [{}, dict(window=2), dict(softcap=0.7), dict(slopes=np.array([0.5, 0.25]))], ids=["plain", "window", "softcap", "alibi"])
def test_weights_hold_one_unit_per_row_and_head(kw):
    rng = np.random.default_rng(3)
    q, keys = _rows(rng, 3, 2, 3, 4), [_rows(rng, n, 1, 4) for n in (7, 3, 1)]
    old = rng.random((3, 1, 9))
    w = co.key_weights(q, keys, old, scale=0.5, **kw)
    for b, n in enumerate((7, 3, 1)):
        live = min(n, 3)                           # rows of the chunk that are tokens of the sequence
        assert np.isclose(w[b, 0, :n].sum(), 2 * live + old[b, 0, :max(0, n - 3)].sum())
        assert np.array_equal(w[b, 0, n:], old[b, 0, n:])


def test_probabilities_are_the_decode_oracles():
    rng = np.random.default_rng(4)
    q, k, v = _rows(rng, 1, 2, 4), _rows(rng, 1, 5, 1, 4), _rows(rng, 1, 5, 1, 4)
    out, _ = do.decode_attention(q, k, v, np.zeros((1, 1), int), np.array([5]), scale=0.4, softcap_value=1.5)
    for h in range(2):
        p = co.probabilities(q[0, h][None], k[0, :, 0], 5, scale=0.4, softcap=1.5)
        assert np.allclose(p @ v[0, :, 0], out[0, h])


def test_eviction_against_every_choice():
    """Of all subsets that hold the protected slots, the kept one is the heaviest, and the first of equal ones."""
    rng = np.random.default_rng(5)
    for _ in range(40):
        n, budget = int(rng.integers(1, 8)), int(rng.integers(1, 8))
        sinks = int(rng.integers(0, budget + 1))
        recent = int(rng.integers(0, budget - sinks + 1))
        w = rng.integers(0, 3, (1, 1, 8)).astype(np.float32)
        lens, kept = co.evict(w, [n], budget, sinks, recent)
        m = min(n, budget)
        assert lens[0] == m and (kept[0, 0, m:] == -1).all()
        must = {j for j in range(n) if j < sinks or j >= n - recent} if n > budget else set()
        choices = [c for c in itertools.combinations(range(n), m) if must <= set(c)]
        best = max(choices, key=lambda c: (w[0, 0, list(c)].sum(), [-j for j in c]))
        assert w[0, 0, list(best)].sum() == w[0, 0, kept[0, 0, :m]].sum()
        free = sorted(set(range(n)) - must)
        want = sorted(must | set(sorted(free, key=lambda j: (-w[0, 0, j], j))[:m - len(must)])) if n > budget else list(range(n))
        assert kept[0, 0, :m].tolist() == want


def test_a_nan_weight_goes_first():
    w = np.array([[[1.0, np.nan, -np.inf, 2.0]]], dtype=np.float32)
    assert co.evict(w, [4], 3, 0, 0)[1].tolist() == [[[0, 2, 3]]]
