"""Pins of the oracle's norm and rotation of queries and keys."""
import numpy as np
import pytest

import oracle
from oracle.qk import pairs, treat


def rows(n=12, D=32, seed=0):
    return np.random.default_rng(seed).standard_normal((n, D))


@pytest.mark.parametrize("layout", ["adjacent", "halves", "axis_halves"])
def test_every_dim_belongs_to_one_pair(layout):
    p = pairs((8, 4), layout)
    assert sorted(d for lo, hi, _, _ in p for d in (lo, hi)) == list(range(12))
    assert [a for _, _, a, _ in p] == [0] * 4 + [1] * 2


@pytest.mark.parametrize("layout", ["adjacent", "halves", "axis_halves"])
def test_scores_depend_on_the_difference_of_places_only(layout):
    """Turned queries and keys meet as if one stood at the origin: the same content at places
    moved alike gives the same products."""
    q, k = rows(1, 16, 1), rows(1, 16, 2)
    qk = oracle.QK(norm=False, dims=(8, 8), layout=layout)
    grid = 6
    tq, tk = (treat(np.repeat(z, 36, 0), 1, None, qk, grid) for z in (q, k))
    s = tq @ tk.T
    at = lambda r, c: r * grid + c  # noqa: E731
    np.testing.assert_allclose(s[at(1, 2), at(3, 1)], s[at(2, 4), at(4, 3)], rtol=1e-12)
    np.testing.assert_allclose(s[at(0, 0), at(0, 0)], (q @ k.T)[0, 0], rtol=1e-12)
    assert abs(s[at(1, 2), at(3, 1)] - s[at(1, 2), at(3, 2)]) > 1e-6


def test_norm_and_gain():
    x = rows(5, 24)
    g = np.arange(1.0, 9.0)
    y = treat(x, 3, g, oracle.QK(norm=True, eps=0.0), 5).reshape(5, 3, 8)
    np.testing.assert_allclose((y / g * (y / g)).mean(-1), 1.0, rtol=1e-12)
    np.testing.assert_allclose(treat(x, 3, None, oracle.QK(norm=False, dims=(4, 4)), 5).reshape(5, 3, 8)[0], x.reshape(5, 3, 8)[0])


def test_turns_keep_lengths_and_the_other_dims():
    x = rows(20, 32)
    qk = oracle.QK(norm=False, dims=(4, 6), layout="axis_halves")
    y = treat(x, 2, None, qk, 4).reshape(20, 2, 16)
    x = x.reshape(20, 2, 16)
    np.testing.assert_array_equal(y[..., 10:], x[..., 10:])
    for lo, hi, _, _ in pairs(qk.dims, qk.layout):
        np.testing.assert_allclose(np.hypot(y[..., lo], y[..., hi]), np.hypot(x[..., lo], x[..., hi]), rtol=1e-12)
