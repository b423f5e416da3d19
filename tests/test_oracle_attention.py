"""Pins of the oracle's prompt attention and bulk eviction: closed forms and agreement with the one-by-one eviction."""
import numpy as np

from oracle import uncomp_oracle as O


def test_equal_keys_average_the_values_they_see():
    v = np.arange(12.0).reshape(4, 3)
    out, lse, size = O.causal_attention(np.ones((3, 2)), np.zeros((4, 2)), v)
    for i in range(3):
        np.testing.assert_allclose(out[i], v[: i + 2].mean(axis=0))
        np.testing.assert_allclose(lse[i], np.log(i + 2))
    np.testing.assert_allclose(size, out)


def test_rows_that_see_nothing():
    out, lse, _ = O.causal_attention(np.ones((3, 2)), np.ones((1, 2)), np.full((1, 2), 5.0))
    assert (out[:2] == 0).all() and (lse[:2] == -np.inf).all() and (out[2] == 5.0).all()
    out, lse, _ = O.causal_attention(np.ones((1, 1)), np.full((2, 1), -np.inf), np.ones((2, 1)))
    assert (out == 0).all() and (lse == -np.inf).all()


def test_normalisers_are_those_of_the_window():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((40, 8)), rng.standard_normal((40, 8))
    _, lse, _ = O.causal_attention(q, k, k)
    want = O.window_lse(q[None, None, -5:], k[None, None], 1)
    np.testing.assert_allclose(lse[-5:], want.reshape(-1))


def test_bulk_eviction_removes_what_one_by_one_removes():
    rng = np.random.default_rng(1)
    cum, idx = rng.integers(0, 6, 50).astype(float), rng.permutation(200)[:50]
    order = O.evict_lowest(cum, idx, 20, 180, 10)
    left = sorted((cum[r], idx[r], r) for r in range(50) if idx[r] <= 170)[30:] + [(0, 0, r) for r in range(50) if idx[r] > 170]
    assert sorted(order) == sorted(r for _, _, r in left) and len(order) == 20
    stay = [r for r in order if r < 20]
    assert all(order[r] == r for r in stay) and [r for r in order if r >= 20] == sorted(r for r in order if r >= 20)
    assert O.evict_lowest(cum, idx, 50, 180, 10) == list(range(50))
    assert O.evict_lowest(cum, idx, 0, -1, 0) == list(range(50))
