"""Pins of the oracle of rotary positions and of the paged cache."""
import numpy as np
import pytest

from oracle import paged


def test_frequencies_by_hand():
    assert np.allclose(paged.frequencies(4, 100.0), [1.0, 0.1])
    assert np.allclose(paged.frequencies(4, 100.0, stretch=4.0), [0.25, 0.025])
    # turns in 20 pi tokens: 10 and 1; between 1 and 4 in proportion
    f = paged.frequencies(4, 100.0, stretch=8.0, original=20 * np.pi, slow=1.0, fast=4.0)
    assert np.allclose(f, [1.0, 0.1 / 8])
    f = paged.frequencies(2, 1.0, stretch=2.0, original=5 * np.pi, slow=1.0, fast=4.0)      # 2.5 turns: half and half
    assert np.allclose(f, [0.75])


@pytest.mark.parametrize("interleaved", [False, True])
def test_a_quarter_turn_swaps_a_pair(interleaved):
    x = np.arange(1.0, 9.0)[None]
    y = paged.rotate(x, [1], [np.pi / 2, np.pi], interleaved, factor=2.0)[0]
    want = [-4, 2, -6, -8] if interleaved else [-6, -4, 2, -8]
    assert np.allclose(y[:4], want) and (y[4:] == x[0, 4:]).all()


def test_turning_leaves_products_to_distances():
    r = np.random.RandomState(0)
    q, k, f = r.randn(1, 8), r.randn(1, 8), paged.frequencies(8)
    at = lambda p, t: float((paged.rotate(q, [p], f) @ paged.rotate(k, [t], f).T)[0, 0])  # noqa: E731
    assert np.isclose(at(7, 3), at(104, 100)) and not np.isclose(at(7, 3), at(7, 4))


def test_scores_by_hand():
    q, K = np.array([[1.0], [2.0]]), np.array([[1.0], [2.0], [3.0]])
    assert np.allclose(paged.scores(q, K, 0.5), [[0.5, 1, 1.5], [1, 2, 3]])
    s = paged.scores(q, K, 0.5, softcap=2.0, slopes=[1.0, 0.0], window=2)
    assert np.allclose(s[:, 1:], [[2 * np.tanh(0.5) - 1, 2 * np.tanh(0.75)], [2 * np.tanh(1.0), 2 * np.tanh(1.5)]])
    assert (s[:, 0] == -np.inf).all()
    assert np.allclose(paged.probabilities(s)[:, 0], 0) and np.allclose(paged.probabilities(s).sum(-1), 1)


def test_kept_by_hand():
    w = [5, 1, 7, 1, 0, 1, 0]
    assert list(paged.kept(w, 4, 2)) == [0, 2, 5, 6]
    assert list(paged.kept(w, 4, 1)) == [0, 1, 2, 6]       # among the ones the first
    assert list(paged.kept(w, 3, 3)) == [4, 5, 6] and list(paged.kept(w, 0, 0)) == []
    assert list(paged.kept(w, 7, 2)) == list(range(7))


@pytest.mark.parametrize("page,d", [(32, 64), (64, 96), (128, 128)])
def test_places_of_a_pool_are_all_different(page, d):
    g, h, t, c = np.meshgrid(np.arange(2), np.arange(3), np.arange(page), np.arange(d), indexing="ij")
    for which in "kv":
        at = paged.page_index(which, g, h, t, c, 3, page, d)
        assert (np.sort(at.ravel()) == np.arange(2 * 3 * page * d)).all()
