"""The oracle of draws from given numbers: by hand, and against softmax probabilities (CPU)."""
import math

import numpy as np
import pytest

from oracle import draw as D

L = np.log(np.array([0.1, 0.4, 0.2, 0.3], dtype=np.float64)).astype(np.float32)


@pytest.mark.parametrize("settings, ids", [
    (dict(), [0, 1, 2, 3]),
    (dict(top_k=2), [1, 3]),
    (dict(top_k=9), [0, 1, 2, 3]),
    (dict(top_p=0.39), [1]),
    (dict(top_p=0.41), [1, 3]),
    (dict(top_p=0.0), [1]),
    (dict(top_k=3, top_p=0.77), [1, 3]),       # 0.7 of 0.9 is more than 0.77
    (dict(top_k=3, top_p=0.78), [1, 2, 3]),
    (dict(min_p=0.49), [1, 2, 3]),
    (dict(min_p=0.51), [1, 3]),
    (dict(min_p=7.0), [1]),
    (dict(top_k=2, min_p=0.9), [1]),
    (dict(temperature=0.0), [1]),
    (dict(temperature=0.1, min_p=0.05), [1, 3]),  # (3/4)^10 = 0.056
])
def test_what_is_kept(settings, ids):
    assert list(D.kept(L, **settings)) == ids


def test_probabilities():
    f = D.kept(L)
    total = sum(f.values())
    assert np.allclose([f[i] / total for i in range(4)], [0.1, 0.4, 0.2, 0.3], rtol=4e-7)
    u = (np.arange(1 << 12) + 0.5) / (1 << 12)
    tokens, logp = zip(*(D.draw(L, x) for x in u))
    assert np.allclose(np.bincount(tokens) / len(u), [0.1, 0.4, 0.2, 0.3], atol=1 / 4096)
    assert np.allclose(np.exp(logp), np.take([0.1, 0.4, 0.2, 0.3], tokens), rtol=4e-7)
    assert list(tokens) == sorted(tokens)


def test_ties_go_to_the_lowest_id():
    x = np.float32([1, 2, 2, -0.0, 0.0, 2])
    assert list(D.kept(x, top_k=1)) == [1] and list(D.kept(x, top_k=2)) == [1, 2]
    assert list(D.kept(x, top_k=5)) == [0, 1, 2, 3, 5]
    assert list(D.kept(x, top_p=0.3)) == [1, 2]
    assert D.draw(x, 0.9, temperature=0) == (1, 0.0)


def test_ends():
    inf, nan = np.inf, np.nan
    assert D.draw(np.float32([-inf, nan, -inf]), 0.3) == (-1, -math.inf)
    assert D.draw(np.float32([nan, -inf, 3, -inf]), 0.999) == (2, 0.0)
    assert list(D.kept(np.float32([inf, 5, nan, inf]))) == [0, 3]
    assert D.draw(np.float32([0, 0]), 0.0)[0] == 0 and D.draw(np.float32([0, 0]), 1.0)[0] == 1
    assert D.draw(np.float32([0, 0]), nan)[0] == 0 and D.draw(np.float32([0, 0]), -1.0)[0] == 0
    assert D.draw(np.float32([0, 0]), 0.5)[0] == 1 and D.draw(np.float32([0, 0]), np.nextafter(np.float32(0.5), np.float32(0)))[0] == 0
    assert list(D.kept(np.float32([0, -28, -29]))) == [0, 1]  # e^-29 2^40 = 0.28
