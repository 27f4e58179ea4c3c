"""The oracle of the cache operators on infinities, and refusals of the binding (no GPU)."""

import numpy as np

from oracle import cache as O

INF = np.inf


def test_a_head_with_an_infinite_normaliser_adds_nothing_to_any_token():
    q = np.array([[[1.0, 2.0], [1.0, 1.0]], [[0.5, -1.0], [np.nan, 1.0]]])           # 2 queries of 2 heads
    K = np.array([[0.1, 0.2], [INF, 0.0], [-INF, 1.0], [0.3, -0.4]])
    see = np.ones((2, 4), dtype=bool)
    lse = np.array([[1.0, INF], [-INF, INF]])
    with np.errstate(all="ignore"):
        w = O.attention_weights(q, K, see, lse, 0.5)
    s = 0.5 * (K[[0, 3]] @ q[0, 0])
    assert np.allclose(w[[0, 3]], np.exp(s - 1.0)) and w[1] == INF and w[2] == 0.0
    with np.errstate(all="ignore"):
        assert np.array_equal(O.attention_weights(q, K, see, np.full((2, 2), INF), 0.5), np.zeros(4))
