"""The oracle of the cache operators on infinities, and refusals of the binding (no GPU)."""

import numpy as np
import pytest
import torch

from oracle import cache as O
from paper_2607_09052_amd import cache, cobs

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


@pytest.mark.parametrize("n", [0, cache.MAX_QUERIES + 1])
def test_binding_names_a_number_of_queries_out_of_range(n):
    cfg = cobs.Config(batch=2, num_q_heads=8, num_kv_heads=2, head_dim=128, max_seq_len=128, rank=0, budget=8, window=0)
    k = torch.zeros(2, 2, 128, 128, dtype=torch.bfloat16)
    q, seq, lse = torch.zeros(2, n, 8, 128), torch.zeros(2, dtype=torch.int32), torch.zeros(2, n, 8)
    with pytest.raises(cobs.CobsError, match="queries"):
        cache.cobs_tree_decode(cfg, q, k, k, seq, None, None, torch.zeros_like(q), torch.zeros(1 << 16))
    with pytest.raises(cobs.CobsError, match="queries"):
        cache.cobs_attention_weights(cfg, q, k, k, seq, None, None, lse, torch.zeros(2, 2, 128))
