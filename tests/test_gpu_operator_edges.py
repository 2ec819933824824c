"""Edges of the cache and loss operators at which a call once went wrong."""
import math

import numpy as np
import pytest
import torch

from operator_cases import AttentionCase

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


# P: prompt in the row kernel (or none), on the tensor cores with one and with two tiles of query rows
@pytest.mark.parametrize("P,B", [(0, 2), (33, 2), (700, 2), (700, 40)])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_a_single_token_is_not_reached_by_slots_it_does_not_see(dtype, value, P, B):
    c = AttentionCase(51, B, 1, 8, 2, 64, P, 40, dtype, causal=True, lens=[40, 21] * (B // 2))
    for b in range(B):
        for h in range(2):
            j = int(np.argmax(c.age[b, h, :c.lens[b]] == 7))
            c.age[b, h, j] = c.pos[b] + 3                  # younger than the token
            c.ck[b, j, h] = value
            c.cv[b, j, h] = value
    c.dev()
    c.run()
    c.check()
    assert torch.isfinite(c.out).all() and torch.isfinite(c.d_w).all()


# long caches of one row whose weights are computed from the keys again (63 and 8 query rows), and
# one whose scores are kept
@pytest.mark.parametrize("P,cap,T,G,D", [(100, 10000, 9, 7, 128), (600, 10000, 9, 7, 128), (100, 48000, 4, 2, 128),
                                         (0, 300, 9, 7, 64)])
@pytest.mark.parametrize("value", [math.nan, math.inf, 3e38])
def test_queries_past_n_query_do_not_reach_the_weights(value, P, cap, T, G, D):
    c = AttentionCase(52, 1, T, G, 1, D, P, cap, BF, causal=True, lens=[cap - 7], n_query=[2])
    c.q[0, 2:] = value                                     # padding: may hold anything
    c.dev()
    c.run()
    c.check()
    assert torch.isfinite(c.d_w).all()
