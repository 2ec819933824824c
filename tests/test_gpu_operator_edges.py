"""Edges of the cache and loss operators at which a call once went wrong."""
import math

import numpy as np
import pytest
import torch

from paper_2407_08103_b200 import cstr

from operator_cases import DEV, AttentionCase

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


# rows shared by clusters of 2 to 16 blocks, the last ones with short shares or (narrow rows) none
@pytest.mark.parametrize("N,V", [(1, 8193), (2, 16385), (1, 65537), (40, 32769), (9, 131073), (300, 16390)])
@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_loss_of_rows_shared_by_a_cluster(dtype, N, V):
    g = torch.Generator(device=DEV).manual_seed(V)
    x = torch.randn(N, V, generator=g, device=DEV).to(dtype)
    act = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    adv = torch.ones(N, device=DEV)
    want = torch.log_softmax(x.double(), 1).gather(1, act.long()[:, None])[:, 0]
    runs = []
    for _ in range(20):
        loss, logp, d = torch.empty(N, device=DEV), torch.empty(N, device=DEV), torch.empty_like(x)
        cstr.cstr_policy_loss(None, x, None, act, want.float(), adv, loss, logp, dlogits=d)
        runs.append((loss, logp, d))
    assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(runs[0], r))
    # logits below 8 and log probabilities below 32 in 32 bits, the sum of the exponentials to 2^-18
    assert (runs[0][1].double() - want).abs().max() <= 2.0 ** -21 * 41 + 2.0 ** -18
