"""The oracle of the cache and loss operators against differences, identities and small examples."""
import numpy as np
import pytest

from oracle import operators as ref


def test_attention_of_one_key_returns_its_value_and_none_returns_zero():
    q = np.ones((1, 2, 2, 4))
    pk, pv = np.zeros((0, 1, 4)), np.zeros((0, 1, 4))
    ck = np.ones((1, 3, 1, 4))
    cv = np.arange(12.0).reshape(1, 3, 1, 4)
    age = np.array([[[5, 6, 7]]])
    r = ref.attention(q, pk, pv, ck, cv, [1], 0.5, weight=np.zeros((1, 1, 3)))
    assert np.array_equal(r["out"][0, 0, 1], cv[0, 0, 0]) and r["lse"][0, 0, 0] == 2.0
    assert np.array_equal(r["weight"][0, 0], [4.0, 0.0, 0.0])
    r = ref.attention(q, pk, pv, ck, cv, [3], 0.5, age=age, pos=[4])
    assert np.isneginf(r["lse"][0, 0]).all() and (r["out"][0, 0] == 0).all()
    assert np.array_equal(r["out"][0, 1, 0], cv[0, 0, 0])       # token 1 sees position 5


def test_insert_examples():
    ck = np.arange(6.0).reshape(1, 6, 1, 1)
    w = np.array([[[0.5, 0.1, 0.1, np.nan, 9.0, 9.0]]], np.float32)
    age = np.array([[[0, 1, 2, 3, 9, 9]]], np.int32)
    new = np.array([[[[70.0]], [[71.0]]]])
    # four filled, budget four, two new: the NaN and the first of the equal weights go
    k, v, w2, a2, n = ref.insert(ck, ck, w, age, [4], new, new, [4], 4, 0)
    assert k[0, :, 0, 0].tolist() == [0, 70, 2, 71, 4, 5] and n.tolist() == [4]
    assert a2[0, 0].tolist() == [0, 4, 2, 5, 9, 9] and w2[0, 0, 1] == 0 and w2[0, 0, 3] == 0
    # the last three positions (two new ones, position 3) are kept
    k, *_ = ref.insert(ck, ck, w, age, [4], new, new, [4], 4, 3)
    assert k[0, :, 0, 0].tolist() == [0, 70, 71, 3, 4, 5]
    # shrinking: an old survivor past the budget moves into the freed slot
    k, *_, n = ref.insert(ck, ck, w, age, [4], None, None, [4], 2, 1)
    assert k[0, :2, 0, 0].tolist() == [0, 3] and n.tolist() == [2]


@pytest.mark.parametrize("seed", range(6))
def test_policy_gradient_agrees_with_differences(seed):
    rng = np.random.default_rng(seed)
    N, V = 5, 17
    x = rng.standard_normal((N, V)) * 2
    allowed = rng.random((N, V)) < 0.7
    allowed[:, 3] = True
    act = np.full(N, 3)
    kw = dict(ref_logp=rng.standard_normal(N) - 2, weight=rng.random(N), kl_coef=0.3, temperature=0.7)
    _, lp, _ = ref.policy_loss(x, allowed, act, np.zeros(N), np.ones(N))
    old, adv = lp + rng.standard_normal(N) * 0.5, rng.standard_normal(N)
    _, _, g = ref.policy_loss(x, allowed, act, old, adv, **kw)
    h = 1e-6
    for i in range(N):
        for v in range(V):
            up, dn = x.copy(), x.copy()
            up[i, v] += h
            dn[i, v] -= h
            above = ref.policy_loss(up, allowed, act, old, adv, **kw)[0][i]
            below = ref.policy_loss(dn, allowed, act, old, adv, **kw)[0][i]
            # the two losses' rounding (a few units of 2^-53 of their terms) over 2 h
            noise = 2.0 ** -48 * (abs(above) + abs(adv[i]) + 1.0) / h
            assert abs((above - below) / (2 * h) - g[i, v]) < 1e-6 * (1 + abs(g[i, v])) + noise
