"""The oracle of the operators over whole distributions against small examples and identities."""
import numpy as np
import pytest

from oracle import distributions as ref


def test_cuts_of_a_known_row():
    # probabilities 0.1, 0.4, 0.2, 0.3 and one token that is not allowed
    x = np.log(np.array([[0.1, 0.4, 0.2, 0.3, 9.0]]))
    ok = np.array([[True] * 4 + [False]])

    def draw(u, **kw):
        return ref.sample(x, ok, [u], **{k: [v] for k, v in kw.items()})
    assert [int(draw(u)[0][0]) for u in (0.05, 0.15, 0.55, 0.75, 0.999)] == [0, 1, 2, 3, 3]
    assert [int(draw(u, top_k=2)[0][0]) for u in (0.0, 0.56, 0.58)] == [1, 1, 3]
    # 0.4 + 0.3 reach 0.65 and 0.75 does not: of {1, 3}, then {1, 2, 3}
    assert [int(draw(u, top_p=0.65)[0][0]) for u in (0.0, 0.58)] == [1, 3]
    assert [int(draw(u, top_p=0.75)[0][0]) for u in (0.4, 0.5, 0.7)] == [1, 2, 3]
    assert [int(draw(u, min_p=0.5)[0][0]) for u in (0.4, 0.5, 0.7)] == [1, 2, 3]
    assert draw(0.3, min_p=0.6)[2][0] == pytest.approx(0.7) and draw(0.3, top_k=2)[1][0] == pytest.approx(np.log(0.4))
    # top_p counts what top_k leaves: 0.5 of {1, 3} is in {1}
    assert draw(0.9, top_k=2, top_p=0.5)[0][0] == 1
    assert draw(0.9, temperature=0.0)[0][0] == 1 and draw(0.9, temperature=0.0)[1][0] == 0.0


def test_rows_without_probability():
    x = np.array([[-np.inf, -np.inf, np.nan], [np.nan, np.nan, np.nan], [0.0, 0.0, 0.0], [np.inf, 1.0, np.inf]])
    ok = np.array([[False, True, True], [True] * 3, [False] * 3, [True] * 3])
    token, logp, kept = ref.sample(x, ok, [0.5] * 4)
    assert token.tolist() == [1, -1, -1, 2] and np.isneginf(logp[:3]).all() and logp[3] == pytest.approx(-np.log(2))
    ids, logp, lse = ref.top(x, ok, 3)
    assert ids.tolist() == [[-1] * 3, [-1] * 3, [-1] * 3, [0, 2, 1]] and np.isneginf(logp[3, 2]) and lse[3] == np.inf


def test_top_agrees_with_a_sorted_softmax():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((5, 40)) * 3
    x[:, 7] = x[:, 3]
    ids, logp, lse = ref.top(x, np.ones((5, 40), bool), 40, 0.7)
    p = np.exp(x / 0.7)
    assert np.allclose(np.exp(logp), np.take_along_axis(p / p.sum(1, keepdims=True), ids, 1))
    assert np.allclose(lse, np.log(p.sum(1))) and (np.diff(logp, axis=1) <= 0).all()
    for i in range(5):
        assert list(ids[i]).index(3) + 1 == list(ids[i]).index(7)


@pytest.mark.parametrize("tail", [ref.DROP, ref.RENORM, ref.LUMP])
def test_divergence_agrees_with_its_differences_and_is_zero_for_the_teacher(tail):
    rng = np.random.default_rng(tail)
    x = rng.standard_normal((4, 20)) * 2
    ok = rng.random((4, 20)) < 0.8
    ok[:, :3] = True
    ids, logp, _ = ref.top(x + 0.3 * rng.standard_normal(x.shape), ok, 5)
    ids[1, 3] = ids[1, 0]
    ids[2, 4] = -1
    loss, grad = ref.distill(x, ok, ids, logp, tail, temperature=0.8)
    h = 1e-6
    for v in range(20):
        step = np.zeros_like(x)
        step[:, v] = h
        up, down = (ref.distill(x + s * step, ok, ids, logp, tail, temperature=0.8)[0] for s in (1, -1))
        assert np.allclose((up - down) / (2 * h), grad[:, v], atol=1e-8)
    ids, logp, _ = ref.top(x, ok, 5, 0.8)
    same = ref.distill(x, ok, ids, logp, tail, temperature=0.8)
    if tail == ref.LUMP:
        assert np.abs(same[0]).max() < 1e-14 and np.abs(same[1]).max() < 1e-14
    if tail == ref.DROP:
        assert np.abs(same[0]).max() < 1e-14
