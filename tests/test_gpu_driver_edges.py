"""The shared-prompt cache driver with arguments at and past the ends of their ranges."""
import math

import pytest
import torch

from paper_2407_08103_b200.decode import SharedPromptCache

DEV = "cuda:0"
pytestmark = pytest.mark.gpu
B, H, K, D = 4, 4, 2, 64


def normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV).bfloat16()


def fresh(seed=1, budget=12, **kw):
    g = torch.Generator(device=DEV).manual_seed(seed)
    cache = SharedPromptCache(normal(g, 20, K, D), normal(g, 20, K, D), B, H, budget=budget, **dict(dict(max_tokens=3), **kw))
    return g, cache


def test_counts_past_the_tokens_given_are_clamped_in_the_positions_too():
    g, cache = fresh()
    q, k, v = normal(g, B, 2, H, D), normal(g, B, 2, K, D), normal(g, B, 2, K, D)
    n = torch.tensor([-3, 1, 2, 9], dtype=torch.int32, device=DEV)
    cache.step(q, k, v, n_new=n)
    assert cache.lens.tolist() == cache.pos.tolist() == [0, 1, 2, 2]
    cache.step(q, k, v, n_new=n[:, None])                  # one entry per row is what counts
    assert cache.lens.tolist() == cache.pos.tolist() == [0, 2, 4, 4]
    assert [sorted(cache.age[b, 0, :x].tolist()) for b, x in enumerate([0, 2, 4, 4])] == [[], [0, 1], [0, 1, 2, 3], [0, 1, 2, 3]]


def test_a_refused_step_changes_nothing():
    g, cache = fresh()
    q, k, v = normal(g, B, 2, H, D), normal(g, B, 2, K, D), normal(g, B, 2, K, D)
    cache.step(q, k, v)
    before = [t.clone() for t in (cache.k, cache.v, cache.weight, cache.age, cache.lens, cache.pos)]
    wide = torch.zeros(B, 2, H, D + 4, dtype=torch.bfloat16, device=DEV)
    shifted = torch.zeros(B * 2 * H * D + 4, dtype=torch.bfloat16, device=DEV)[4:].view(B, 2, H, D)
    for kw in (dict(q=q[:, :1]), dict(k=k[:, :1], v=v[:, :1]), dict(v=v[:, :1]), dict(q=q.float()), dict(q=q[:, :, :2]),
               dict(q=wide[..., :D]), dict(q=shifted), dict(q=q[0]), dict(q=q.cpu()), dict(scale=math.inf), dict(scale=math.nan), dict(scale=1e39),
               dict(n_new=torch.ones(B, device=DEV)), dict(n_new=torch.ones(B - 1, dtype=torch.int32, device=DEV)),
               dict(q=q[:, :0], k=k[:, :0], v=v[:, :0]),
               dict(q=q.repeat(1, 2, 1, 1), k=k.repeat(1, 2, 1, 1), v=v.repeat(1, 2, 1, 1))):
        with pytest.raises((TypeError, ValueError, RuntimeError)):
            cache.step(**dict(dict(q=q, k=k, v=v), **kw))
        after = (cache.k, cache.v, cache.weight, cache.age, cache.lens, cache.pos)
        assert all(torch.equal(x.nan_to_num(), y.nan_to_num()) for x, y in zip(before, after)), kw.keys()
