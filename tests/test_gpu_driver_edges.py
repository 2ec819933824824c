"""The shared-prompt cache driver with arguments at and past the ends of their ranges."""
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
