"""The differentiable policy loss, the shared-prompt cache driver and the example that runs them together."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from helpers import ROOT
from paper_2407_08103_b200 import cstr
from paper_2407_08103_b200.decode import SharedPromptCache
from paper_2407_08103_b200.train import constrained_policy_loss

DEV = "cuda:0"
pytestmark = pytest.mark.gpu


def test_autograd_matches_a_plain_loss_in_64_bits():
    g = torch.Generator().manual_seed(0)
    N, V = 12, 50
    x = torch.randn(N, V, generator=g, dtype=torch.float64)
    act = torch.randint(0, V, (N,), generator=g)
    adv, up = torch.randn(N, generator=g), torch.randn(N, generator=g)
    w = torch.rand(N, generator=g)
    plain = x.clone().requires_grad_()
    lp = torch.log_softmax(plain / 0.7, 1).gather(1, act[:, None])[:, 0]
    old = (lp.detach() + 0.1 * torch.randn(N, generator=g)).float()
    ratio = torch.exp(lp - old)
    diff = old - lp
    want = w * (-torch.minimum(ratio * adv, ratio.clamp(0.8, 1.2) * adv) + 0.1 * (torch.exp(diff) - diff - 1))
    (want * up).sum().backward()
    dev = x.float().to(DEV).requires_grad_()
    loss, logp = constrained_policy_loss(dev, act.int().to(DEV), old.to(DEV), adv.to(DEV), ref_logp=old.to(DEV),
                                         weight=w.to(DEV), kl_coef=0.1, temperature=0.7)
    (loss * up.to(DEV)).sum().backward()
    # 32-bit logits up to 4 / 0.7 and a few 2^-20 in the ratio
    assert torch.allclose(loss.double().cpu(), want.detach(), rtol=0, atol=2e-5)
    assert torch.allclose(logp.double().cpu(), lp.detach(), rtol=0, atol=1e-5)
    assert torch.allclose(dev.grad.double().cpu(), plain.grad, rtol=0, atol=5e-5)
    assert not logp.requires_grad


def test_driver_matches_a_growing_context():
    # with a budget that nothing exceeds, step by step equals attention over all tokens so far
    g = torch.Generator(device=DEV).manual_seed(1)
    B, H, K, D, P, steps = 3, 4, 2, 64, 150, 6

    def normal(*s):
        return torch.randn(s, generator=g, device=DEV).bfloat16()
    pk, pv = normal(P, K, D), normal(P, K, D)
    cache = SharedPromptCache(pk, pv, B, H, budget=16, recent=2, max_tokens=2)
    ks, vs = [], []
    for t in range(steps):
        T = 2 if t % 3 == 1 else 1
        q, k, v = normal(B, T, H, D), normal(B, T, K, D), normal(B, T, K, D)
        out = cache.step(q, k, v)
        for i in range(T):
            ks.append(k[:, i])
            vs.append(v[:, i])
            allk = torch.cat([pk.expand(B, P, K, D), torch.stack(ks, 1)], 1).double().repeat_interleave(H // K, 2)
            allv = torch.cat([pv.expand(B, P, K, D), torch.stack(vs, 1)], 1).double().repeat_interleave(H // K, 2)
            p = torch.softmax(torch.einsum("bhd,bxhd->bhx", q[:, i].double(), allk) / D ** 0.5, -1)
            want = torch.einsum("bhx,bxhd->bhd", p, allv)
            size = torch.einsum("bhx,bxhd->bhd", p, allv.abs())
            assert ((out[:, i].double() - want).abs() <= 2.0 ** -8 * (want.abs() + size)).all()
    assert cache.lens.tolist() == [len(ks)] * B == cache.pos.tolist()
    cache.reset()
    assert cache.lens.sum() == 0
    assert cstr.cstr_cache_status(cache.handle) == 0


def test_example_runs_and_its_loss_falls():
    spec = importlib.util.spec_from_file_location("group_rollout", os.path.join(ROOT, "examples", "group_rollout.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    losses, cache = m.main(rows=16, steps=30, updates=3)
    assert np.isfinite(losses).all() and losses[-1] < losses[0]
    assert int(cache.lens.max()) <= m.BUDGET
