"""What the differentiable distillation loss takes as constants, and records that the student has learned."""
import numpy as np
import pytest
import torch

from paper_2407_08103_b200 import cstr
from paper_2407_08103_b200.train import constrained_distill_loss

from distribution_cases import F32, logits
from operator_cases import DEV

pytestmark = pytest.mark.gpu


def batch(N=6, V=500, k=8):
    g = torch.Generator(device=DEV).manual_seed(1)
    ids = torch.stack([torch.randperm(V, generator=g, device=DEV)[:k] for _ in range(N)]).int()
    logp = torch.log_softmax(torch.randn(N, k + 1, generator=g, device=DEV), 1)[:, :k].contiguous()
    return logits(1, N, V, F32), ids, logp, torch.rand(N, generator=g, device=DEV)


def test_a_loss_of_constants_claims_no_gradient():
    x, ids, logp, w = batch()
    want = constrained_distill_loss(x, ids, logp, weight=w)
    lp, ww = logp.clone().requires_grad_(), w.clone().requires_grad_()
    for kw in (dict(teacher_logp=lp, weight=w), dict(teacher_logp=logp, weight=ww), dict(teacher_logp=lp, weight=ww)):
        loss = constrained_distill_loss(x, ids, **kw)
        assert torch.equal(loss, want) and not loss.requires_grad
        with pytest.raises(RuntimeError):
            loss.sum().backward()


@pytest.mark.parametrize("tail", [cstr.CSTR_TAIL_DROP, cstr.CSTR_TAIL_RENORM, cstr.CSTR_TAIL_LUMP])
def test_the_logits_gradient_beside_constants_that_track_theirs(tail):
    x, ids, logp, w = batch()
    grads = []
    for track in (False, True):
        a = x.clone().requires_grad_()
        lp, ww = logp.clone().requires_grad_(track), w.clone().requires_grad_(track)
        constrained_distill_loss(a, ids, 2.0 * lp, weight=0.5 * ww, tail=tail).sum().backward()
        assert lp.grad is None and ww.grad is None
        grads.append(a.grad)
    assert torch.equal(*grads) and np.isfinite(grads[0].abs().sum().item())
