"""Training on constrained answers: the policy loss as a differentiable torch function.

The loss is over the constrained distribution (disallowed logits are -infinity, as
in Algorithm 2's loop body), because that is the distribution the answers were sampled from.
"""

from __future__ import annotations

import torch

from . import cstr


def _builds(tables):
    return [t.builds for t in tables]


class _Once(torch.autograd.Function):
    """A gradient whose own derivative is not there."""

    @staticmethod
    def forward(ctx, gradient, *inputs):
        return gradient

    @staticmethod
    def backward(ctx, _):
        raise RuntimeError("constrained_policy_loss is differentiable once only")


class _PolicyLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, actions, old_logp, advantages, ref_logp, weight, args):
        n = logits.shape[0]
        loss, logp = (torch.empty(n, dtype=torch.float32, device=logits.device) for _ in range(2))
        cstr.cstr_policy_loss(args["tables"], logits, args["states"], actions, old_logp, advantages,
                              loss, logp, ref_logp=ref_logp, weight=weight, **args["options"])
        # The backward pass takes the loss again.  The library writes states and tokens in place through
        # their addresses (a decoder that steps on), which autograd's versions do not show: so the
        # per-row arrays are kept as copies, a few bytes a row.
        if ctx.needs_input_grad[0]:
            rows = (args["states"], actions, old_logp, advantages, ref_logp, weight, args["options"]["row_table"])
            ctx.save_for_backward(logits, *(None if t is None else t.clone() for t in rows))
            ctx.builds = _builds(args["tables"])
        ctx.args = args
        ctx.mark_non_differentiable(logp)
        return loss, logp

    @staticmethod
    def backward(ctx, grad_loss, _):
        if not ctx.needs_input_grad[0]:
            return (None,) * 7
        if _builds(ctx.args["tables"]) != ctx.builds:
            raise RuntimeError("a table of this loss was built again before its backward pass")
        # the gradient of row n is linear in its weight, so the upstream gradient enters there;
        # nothing but the logits is kept in between
        logits, states, actions, old_logp, advantages, ref_logp, weight, row_table = ctx.saved_tensors
        grad = grad_loss.float()
        grad = grad.contiguous() if weight is None else grad * weight.flatten()[:grad.shape[0]]
        dlogits = torch.empty_strided(logits.shape, logits.stride(), dtype=logits.dtype,
                                      device=logits.device)
        loss, logp = torch.empty_like(grad), torch.empty_like(grad)
        cstr.cstr_policy_loss(ctx.args["tables"], logits, states, actions, old_logp, advantages, loss, logp,
                              ref_logp=ref_logp, weight=grad, dlogits=dlogits,
                              **dict(ctx.args["options"], row_table=row_table))
        if torch.is_grad_enabled():              # create_graph: the gradient is a function of these, too
            dlogits = _Once.apply(dlogits, logits, grad_loss)
        return dlogits, None, None, None, None, None, None


def constrained_policy_loss(logits, actions, old_logp, advantages, tables=None, states=None,
                            ref_logp=None, weight=None, row_table=None, clip_low: float = 0.2,
                            clip_high: float = 0.2, kl_coef: float = 0.0, temperature: float = 1.0):
    """``(loss [N], logp [N])`` of ``cstr_policy_loss``; the loss is differentiable in ``logits``
    (float32 or bfloat16 ``[N][V]``), the log probabilities are not."""
    tables = [tables] if isinstance(tables, cstr.Table) else list(tables or [])
    args = dict(tables=tables, states=states,
                options=dict(row_table=row_table, clip_low=clip_low, clip_high=clip_high,
                             kl_coef=kl_coef, temperature=temperature))
    return _PolicyLoss.apply(logits, actions, old_logp, advantages, ref_logp, weight, args)
