"""A group of constrained answers to one prompt, and an update of the model from them.

    python examples/group_rollout.py [--rows N] [--steps K] [--updates U]

A small random language model (one attention layer) answers a 256-token prompt under the API-call
constraint: the rows share the prompt's keys and values, each keeps at most 16 tokens of its own
(the least attended ones are evicted), and every token is sampled under the constraint's mask.
Then the output layer is trained on the group with the clipped policy loss over the constrained
distribution; an answer's reward is the share of ``(`` among its tokens.
"""

from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2407_08103_b200 import cstr  # noqa: E402
from paper_2407_08103_b200.decode import ConstrainedDecoder, SharedPromptCache  # noqa: E402
from paper_2407_08103_b200.train import constrained_policy_loss  # noqa: E402
from synth.configs import config_dfas, config_vocab  # noqa: E402

HEADS, KV_HEADS, DIM, PROMPT, BUDGET, RECENT = 8, 2, 64, 256, 16, 4


class Model:
    def __init__(self, vocab, device, seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        width = HEADS * DIM

        def normal(*shape):
            return torch.randn(shape, generator=g, device=device) / shape[-1] ** 0.5
        self.embed = normal(vocab, width) * width ** 0.5
        self.wq, self.wk, self.wv = normal(width, width), normal(KV_HEADS * DIM, width), normal(KV_HEADS * DIM, width)
        self.head = normal(vocab, width).requires_grad_()

    def project(self, tokens):
        x = self.embed[tokens]

        def split(w, heads):
            return (x @ w.T).bfloat16().view(*tokens.shape, heads, DIM)
        return x, split(self.wq, HEADS), split(self.wk, KV_HEADS), split(self.wv, KV_HEADS)


def rollout(model, table, rows, steps, g, device):
    """Sampled tokens, the states before them and the hidden vectors, ``[steps][rows]``."""
    prompt = torch.randint(0, model.embed.shape[0], (PROMPT,), generator=g, device=device)
    _, _, pk, pv = model.project(prompt)
    cache = SharedPromptCache(pk, pv, rows, HEADS, BUDGET, RECENT)
    dec = ConstrainedDecoder(table, rows, device=device)
    token = prompt[-1:].expand(rows)
    states, tokens, hidden = [], [], []
    for _ in range(steps):
        x, q, k, v = model.project(token[:, None])
        alive = (dec.states >= 0).int()
        h = x[:, 0] + cache.step(q, k, v, n_new=alive).float().reshape(rows, -1)
        with torch.no_grad():
            logits = h @ model.head.T
        states.append(dec.states.clone())
        u = torch.rand(logits.shape, generator=g, device=device).clamp_(1e-20)
        out, _ = dec.step(logits, noise=-torch.log(-torch.log(u)))
        tokens.append(out.clone())
        hidden.append(h)
        token = out.clamp(min=0)
    assert cstr.cstr_cache_status(cache.handle) == 0
    return torch.stack(tokens), torch.stack(states), torch.stack(hidden), cache


def main(rows=32, steps=40, updates=5, seed=0):
    device = torch.device("cuda:0")
    dfa = config_dfas("api_1k")[0]
    vb, vo = config_vocab("api_1k")
    table = cstr.cstr_build_token_table(cstr.cstr_load_dfa(*dfa), vb, vo)
    model = Model(vo.size - 1, device, seed)
    g = torch.Generator(device=device).manual_seed(seed + 1)
    tokens, states, hidden, cache = rollout(model, table, rows, steps, g, device)
    real = tokens >= 0
    opening = torch.tensor([b"(" in bytes(vb[vo[i]:vo[i + 1]]) for i in range(vo.size - 1)], device=device)
    reward = (opening[tokens.clamp(min=0).long()] & real).float().sum(0) / real.sum(0).clamp(min=1)
    adv = ((reward - reward.mean()) / (reward.std() + 1e-6)).expand(steps, rows)
    flat = dict(actions=tokens.clamp(min=0).reshape(-1), advantages=adv.reshape(-1).contiguous(), tables=table,
                states=torch.where(real, states, -1).int().reshape(-1),
                weight=(real / real.sum()).reshape(-1).contiguous())
    h = hidden.reshape(-1, hidden.shape[-1])
    with torch.no_grad():
        zero = torch.zeros(h.shape[0], device=device)
        _, old = constrained_policy_loss(h @ model.head.T, old_logp=zero, **flat)
    old = torch.where(torch.isfinite(old), old, 0.0)
    losses = []
    for _ in range(updates):
        loss, _ = constrained_policy_loss(h @ model.head.T, old_logp=old, ref_logp=old, kl_coef=0.01, **flat)
        total = loss.sum()
        total.backward()
        with torch.no_grad():
            model.head -= 0.5 * model.head.grad
            model.head.grad = None
        losses.append(float(total.detach()))
    answer = b"".join(bytes(vb[vo[t]:vo[t + 1]]) for t in tokens[:, 0].tolist() if t >= 0)
    print("first answer: %r" % answer)
    print("cache lengths:", cache.lens.min().item(), "..", cache.lens.max().item())
    print("loss per update:", " ".join("%.5f" % x for x in losses))
    return losses, cache


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--rows", type=int, default=32)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--updates", type=int, default=5)
    a = ap.parse_args()
    main(a.rows, a.steps, a.updates)
