"""A constrained student learns a constrained teacher's answers.

    python examples/distill.py [--rows N] [--steps K] [--updates U]

A small random language model, the teacher, answers under the API-call constraint: every token is drawn with
temperature and top-p from one uniform number a row, and the teacher's most likely tokens at every position are kept
as a record.  Then a student - the same embedding, another output layer - is trained on the records: the divergence of
its constrained distribution from them, the tail as one event.
"""

from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2407_08103_b200 import cstr  # noqa: E402
from paper_2407_08103_b200.decode import ConstrainedDecoder  # noqa: E402
from paper_2407_08103_b200.train import constrained_distill_loss  # noqa: E402
from synth.configs import config_dfas, config_vocab  # noqa: E402

WIDTH, RECORD = 128, 16


def answers(table, embed, head, rows, steps, g, device):
    """Hidden vectors, the states before each token and the teacher's records, ``[steps][rows]``, and the tokens."""
    dec = ConstrainedDecoder(table, rows, device=device)
    h = embed[torch.randint(0, embed.shape[0], (rows,), generator=g, device=device)]
    hidden, states, ids, logps, tokens = [], [], [], [], []
    for _ in range(steps):
        logits = h @ head.T
        hidden.append(h)
        states.append(dec.states.clone())
        record = dec.top_logprobs(logits, RECORD, temperature=0.8)
        ids.append(record[0])
        logps.append(record[1])
        u = torch.rand(rows, generator=g, device=device)
        token, _ = dec.sample(logits, u, temperature=0.8, top_p=0.95)
        tokens.append(token.clone())
        h = 0.5 * h + embed[token.clamp(min=0).long()]
    return tuple(torch.stack(x) for x in (hidden, states, ids, logps, tokens))


def main(rows=32, steps=40, updates=5, seed=0):
    device = torch.device("cuda:0")
    dfa = config_dfas("api_1k")[0]
    vb, vo = config_vocab("api_1k")
    table = cstr.cstr_build_token_table(cstr.cstr_load_dfa(*dfa), vb, vo)
    g = torch.Generator(device=device).manual_seed(seed)
    vocab = vo.size - 1
    embed = torch.randn(vocab, WIDTH, generator=g, device=device)
    teacher = torch.randn(vocab, WIDTH, generator=g, device=device) / WIDTH ** 0.5
    student = (0.1 * torch.randn(vocab, WIDTH, generator=g, device=device)).requires_grad_()
    hidden, states, ids, logps, tokens = answers(table, embed, teacher, rows, steps, g, device)
    h, real = hidden.reshape(-1, WIDTH), tokens.reshape(-1) >= 0
    flat = dict(teacher_ids=ids.reshape(-1, RECORD), teacher_logp=logps.reshape(-1, RECORD), tables=table,
                states=states.reshape(-1), weight=(real / real.sum()).contiguous(), tail=cstr.CSTR_TAIL_LUMP, temperature=0.8)
    losses = []
    for _ in range(updates):
        total = constrained_distill_loss(h @ student.T, **flat).sum()
        total.backward()
        with torch.no_grad():
            student -= 2.0 * student.grad
            grad, student.grad = student.grad, None
        losses.append(float(total.detach()))
    answer = b"".join(bytes(vb[vo[t]:vo[t + 1]]) for t in tokens[:, 0].tolist() if t >= 0)
    print("first answer: %r" % answer)
    print("divergence per update:", " ".join("%.5f" % x for x in losses))
    return losses, grad, dict(flat, hidden=h)


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--rows", type=int, default=32)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--updates", type=int, default=5)
    a = ap.parse_args()
    main(a.rows, a.steps, a.updates)
