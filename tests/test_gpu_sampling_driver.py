"""The decoder's sampling step, the teacher's records and the example that runs them into the distillation loss."""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

import oracle
from helpers import ROOT
from oracle import distributions as ref
from paper_2407_08103_b200 import cstr
from paper_2407_08103_b200.decode import ConstrainedDecoder
from paper_2407_08103_b200.train import constrained_distill_loss, constrained_policy_loss
from synth.configs import config_dfas, config_vocab

from distribution_cases import F32, dev, logits
from gpu_common import gpu_tables
from operator_cases import DEV, f8

pytestmark = pytest.mark.gpu


def decoder(B, names=("api_1k", "api_1k")):
    vb, vo = config_vocab(names[0])
    dfas = [config_dfas(n)[0] for n in names]
    tables = gpu_tables(dfas, vb, vo)
    nexts = [oracle.token_table(d[0], d[1], vb, vo)[0] for d in dfas]
    row_table = np.arange(B) % len(names)
    return ConstrainedDecoder(tables, B, row_table=row_table), nexts, row_table, vo.size - 1


def test_steps_follow_the_oracle_and_numbers_equal_tensors():
    B = 24
    rng = np.random.default_rng(1)
    dec, nexts, row_table, V = decoder(B)
    twin, _, _, _ = decoder(B)
    states = dec.states.cpu().numpy()
    for step in range(12):
        x = logits(step, B, V, F32)
        u = rng.random(B).astype(np.float32)
        allowed = np.stack([nexts[t][q] >= 0 if q >= 0 else np.zeros(V, bool) for t, q in zip(row_table, states)])
        want = ref.sample(f8(x), allowed, u, np.full(B, float(np.float32(0.8))), np.full(B, 30), np.full(B, float(np.float32(0.9))))
        ids, logp = dec.top_logprobs(x, 5, temperature=0.8)
        assert np.array_equal(ids.cpu().numpy(), ref.top(f8(x), allowed, 5, float(np.float32(0.8)))[0])
        tokens, lp = dec.sample(x, dev(u), temperature=0.8, top_k=30, top_p=0.9)
        assert np.array_equal(tokens.cpu().numpy(), want[0])
        states = np.array([nexts[t][q, w] if w >= 0 else -1 for t, q, w in zip(row_table, states, want[0])])
        assert np.array_equal(dec.states.cpu().numpy(), states)
        same, _ = twin.sample(x, dev(u), temperature=torch.full((B,), 0.8, device=DEV),
                              top_k=torch.full((B,), 30, dtype=torch.int32, device=DEV), top_p=torch.full((B,), 0.9, device=DEV))
        assert torch.equal(same, tokens) and torch.equal(twin.kept, dec.kept) and torch.equal(twin.accept, dec.accept)
    assert len(dec._settings) == 3


def test_greedy_sampling_is_the_step():
    B = 16
    dec, _, _, V = decoder(B)
    twin, _, _, _ = decoder(B)
    u = torch.rand(B, device=DEV)
    for step in range(8):
        x = logits(100 + step, B, V, F32)
        a, logp = dec.sample(x, u, temperature=0.0)
        b, _ = twin.step(x)
        assert torch.equal(a, b) and torch.equal(dec.states, twin.states) and torch.equal(dec.accept, twin.accept)
        assert ((logp == 0) | (a < 0)).all()


def test_settings_of_any_number_and_capture():
    B = 4
    dec, _, _, V = decoder(B)
    x, u = logits(3, B, V, F32), torch.rand(B, device=DEV)
    for i in range(70):                                       # an annealed temperature does not pile up
        dec.sample(x, u, temperature=0.5 + i / 100)
    assert len(dec._settings) <= 64
    with pytest.raises(ValueError, match="not a number"):
        dec.sample(x, u, top_p=math.nan)
    dec.reset()
    dec.sample(x, u, temperature=0.7)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with pytest.raises(RuntimeError, match="before the capture"):
        with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=side):
            dec.sample(x, u, temperature=0.123)
    torch.cuda.synchronize()
    dec.reset()
    want, _ = dec.sample(x, u, temperature=0.7)
    want = want.clone()
    with torch.cuda.graph(graph):
        dec.sample(x, u, temperature=0.7)
    dec.reset()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(dec.tokens, want)


def test_drawn_tokens_feed_the_policy_loss():
    # the log probabilities of a rollout are the old ones of its update: the ratio is 1, the gradient exact
    B = 32
    dec, _, _, V = decoder(B)
    x = logits(5, B, V, F32)
    before = dec.states.clone()
    tokens, logp = dec.sample(x, torch.rand(B, device=DEV), temperature=0.9)
    a = x.clone().requires_grad_()
    loss, again = constrained_policy_loss(a, tokens, logp, torch.ones(B, device=DEV), tables=dec.tables, states=before,
                                          row_table=dec.row_table, temperature=0.9)
    real = tokens >= 0
    # two roundings of a log-sum (units of 2^-24: log2 of the vocabulary, 36 additions and the result, each twice)
    assert ((loss + 1.0)[real].abs() <= 2 * 2.0 ** -24 * (2.1 * 10 + 36 + 30)).all()
    assert torch.equal(torch.isfinite(again), real)


def test_example_runs_and_its_gradient_is_that_of_the_formula():
    spec = importlib.util.spec_from_file_location("distill", os.path.join(ROOT, "examples", "distill.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    losses, grad, flat = m.main(rows=8, steps=12, updates=2)
    assert np.isfinite(losses).all() and torch.isfinite(grad).all() and grad.abs().sum() > 0
    # the gradient of the logits against the oracle, at the student's start
    h = flat.pop("hidden")
    a = (h @ torch.zeros(1024, h.shape[1], device=DEV).T + 0.01 * h[:, :1]).requires_grad_()
    constrained_distill_loss(a, **flat).sum().backward()
    d = config_dfas("api_1k")[0]
    vb, vo = config_vocab("api_1k")
    nxt = oracle.token_table(d[0], d[1], vb, vo)[0]
    q = flat["states"].cpu().numpy()
    allowed = np.stack([nxt[s] >= 0 if s >= 0 else np.zeros(1024, bool) for s in q])
    want = ref.distill(f8(a), allowed, flat["teacher_ids"].cpu().numpy(), f8(flat["teacher_logp"]), cstr.CSTR_TAIL_LUMP,
                       f8(flat["weight"]), float(np.float32(0.8)))
    assert np.abs(f8(a.grad) - want[1]).max() <= 2.0 ** -24 * 1000 * f8(flat["weight"]).max() / 0.8
