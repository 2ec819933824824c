"""Records of the student's own distribution: what every way to treat the tail has to give, loss and gradient."""
import numpy as np
import pytest
import torch

from paper_2407_08103_b200 import cstr
from paper_2407_08103_b200.train import constrained_distill_loss, top_logprobs

from distribution_cases import BF, F32, allowed_rows, constrained, dev
from operator_cases import f8

pytestmark = pytest.mark.gpu
TAU = float(np.float32(0.9))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("tail", [cstr.CSTR_TAIL_DROP, cstr.CSTR_TAIL_RENORM, cstr.CSTR_TAIL_LUMP])
def test_loss_and_gradient_of_a_learned_record(dtype, tail):
    N, k = 30, 50
    _, x, tables, nexts, row_table, states = constrained(["json_32k"], 10, N, dtype)
    V = x.shape[1]
    allowed = allowed_rows(nexts, row_table, states, V)
    q = dev(states)
    ids, logp = top_logprobs(x, k, tables, q, temperature=TAU)
    a = x.clone().requires_grad_()
    loss = constrained_distill_loss(a, ids, logp, tables, q, tail=tail, temperature=TAU)
    loss.sum().backward()
    z = np.where(allowed, f8(x) / TAU, -np.inf)
    some = allowed.any(1)
    p = np.zeros((N, V))
    p[some] = np.exp(z[some] - z[some].max(1, keepdims=True))
    p[some] /= p[some].sum(1, keepdims=True)
    at = ids.cpu().numpy()
    listed = np.zeros((N, V + 1), bool)
    listed[np.arange(N)[:, None], np.where(at >= 0, at, V)] = True
    mine = np.where(listed[:, :V], p, 0.0)
    T = mine.sum(1)
    want_loss, want = np.zeros(N), np.zeros((N, V))
    if tail == cstr.CSTR_TAIL_DROP:                          # sum of q (log q - log q), and T q - q of the record
        want = (T[:, None] * p - mine) / TAU
    if tail == cstr.CSTR_TAIL_RENORM:                        # q / T against q
        want_loss[some] = -np.log(T[some])
        want[some] = (p - mine / np.maximum(T, 1e-300)[:, None])[some] / TAU
    # the record's own rounding (2^-24 of up to 30) enters once for every entry, log q's error besides: 400 units of
    # 2^-24 in the loss; the gradient's sums of probabilities carry as much of 1, the lumped rest's as much again, over
    # the temperature: 1,000; and its type's rounding, half a step
    assert (np.abs(f8(loss) - want_loss) <= 2.0 ** -24 * (400 + want_loss)).all()
    unit = {F32: 2.0 ** -24, BF: 2.0 ** -8}[dtype]
    assert (np.abs(f8(a.grad) - want) <= unit * np.abs(want) + 2.0 ** -24 * 1000).all()
    assert (f8(a.grad)[~allowed] == 0).all() and (f8(loss)[~some] == 0).all()
    if tail == cstr.CSTR_TAIL_RENORM:
        assert want_loss.max() > 0.01 and np.abs(want).max() > 1e-3
