"""Divergence from a teacher's records, and its gradient, against the oracle's statement in 64 bits."""
import math

import numpy as np
import pytest
import torch

from oracle import distributions as ref
from paper_2407_08103_b200 import cstr
from paper_2407_08103_b200.train import constrained_distill_loss, top_logprobs
from synth.configs import config_dfas, config_vocab

from distribution_cases import BF, F32, allowed_rows, check_distill, constrained, dev, logits
from gpu_common import gpu_tables
from operator_cases import DEV, f8

pytestmark = pytest.mark.gpu
TAILS = [cstr.CSTR_TAIL_DROP, cstr.CSTR_TAIL_RENORM, cstr.CSTR_TAIL_LUMP]


def records(rng, x, k, allowed=None, noise=0.5):
    """A teacher that agrees with the rows up to some noise: its k most likely tokens."""
    N, V = x.shape
    z = f8(x) + noise * rng.standard_normal((N, V))
    z = z if allowed is None else np.where(allowed, z, -np.inf)
    z = np.where(np.isnan(z), -np.inf, z)
    ids, logp, _ = ref.top(z, np.ones((N, V), bool), k)
    return ids.astype(np.int32), logp.astype(np.float32)


@pytest.mark.parametrize("N,V,k", [(1, 1, 1), (3, 2, 5), (5, 31, 4), (4, 33, 33), (3, 1000, 64), (3, 1024, 16),
                                   (2, 8200, 300), (2, 40001, 1), (1, 128256, 1024), (1, 300007, 100)])
@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("tail", TAILS)
def test_shapes(N, V, k, dtype, tail):
    rng = np.random.default_rng(N * V + k)
    x = logits(N * V + k, N, V, dtype)
    ids, logp = records(rng, x, k)
    check_distill(x, ids, logp, tail, weight=rng.random(N))
    check_distill(x, ids, logp, tail, gradient=False, temperature=1.7)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("ld,offset,shift", [(1024, 0, 0), (1031, 0, 0), (1040, 3, 0), (1024, 1, 0), (1008, 8, 1), (1031, 2, 3)])
def test_row_strides_alignment_and_in_place(dtype, ld, offset, shift):
    rng = np.random.default_rng(ld + offset)
    x = logits(ld + offset, 6, 1003, dtype, ld, offset)
    ids, logp = records(rng, x, 40)
    for tail in TAILS:
        check_distill(x, ids, logp, tail, shift=shift, temperature=0.7)
    whole = x.as_strided((6 * ld - (ld - 1003),), (1,))
    before = whole.clone()
    check_distill(x, ids, logp, cstr.CSTR_TAIL_LUMP, in_place=True)
    pad = torch.ones(whole.numel(), dtype=torch.bool, device=DEV)
    pad.as_strided((6, 1003), (ld, 1)).fill_(False)
    assert torch.equal(whole[pad], before[pad]) and not torch.equal(whole, before)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("tail", TAILS)
def test_constrained_rows_and_foreign_records(dtype, tail):
    N = 40
    rng, x, tables, nexts, row_table, states = constrained(["api_1k", "api_1k"], 3, N, dtype)
    states[3], states[4], row_table[6], row_table[7] = -1, 10 ** 6, 2, -1
    allowed = allowed_rows(nexts, row_table, states, x.shape[1])
    kw = dict(tables=tables, states=states, row_table=row_table, allowed=allowed, weight=rng.random(N))
    ids, logp = records(rng, x, 30, allowed)
    want = check_distill(x, ids, logp, tail, **kw)
    assert (want[0][[3, 4, 6, 7]] == 0).all()
    ids, logp = records(rng, x, 30)                          # a teacher without the constraint
    check_distill(x, ids, logp, tail, **kw)
    x[torch.from_numpy(~allowed).to(DEV)] = math.nan
    check_distill(x, ids, logp, tail, **kw)


@pytest.mark.parametrize("tail", TAILS)
def test_ids_twice_out_of_range_and_missing(tail):
    rng = np.random.default_rng(4)
    x = logits(4, 8, 5000, F32)
    ids, logp = records(rng, x, 20)
    ids[0, 3], ids[0, 9] = ids[0, 0], ids[0, 0]              # thrice
    ids[1, 1::2] = ids[1, ::2]
    ids[2, 4:] = -1
    ids[3, :] = -1
    ids[4, 2], ids[4, 3], ids[4, 4] = 5000, -2 ** 31, 2 ** 31 - 1
    logp[5, 3:] = -np.inf
    logp[6, :] = -np.inf
    check_distill(x, ids, logp, tail)
    check_distill(x.bfloat16(), ids, logp, tail, weight=rng.random(8))


def test_record_that_holds_everything_or_lies_far_above_the_rest():
    x = logits(5, 6, 600, F32)
    rng = np.random.default_rng(5)
    for k in (600, 599):                                     # no other token, one other
        ids, logp = records(rng, x, k)
        for tail in TAILS:
            check_distill(x, ids, logp, tail)
    # the rest's probability is far below what a float holds: its gradient is not lost
    ids, logp = records(rng, x, 10)
    far = x.clone()
    far.scatter_add_(1, dev(ids).long(), torch.full((6, 10), 400.0, device=DEV))
    logp = logp - 0.5
    want = check_distill(far, ids, logp, cstr.CSTR_TAIL_LUMP)
    assert (want[0] > 10).all() and (np.abs(want[1]).sum(1) > 0.5).all()


@pytest.mark.parametrize("scale", [1.0, 300.0])
def test_renormalised_records_may_be_logits(scale):
    rng = np.random.default_rng(6)
    x = logits(6, 6, 900, F32)
    ids, logp = records(rng, x, 12)
    check_distill(x, ids, logp + np.float32(scale) * rng.standard_normal((6, 1)).astype(np.float32), cstr.CSTR_TAIL_RENORM)


@pytest.mark.parametrize("tail", TAILS)
def test_nonfinite_logits_and_records(tail):
    rng = np.random.default_rng(7)
    x = logits(7, 9, 2500, F32)
    ids, logp = records(rng, x, 8)
    x[0, 5] = math.nan
    x[1] = -math.inf
    x[2, int(ids[2, 0])] = -math.inf
    x[3] = torch.finfo(F32).min
    x[4] = math.nan
    x[5, int(ids[5, 1])] = math.nan
    logp[6, 2] = math.nan
    x[7, 100:] = -math.inf
    weight = np.ones(9)
    weight[4] = 0.0                                          # padding: nothing comes of its NaN
    want = check_distill(x, ids, logp, tail, weight=weight)
    assert np.isnan(want[0][[0, 5, 6]]).all() and want[0][1] == 0 and want[0][4] == 0


@pytest.mark.parametrize("tail", TAILS)
def test_gradient_agrees_with_differences_of_the_loss(tail):
    N = 24
    rng, x, tables, nexts, row_table, states = constrained(["api_1k"], 8, N, F32)
    allowed = allowed_rows(nexts, row_table, states, x.shape[1])
    ids, logp = (dev(a) for a in records(rng, x, 12, allowed))
    q = dev(states)

    def loss(at, d=None):
        out = torch.empty(N, device=DEV)
        cstr.cstr_distill_loss(tables, at, q, ids, logp, out, dlogits=d, tail=tail)
        return out.double()
    d = torch.empty_like(x)
    size = loss(x, d).abs().max()
    way = torch.randn(x.shape, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    h = 2.0 ** -7
    slope = (loss(x + h * way) - loss(x - h * way)) / (2 * h)
    want = (d.double() * way.double()).sum(1)
    # third derivative of a log-sum (up to 4^3 along directions of size up to 4) times h^2 / 6, twice with a
    # lumped tail; the two losses' errors of log q (300 units of 2^-24) over 2 h
    assert ((slope - want).abs() <= 25 * h * h * (1 + want.abs()) + 2.0 ** -24 * (300 + size) * 2 / h).all()


def test_autograd_upstream_gradients_and_what_happens_in_between():
    N, k = 20, 12
    rng, x, tables, nexts, row_table, states = constrained(["api_1k", "api_1k"], 9, N, F32)
    allowed = allowed_rows(nexts, row_table, states, x.shape[1])
    ids, logp = records(rng, x, k, allowed)
    w, up = rng.random(N).astype(np.float32), rng.standard_normal(N).astype(np.float32)
    arrays = dict(teacher_ids=dev(ids), teacher_logp=dev(logp), states=dev(states), weight=dev(w), row_table=dev(row_table))
    for tail in TAILS:
        a = x.clone().requires_grad_()
        loss = constrained_distill_loss(a, tables=tables, tail=tail, temperature=0.8, **arrays)
        want = ref.distill(f8(x), allowed, ids, logp.astype(np.float64), tail, w.astype(np.float64) , float(np.float32(0.8)))
        kept = {n: t.clone() for n, t in arrays.items()}
        for n, t in arrays.items():                          # as a kernel writes them: autograd does not see it
            t.data.fill_(-1)
        loss.backward(dev(up))
        for n, t in arrays.items():
            t.data.copy_(kept[n])
        expect = want[1] * up[:, None].astype(np.float64)
        assert np.abs(f8(a.grad) - expect).max() <= 2.0 ** -24 * 1000 * np.abs(up).max() / 0.8
        assert np.abs(f8(loss) - want[0]).max() <= 2.0 ** -24 * 1000
    a = x.clone().requires_grad_()
    loss = constrained_distill_loss(a, tables=tables, **arrays)
    (g,) = torch.autograd.grad(loss.sum(), a, create_graph=True)
    with pytest.raises(RuntimeError, match="once only"):
        (g * a).sum().backward()
    assert constrained_distill_loss(x, tables=tables, **arrays).requires_grad is False


def test_records_of_the_student_itself_have_no_divergence():
    # records and loss together: top_logprobs of the same rows, with every way to treat the tail
    rng, x, tables, nexts, row_table, states = constrained(["json_32k"], 10, 30, F32)
    q = dev(states)
    ids, logp = top_logprobs(x, 50, tables, q, temperature=0.9)
    for tail in TAILS:
        a = x.clone().requires_grad_()
        loss = constrained_distill_loss(a, ids, logp, tables, q, tail=tail, temperature=0.9)
        loss.sum().backward()
        if tail == cstr.CSTR_TAIL_LUMP:
            # the record's own rounding (2^-24 of up to 30) enters once for every entry, log q's error besides
            assert loss.abs().max() <= 2.0 ** -24 * 400 and a.grad.abs().max() <= 2.0 ** -24 * 1000
        if tail == cstr.CSTR_TAIL_DROP:
            assert loss.abs().max() <= 2.0 ** -24 * 400


def test_streams_graphs_and_repeatability():
    N, V, k = 50, 33000, 64
    rng = np.random.default_rng(2)
    x = logits(2, N, V, BF)
    ids, logp = records(rng, x, k)
    side = torch.cuda.Stream()
    check_distill(x, ids, logp, cstr.CSTR_TAIL_LUMP, stream=side)
    i, t = dev(ids), dev(logp)
    loss = [torch.empty(N, device=DEV) for _ in range(2)]
    d = [torch.empty_like(x) for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cstr.cstr_distill_loss(None, x, None, i, t, loss[0], dlogits=d[0], tail=cstr.CSTR_TAIL_LUMP)
    for seed in (3, 4):
        x.copy_(logits(seed, N, V, BF))
        graph.replay()
        cstr.cstr_distill_loss(None, x, None, i, t, loss[1], dlogits=d[1], tail=cstr.CSTR_TAIL_LUMP)
        torch.cuda.synchronize()
        assert torch.equal(loss[0], loss[1]) and torch.equal(d[0], d[1])


def test_refusals_on_a_device():
    N, V, k = 6, 100, 4
    x = logits(1, N, V, F32)
    i, f, out = torch.zeros(N, k, dtype=torch.int32, device=DEV), torch.zeros(N, k, device=DEV), torch.zeros(N, device=DEV)
    vb, vo = config_vocab("api_1k")
    table = gpu_tables([config_dfas("api_1k")[0]], vb, vo)
    with pytest.raises(cstr.CstrError) as e:
        cstr.cstr_distill_loss(table, x, out.int(), i, f, out)
    assert e.value.code == -6
    for kw in (dict(teacher_ids=f), dict(teacher_logp=i), dict(teacher_ids=i[:, :3]), dict(teacher_logp=f[:3]),
               dict(loss_out=i[:, 0]), dict(loss_out=None), dict(weight=out[:2]), dict(weight=out.double()),
               dict(dlogits=x[:, :5]), dict(dlogits=x.bfloat16()), dict(states=out.int()), dict(row_table=out),
               dict(teacher_ids=i.T.contiguous().T), dict(logits=x.half()), dict(teacher_logp=f.cpu())):
        a = dict(dict(tables=None, logits=x, states=None, teacher_ids=i, teacher_logp=f, loss_out=out), **kw)
        with pytest.raises((TypeError, ValueError)):
            cstr.cstr_distill_loss(**a)
    for kw in (dict(tail=3), dict(tail=-1), dict(temperature=0.0), dict(temperature=math.nan)):
        with pytest.raises(cstr.CstrError) as e:
            cstr.cstr_distill_loss(None, x, None, i, f, out, **kw)
        assert e.value.code == -2
    cstr.cstr_distill_loss(None, x[:0], None, i[:0], f[:0], out[:0])


def test_longest_rows():
    # bitmaps of many words; more rows than CTAs of one row each could keep such bitmaps for
    rng = np.random.default_rng(16)
    x = logits(16, 1, 2000003, BF, offset=1)
    ids = np.stack([rng.choice(2000003, 700, replace=False)]).astype(np.int32)
    logp = np.log(rng.dirichlet(np.ones(701), 1)[:, :700]).astype(np.float32)
    check_distill(x, ids, logp, cstr.CSTR_TAIL_LUMP)
    N, V = 900, 600011
    x = torch.zeros(N, V, dtype=BF, device=DEV)
    loss = torch.empty(N, device=DEV)
    i = torch.randint(0, V, (N, 1), dtype=torch.int32, device=DEV)
    cstr.cstr_distill_loss(None, x, None, i, torch.zeros(N, 1, device=DEV), loss, tail=cstr.CSTR_TAIL_LUMP)
    # log V, from sums of 600,011 ones in 32 bits: exact but for the joins (16 of them) and the logarithm's rounding
    assert (loss - math.log(V)).abs().max() <= 2.0 ** -24 * (16 * 12 + 14)
