"""Inputs and comparisons shared by the tests of the operators over whole constrained distributions."""
import math

import numpy as np
import torch

import oracle
from oracle import distributions as ref
from paper_2407_08103_b200 import cstr
from synth.configs import config_dfas, config_vocab

from gpu_common import gpu_tables
from operator_cases import DEV, f8

BF, F32 = torch.bfloat16, torch.float32


def logits(seed, N, V, dtype, ld=None, offset=0, sigma=2.0, peaks=6):
    """Normal logits with a few likely tokens; any row stride and start."""
    g = torch.Generator().manual_seed(seed)
    ld = V if ld is None else ld
    x = torch.randn(N * ld + offset, generator=g).mul_(sigma)[offset:].as_strided((N, V), (ld, 1), 0).clone() \
        if N * ld else torch.zeros(N, V)
    for i in range(N):
        at = torch.randint(0, V, (peaks,), generator=g)
        x[i, at] += math.log(V) + torch.rand(1, generator=g) * 6 - torch.arange(peaks) * 0.7
    whole = torch.randn(N * ld + offset, generator=g).to(dtype).to(DEV)
    out = whole[offset:].as_strided((N, V), (ld, 1), offset)
    out.copy_(x)
    return out


def settings(rng, N, which="all"):
    """Random per-row settings, each off in some rows."""
    pick = lambda v, t: rng.choice(np.array(v, t), N).astype(t)  # noqa: E731
    s = dict(temperature=pick([0.0, 0.3, 0.7, 1.0, 1.7], np.float32), top_k=pick([-1, 0, 1, 2, 7, 40, 300], np.int32),
             top_p=pick([0.0, 0.3, 0.5, 0.9, 0.999, 1.0], np.float32), min_p=pick([0.0, 0.01, 0.2, 1.0, 1.5], np.float32))
    return s if which == "all" else {k: v for k, v in s.items() if k in which}


def constrained(names, seed, N, dtype, **kw):
    """Tables of the named workloads' automata over one vocabulary, random states, and what they allow."""
    dfas = [config_dfas(n)[0] for n in names]
    vb, vo = config_vocab(names[0])
    tables = gpu_tables(dfas, vb, vo)
    nexts = [oracle.token_table(d[0], d[1], vb, vo)[0] for d in dfas]
    rng = np.random.default_rng(seed)
    x = logits(seed, N, vo.size - 1, dtype, **kw)
    row_table = rng.integers(0, len(names), N).astype(np.int32)
    states = np.array([rng.integers(0, nexts[t].shape[0]) for t in row_table], np.int32)
    return rng, x, tables, nexts, row_table, states


def allowed_rows(nexts, row_table, states, V):
    """bool [N][V]; inactive rows allow nothing."""
    out = np.zeros((len(states), V), bool)
    for i, (t, q) in enumerate(zip(row_table, states)):
        if 0 <= t < len(nexts) and 0 <= q < nexts[t].shape[0]:
            out[i] = nexts[t][q] >= 0
    return out


def dev(a, dtype=None):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, dtype)).to(DEV)


def close(got, want, V):
    """log probabilities: exponentials with arguments up to |t| rounded three times (the mean |t| under
    the distribution is at most log2 V), 2^-22 of their own, 32 additions in 32 bits, and the result's rounding."""
    fine = np.isfinite(want)
    assert np.array_equal(np.isneginf(got), np.isneginf(want)) and np.array_equal(np.isfinite(got), fine)
    size = np.where(fine, np.abs(np.where(fine, want, 0.0)), 0.0)
    tol = 2.0 ** -24 * (2.1 * math.log2(V + 1) + 36.0 + size)
    err = np.abs(got[fine] - want[fine]) - tol[fine]
    assert (err <= 0).all(), "off by %g" % err.max()


def check_sample(x, uniform, allowed=None, tables=None, states=None, row_table=None, nexts=None, stream=None,
                 in_place=True, **cuts):
    """``x``: device logits; compares tokens, probabilities and states with the oracle."""
    N, V = x.shape
    allowed = np.ones((N, V), bool) if allowed is None else allowed
    tokens = torch.full((N,), -7, dtype=torch.int32, device=DEV)
    logp, kept = (torch.full((N,), math.nan, device=DEV) for _ in range(2))
    accept = torch.full((N,), 9, dtype=torch.uint8, device=DEV)
    d_states, d_uniform, d_rows = dev(states, np.int32), dev(uniform, np.float32), dev(row_table, np.int32)
    after = None if in_place or states is None else torch.full((N,), -7, dtype=torch.int32, device=DEV)
    d_cuts = {k: dev(v) for k, v in cuts.items()}
    torch.cuda.synchronize()
    cstr.cstr_sample(tables, x, d_states, tokens, d_uniform, logp_out=logp, kept_out=kept, row_table=d_rows,
                     accept_out=accept, states_out=after, stream=stream, **d_cuts)
    torch.cuda.synchronize()
    want = ref.sample(f8(x), allowed, uniform, **{k: np.asarray(v, np.float64 if v.dtype != np.int32 else np.int32)
                                                  for k, v in cuts.items()})
    got = tokens.cpu().numpy()
    assert np.array_equal(got, want[0]), "rows %s" % np.flatnonzero(got != want[0])[:8]
    close(f8(logp), want[1], V)
    rel = 2.0 ** -24 * (2.1 * math.log2(V + 1) + 38.0)
    assert (np.abs(f8(kept) - want[2]) <= rel * want[2]).all()
    if states is not None:
        t = np.zeros(N, int) if row_table is None else row_table
        q = np.array([nexts[t[i]][states[i], got[i]] if got[i] >= 0 else -1 for i in range(N)])
        assert np.array_equal((d_states if after is None else after).cpu().numpy(), q)
        if after is not None:
            assert np.array_equal(d_states.cpu().numpy(), states)
    return want


def check_top(x, n, allowed=None, temperature=1.0, lse=True, tables=None, states=None, row_table=None, stream=None):
    N, V = x.shape
    allowed = np.ones((N, V), bool) if allowed is None else allowed
    ids = torch.full((N, n), -7, dtype=torch.int32, device=DEV)
    logp = torch.full((N, n), math.nan, device=DEV)
    d_lse = torch.full((N,), math.nan, device=DEV) if lse else None
    d_states, d_rows = dev(states, np.int32), dev(row_table, np.int32)
    torch.cuda.synchronize()
    cstr.cstr_top_logprobs(tables, x, d_states, ids, logp, temperature=temperature, lse_out=d_lse, row_table=d_rows,
                           stream=stream)
    torch.cuda.synchronize()
    want = ref.top(f8(x), allowed, n, float(np.float32(temperature)))
    assert np.array_equal(ids.cpu().numpy(), want[0])
    close(f8(logp), want[1], V)
    if lse:
        top = f8(d_lse)
        fine = np.isfinite(want[2])
        assert np.array_equal(top[~fine], want[2][~fine])
        assert (np.abs(top[fine] - want[2][fine]) <= 2.0 ** -24 * (2.1 * math.log2(V + 1) + 36.0 + np.abs(want[2][fine]))).all()
    return want


def check_distill(x, ids, teacher, tail, allowed=None, weight=None, tables=None, states=None, row_table=None,
                  gradient=True, in_place=False, shift=0, stream=None, temperature=1.0):
    """``x``: device logits (any row stride); ``ids`` / ``teacher``: host arrays.  ``shift``: elements by which
    the gradient's rows begin later in their 16 bytes than the logits'."""
    N, V = x.shape
    allowed = np.ones((N, V), bool) if allowed is None else allowed
    host = f8(x)
    loss = torch.full((N,), math.nan, device=DEV)
    d, space = None, None
    if gradient:
        space = torch.full((max(N, 1) * x.stride(0) + 8,), 77.0, dtype=x.dtype, device=DEV)
        d = x if in_place else space.as_strided((N, V), x.stride(), (x.storage_offset() + shift) % 8)
    args = [dev(ids, np.int32), dev(teacher, np.float32), dev(weight, np.float32), dev(states, np.int32), dev(row_table, np.int32)]
    torch.cuda.synchronize()
    cstr.cstr_distill_loss(tables, x, args[3], args[0], args[1], loss, weight=args[2], dlogits=d, tail=tail,
                           temperature=temperature, row_table=args[4], stream=stream)
    torch.cuda.synchronize()
    given = np.asarray(teacher, np.float32).astype(np.float64)
    w = None if weight is None else np.asarray(weight, np.float32).astype(np.float64)
    tau = float(np.float32(temperature))
    want = ref.distill(host, allowed, ids, given, tail, w, tau)
    # log q: arguments rounded three times (their mean is at most log2 V), 2^-22 of an exponential, up to 128
    # additions of a thread (more where 16 CTAs of 256 have more than that in each of two sums) and 13 joins with two exponentials each; a lumped tail has two such sums
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        e_log = 2.0 ** -24 * (2.1 * math.log2(V + 1) + max(128, V / 8192) + 13 * 12)
        lw = np.ones(N) if w is None else np.abs(w)
        t = np.where((ids >= 0) & (ids < V), np.exp(given), 0.0)
        size = lw if tail == ref.RENORM else lw * (t.sum(1) + (1.0 if tail == ref.LUMP else 0.0))
        fine = np.isfinite(want[0])
        got = f8(loss)
        assert np.array_equal(np.isfinite(got), fine), (got, want[0])
        assert (np.abs(got - want[0])[fine] <= (3 * size * e_log + 2.0 ** -24 * np.abs(want[0]) + 1e-37)[fine]).all()
        if gradient:
            got = f8(d)
            fine = np.isfinite(want[1])
            assert np.array_equal(np.isfinite(got), fine)
            z = np.where(allowed, host / tau, -np.inf)
            q = np.exp(z - np.nanmax(z, 1, keepdims=True, initial=-1e300))
            q = np.nan_to_num(q / q.sum(1, keepdims=True))
            listed = np.zeros((N, V + 1))
            for i in range(N):
                np.add.at(listed[i], np.where((ids[i] >= 0) & (ids[i] < V), ids[i], V), t[i] if tail != ref.RENORM else 1.0)
            listed = np.minimum(listed[:, :V], np.maximum(size / np.maximum(lw, 1e-300), 1.0)[:, None])
            others = np.where(listed > 0, 0.0, q)
            others = others / np.maximum(others.sum(1, keepdims=True), 1e-300) if tail == ref.LUMP else 0.0 * q
            mine = size[:, None] * (q + others) + lw[:, None] * listed
            far = 2.0 ** -24 * 2.1 * np.maximum(0.0, -np.log2(np.maximum(np.maximum(q, others), 1e-300)))
            unit = {F32: 2.0 ** -24, BF: 2.0 ** -8}[x.dtype]
            tol = unit * np.abs(want[1]) + mine * (3 * e_log + far) / tau + 1e-37
            err = (np.abs(got - want[1]) - tol)[fine]
            assert (err <= 0).all(), "gradient off by %g" % err.max()
            assert (got[~allowed & fine] == 0).all()
            if not in_place:
                outside = torch.ones_like(space, dtype=torch.bool)
                outside.as_strided((N, V), x.stride(), d.storage_offset()).fill_(False)
                assert (space[outside] == 77.0).all()
    return want
