"""The operators over whole distributions where masks, rows and automata are not as even as the workloads'."""
import numpy as np
import pytest
import torch

import oracle
from oracle import distributions as ref
from paper_2407_08103_b200 import cstr
from synth.configs import config_dfas

from distribution_cases import BF, F32, allowed_rows, check_distill, check_sample, check_top, dev, logits, settings
from gpu_common import gpu_tables
from operator_cases import DEV, f8

pytestmark = pytest.mark.gpu


def odd_vocabulary(rng, V):
    """Strings of one to four printable bytes; the first 95 are the single bytes."""
    length = rng.integers(1, 5, V)
    text = rng.integers(32, 127, (V, 4)).astype(np.uint8)
    length[:95], text[:95, 0] = 1, np.arange(32, 127)
    return text[np.arange(4)[None, :] < length[:, None]], np.concatenate([[0], np.cumsum(length)]).astype(np.int64)


def random_dfa(rng, states):
    trans = rng.integers(0, states, (states, 256)).astype(np.int32)
    trans[rng.random((states, 256)) < np.where(np.arange(states) % 3 == 0, 0.9, 0.2)[:, None]] = -1
    return trans, (rng.random(states) < 0.4).astype(np.uint8), 0


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("V,ld,offset", [(1003, 1003, 0), (1003, 1031, 3), (4099, 4100, 1), (20011, 20011, 0), (20011, 20016, 5)])
def test_masks_under_rows_of_any_alignment(dtype, V, ld, offset):
    rng = np.random.default_rng(V + ld)
    vb, vo = odd_vocabulary(rng, V)
    dfas = [random_dfa(rng, 7), random_dfa(rng, 40)]
    tables = gpu_tables(dfas, vb, vo)
    nexts = [oracle.token_table(d[0], d[1], vb, vo)[0] for d in dfas]
    N = 14
    row_table = rng.integers(0, 2, N).astype(np.int32)
    states = np.array([rng.integers(0, nexts[t].shape[0]) for t in row_table], np.int32)
    x = logits(V, N, V, dtype, ld, offset)
    allowed = allowed_rows(nexts, row_table, states, V)
    kw = dict(allowed=allowed, tables=tables, states=states, row_table=row_table)
    u = rng.random(N).astype(np.float32)
    check_sample(x, u, nexts=nexts, **kw)
    check_sample(x, u, nexts=nexts, in_place=False, top_p=np.full(N, 0.97, np.float32), **kw)
    check_sample(x, u, nexts=nexts, **settings(rng, N), **kw)
    check_top(x, 100, **kw)
    ids, logp, _ = ref.top(f8(x) + 0.3 * rng.standard_normal((N, V)), allowed, 25)
    for tail in (cstr.CSTR_TAIL_RENORM, cstr.CSTR_TAIL_LUMP):
        check_distill(x, ids.astype(np.int32), logp.astype(np.float32), tail, shift=1, **kw)


def test_renumbered_automata_and_accepting_states():
    # hundreds of states that allow few bytes: the table numbers them in its own way
    rng = np.random.default_rng(3)
    vb, vo = odd_vocabulary(rng, 2050)
    dfa = config_dfas("schema40_128k")[0]
    (table,) = gpu_tables([dfa], vb, vo)
    nxt = oracle.token_table(dfa[0], dfa[1], vb, vo)[0]
    N = 400
    live = np.flatnonzero((nxt >= 0).any(1))
    states = rng.choice(live, N).astype(np.int32)
    x, u = logits(3, N, 2050, F32), rng.random(N).astype(np.float32)
    tokens, after, q = torch.empty(N, dtype=torch.int32, device=DEV), torch.empty(N, dtype=torch.int32, device=DEV), dev(states)
    accept = torch.full((N,), 9, dtype=torch.uint8, device=DEV)
    cstr.cstr_sample(table, x, q, tokens, dev(u), accept_out=accept, states_out=after)
    want = ref.sample(f8(x), nxt[states] >= 0, u)
    assert np.array_equal(tokens.cpu().numpy(), want[0])
    to = nxt[states, want[0]]
    assert np.array_equal(after.cpu().numpy(), to) and (to != states).any()
    assert np.array_equal(accept.cpu().numpy(), (np.asarray(dfa[1])[to] != 0).astype(np.uint8))


def test_states_that_allow_nothing_and_one_string():
    vb, vo = odd_vocabulary(np.random.default_rng(4), 500)
    trans = np.full((3, 256), -1, np.int32)
    trans[1, 65] = 2                                          # state 1 allows "A" alone, states 0 and 2 nothing
    tables = gpu_tables([(trans, np.array([0, 0, 1], np.uint8), 1)], vb, vo)
    nxt = oracle.token_table(trans, np.array([0, 0, 1], np.uint8), vb, vo)[0]
    states = np.array([0, 1, 2, 1], np.int32)
    x = logits(4, 4, 500, F32)
    allowed = allowed_rows([nxt], np.zeros(4, int), states, 500)
    kw = dict(tables=tables, states=states, allowed=allowed)
    u = np.array([0.1, 0.2, 0.3, 0.99], np.float32)
    for cuts in ({}, dict(top_p=np.full(4, 0.5, np.float32)), dict(top_k=np.full(4, 5, np.int32)), dict(min_p=np.full(4, 0.5, np.float32)),
                 dict(temperature=np.zeros(4, np.float32))):
        want = check_sample(x, u, nexts=[nxt], row_table=np.zeros(4, np.int32), **kw, **cuts)
        assert (want[0][[0, 2]] == -1).all()
        assert all(bytes(vb[vo[t]:vo[t + 1]]) == b"A" for t in want[0][[1, 3]])     # (some of the 500 tokens read so)
    check_top(x, 3, **kw)
    ids = np.array([[33, 5], [33, 5], [33, 33], [5, 6]], np.int32)      # "A" is the 34th single byte
    logp = np.log(np.array([[0.5, 0.5], [0.9, 0.1], [0.5, 0.5], [0.5, 0.5]])).astype(np.float32)
    for tail in (cstr.CSTR_TAIL_DROP, cstr.CSTR_TAIL_RENORM, cstr.CSTR_TAIL_LUMP):
        want = check_distill(x, ids, logp, tail, **kw)
        assert (want[0][[0, 2]] == 0).all()


@pytest.mark.parametrize("capture", [False, True])
def test_one_after_another_on_one_stream(capture):
    # a decoding loop of draws, each kernel set up beside its predecessor: states and tokens go from one to the next
    rng = np.random.default_rng(5)
    vb, vo = odd_vocabulary(rng, 3000)
    dfa = random_dfa(rng, 30)
    (table,) = gpu_tables([dfa], vb, vo)
    nxt = oracle.token_table(dfa[0], dfa[1], vb, vo)[0]
    N, steps = 9, 12
    xs = [logits(50 + i, N, 3000, BF) for i in range(steps)]
    us = rng.random((steps, N)).astype(np.float32)
    du, states, tokens = dev(us), torch.zeros(N, dtype=torch.int32, device=DEV), torch.empty(steps, N, dtype=torch.int32, device=DEV)
    p = torch.full((N,), 0.95, device=DEV)

    def loop():
        for i in range(steps):
            cstr.cstr_sample(table, xs[i], states, tokens[i], du[i], top_p=p)
    if capture:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            loop()
        states.zero_()
        graph.replay()
    else:
        loop()
    torch.cuda.synchronize()
    q = np.zeros(N, int)
    for i in range(steps):
        allowed = np.stack([nxt[s] >= 0 if s >= 0 else np.zeros(3000, bool) for s in q])
        want = ref.sample(f8(xs[i]), allowed, us[i], top_p=np.full(N, float(np.float32(0.95))))
        assert np.array_equal(tokens[i].cpu().numpy(), want[0]), i
        q = np.array([nxt[s, t] if t >= 0 else -1 for s, t in zip(q, want[0])])
    assert np.array_equal(states.cpu().numpy(), q)
