"""Sampling under cuts and the most likely tokens against the oracle's statement in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2407_08103_b200 import cstr
from synth.configs import config_dfas, config_vocab

from distribution_cases import BF, F32, allowed_rows, check_sample, check_top, constrained, dev, logits, settings
from gpu_common import gpu_tables
from operator_cases import DEV, f8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,V", [(1, 1), (3, 2), (40, 31), (30, 33), (30, 1000), (30, 1024), (20, 2051), (12, 8200),
                                 (8, 40001), (3, 128256), (2, 300007)])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_sample_shapes(N, V, dtype):
    rng = np.random.default_rng(N * V)
    x = logits(N * V, N, V, dtype)
    check_sample(x, rng.random(N).astype(np.float32), **settings(rng, N))
    check_sample(x, rng.random(N).astype(np.float32))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("which", [("top_k",), ("top_p",), ("min_p",), ("temperature",), ("top_k", "top_p"),
                                   ("temperature", "top_p", "min_p")])
def test_each_cut_alone_and_in_pairs(dtype, which):
    rng = np.random.default_rng(len(which[0]) + len(which))
    for V in (700, 5003):
        x = logits(V, 24, V, dtype)
        check_sample(x, rng.random(24).astype(np.float32), **settings(rng, 24, which))


@pytest.mark.parametrize("dtype", [F32, BF])
def test_long_prefixes(dtype):
    # nearly flat rows: nuclei of thousands of tokens, top_k above what one record holds
    rng = np.random.default_rng(11)
    N, V = 10, 20011
    x = logits(11, N, V, dtype, sigma=0.5, peaks=1)
    pick = lambda v, t: rng.choice(np.array(v, t), N)  # noqa: E731
    check_sample(x, rng.random(N).astype(np.float32), top_p=pick([0.5, 0.9, 0.99], np.float32))
    check_sample(x, rng.random(N).astype(np.float32), top_k=pick([2000, 5000, 20010, 20011, 30000], np.int32))
    check_sample(x, rng.random(N).astype(np.float32), min_p=pick([1e-6, 1e-3, 0.02], np.float32))
    check_sample(x, rng.random(N).astype(np.float32), top_k=pick([3000, 15000], np.int32),
                 top_p=pick([0.8, 0.95], np.float32), min_p=pick([0.0, 1e-4], np.float32))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("ld,offset", [(1024, 0), (1031, 0), (1040, 3), (1024, 1), (1008, 8)])
def test_row_strides_and_alignment(dtype, ld, offset):
    rng = np.random.default_rng(ld + offset)
    x = logits(ld + offset, 12, 1003, dtype, ld, offset)
    check_sample(x, rng.random(12).astype(np.float32), **settings(rng, 12))
    check_sample(x, rng.random(12).astype(np.float32))
    check_top(x, 37)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("value", [0.0, -0.0, 3.5, -1e30, 1e30])
def test_equal_logits_go_by_id(dtype, value):
    N, V = 24, 3001
    rng = np.random.default_rng(5)
    x = torch.full((N, V), value, dtype=dtype, device=DEV)
    x[1, ::2] = -0.0 if value == 0.0 else value
    u = rng.random(N).astype(np.float32)
    u[:4] = [0.0, 0.5, 0.25, 1.0 - 2.0 ** -24]
    check_sample(x, u)
    check_sample(x, u, top_k=rng.integers(1, V + 5, N).astype(np.int32))
    check_sample(x, u, top_p=np.where(np.arange(N) % 2 == 0, np.float32(0.5), rng.random(N).astype(np.float32)))
    check_sample(x, u, min_p=np.full(N, 1.0, np.float32), top_p=np.full(N, 0.25, np.float32))
    check_top(x, 1000)
    # two values, in blocks and alternating
    x[:, 1::3] = 1.0
    check_sample(x, u, top_k=rng.integers(900, 1200, N).astype(np.int32))
    check_top(x, 1024)


def test_borders_of_uniform_numbers_and_settings():
    x = torch.tensor([[0.0, 0.0, 0.0, 0.0]], device=DEV).expand(12, 4).contiguous()
    u = np.array([0.0, 0.25, 0.5, 0.75, 1.0 - 2.0 ** -24, 1.0, 2.0, -3.0, math.inf, -math.inf, math.nan, 0.2499999], np.float32)
    want = check_sample(x, u)
    assert want[0].tolist() == [0, 1, 2, 3, 3, 3, 3, 0, 3, 0, -1, 0]
    # the shortest prefix that holds 0.5 of four equal tokens is two of them
    want = check_sample(x, u, top_p=np.full(12, 0.5, np.float32))
    assert want[0].tolist() == [0, 0, 1, 1, 1, 1, 1, 0, 1, 0, -1, 0]
    bad = np.array([math.nan, -1.0, math.inf, 1e-39, -math.inf, 0.0, -0.0, 1e-30, 1e30, 4.4e-39, 1.0, 1.0], np.float32)
    want = check_sample(x, np.full(12, 0.6, np.float32), temperature=bad)
    assert want[0].tolist() == [-1] * 5 + [0, 0, 2, 2, 2, 2, 2]
    odd = np.array([math.nan, -1.0, math.inf, 0.0, 1e-40, 1.0, -0.0, 2.0, 0.3, 0.3, 0.3, -math.inf], np.float32)
    check_sample(x, np.full(12, 0.6, np.float32), top_p=odd)
    check_sample(x, np.full(12, 0.6, np.float32), min_p=odd)
    check_sample(x, np.full(12, 0.6, np.float32), top_k=np.array([-2 ** 31, -1, 0, 1, 2, 3, 4, 5, 2 ** 31 - 1, 1, 2, 3], np.int32))


@pytest.mark.parametrize("dtype", [F32, BF])
def test_nonfinite_logits(dtype):
    N, V = 10, 2500
    rng = np.random.default_rng(6)
    x = logits(6, N, V, dtype)
    x[0, ::3] = math.nan
    x[1] = -math.inf
    x[2] = math.nan
    x[3, 5:] = -math.inf
    x[4, 100] = x[4, 2300] = math.inf
    x[5] = math.nan
    x[5, 77] = -math.inf
    x[6] = torch.finfo(dtype).min
    x[7] = torch.finfo(dtype).max
    x[8, 9] = torch.finfo(dtype).max
    u = rng.random(N).astype(np.float32)
    want = check_sample(x, u)
    assert want[0][1] == 0 and want[0][2] == -1 and want[0][5] == 77 and want[0][4] in (100, 2300)
    for _ in range(3):
        check_sample(x, u, **settings(rng, N))
    check_top(x, 12)
    check_top(x, 1024)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("names", [("api_1k",), ("json_32k", "json_32k")])
def test_constrained_rows(dtype, names):
    N = 40
    rng, x, tables, nexts, row_table, states = constrained(list(names), 3, N, dtype)
    states[3], states[4], states[5] = -1, 10 ** 6, -7
    row_table[6], row_table[7] = len(names), -1
    allowed = allowed_rows(nexts, row_table, states, x.shape[1])
    x[torch.from_numpy(~allowed).to(DEV)] = math.nan                # what is not allowed does not matter
    kw = dict(allowed=allowed, tables=tables, states=states, row_table=row_table)
    for _ in range(2):
        u = rng.random(N).astype(np.float32)
        want = check_sample(x, u, nexts=nexts, in_place=False, **kw)
        assert (want[0][3:8] == -1).all()
        check_sample(x, u, nexts=nexts, **kw, **settings(rng, N))
    for n in (1, 20, 500):
        check_top(x, n, **kw)
    check_top(x, 8, temperature=0.6, lse=False, **kw)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("N,V,n", [(1, 1, 1), (3, 2, 5), (5, 33, 33), (20, 1024, 5), (6, 1500, 1024), (4, 8200, 64),
                                   (4, 20011, 1000), (2, 128256, 256), (2, 300007, 20)])
def test_top_shapes(N, V, n, dtype):
    x = logits(N + V + n, N, V, dtype)
    check_top(x, n)
    check_top(x, n, temperature=2.5)


def test_log_probability_is_that_of_the_policy_loss():
    N = 64
    rng, x, tables, nexts, row_table, states = constrained(["json_32k"], 9, N, F32)
    t = {k: torch.empty(N, device=DEV) for k in ("logp", "loss", "again")}
    tokens, after = (torch.empty(N, dtype=torch.int32, device=DEV) for _ in range(2))
    q = dev(states)
    cstr.cstr_sample(tables, x, q, tokens, dev(rng.random(N), np.float32), temperature=torch.full((N,), 0.8, device=DEV),
                     logp_out=t["logp"], states_out=after)
    cstr.cstr_policy_loss(tables, x, q, tokens, t["logp"], torch.ones(N, device=DEV), t["loss"], t["again"],
                          temperature=0.8)
    # two roundings of the same sums (up to 2^-24 of what close() in distribution_cases counts, each)
    fine = torch.isfinite(t["logp"])
    assert torch.equal(fine, torch.isfinite(t["again"]))       # (some states allow nothing)
    assert (t["logp"] - t["again"])[fine].abs().max() <= 2 * 2.0 ** -24 * (2.1 * 15 + 36 + 30)
    assert torch.equal(tokens >= 0, fine)


def test_streams_graphs_and_repeatability():
    N, V = 70, 33000
    rng = np.random.default_rng(2)
    x = logits(2, N, V, BF)
    side = torch.cuda.Stream()
    u, cuts = rng.random(N).astype(np.float32), settings(rng, N)
    check_sample(x, u, stream=side, **cuts)
    check_top(x, 50, stream=side)
    d = {k: dev(v) for k, v in cuts.items()}
    du = dev(u)
    out = torch.empty(3, N, dtype=torch.int32, device=DEV)
    graph = torch.cuda.CUDAGraph()
    ids, logp = torch.empty(N, 9, dtype=torch.int32, device=DEV), torch.empty(N, 9, device=DEV)
    with torch.cuda.graph(graph):
        cstr.cstr_sample(None, x, None, out[0], du, **d)
        cstr.cstr_sample(None, x, None, out[1], du)
        cstr.cstr_top_logprobs(None, x, None, ids, logp)
    for seed in (3, 4):
        x.copy_(logits(seed, N, V, BF))
        du.copy_(torch.rand(N, device=DEV))
        graph.replay()
        cstr.cstr_sample(None, x, None, out[2], du, **d)
        torch.cuda.synchronize()
        assert torch.equal(out[0], out[2])
        cstr.cstr_sample(None, x, None, out[2], du)
        assert torch.equal(out[1], out[2])
        assert torch.equal(ids[:, 0].long(), x.float().argmax(1))
        check_sample(x, du.cpu().numpy(), **cuts)


def test_a_whole_batch_as_drawn():
    # thousands of rows: frequencies of the tokens agree with their probabilities
    N, V = 4096, 50
    x = logits(8, 1, V, F32).expand(N, V).contiguous()
    u = (torch.arange(N, device=DEV) + 0.5) / N
    tokens = torch.empty(N, dtype=torch.int32, device=DEV)
    cstr.cstr_sample(None, x, None, tokens, u)
    p = torch.softmax(x[0].double(), 0)
    share = torch.bincount(tokens.long(), minlength=V).double() / N
    assert (share - p).abs().max() <= 1.0 / N + 1e-6           # a token's interval holds that many of the steps


def test_refusals_on_a_device():
    N, V = 6, 100
    x = logits(1, N, V, F32)
    i, f = torch.zeros(N, dtype=torch.int32, device=DEV), torch.zeros(N, device=DEV)
    vb, vo = config_vocab("api_1k")
    table = gpu_tables([config_dfas("api_1k")[0]], vb, vo)
    with pytest.raises(cstr.CstrError) as e:                  # another vocabulary's table
        cstr.cstr_sample(table, x, i, i.clone(), f)
    assert e.value.code == -6
    for kw in (dict(tokens_out=f), dict(uniform=i), dict(uniform=f[:3]), dict(temperature=f.double()), dict(top_k=f),
               dict(top_p=i), dict(min_p=f.cpu()), dict(states=i), dict(states_out=i), dict(logp_out=i),
               dict(kept_out=f[::2]), dict(accept_out=i), dict(uniform=None), dict(tokens_out=None)):
        a = dict(dict(tables=None, logits=x, states=None, tokens_out=i, uniform=f), **kw)
        with pytest.raises((TypeError, ValueError)):
            cstr.cstr_sample(**a)
    for ids, logp in ((f, f), (torch.zeros(N, 5, dtype=torch.int32, device=DEV), torch.zeros(N, 4, device=DEV)),
                      (torch.zeros(N, 5, device=DEV), torch.zeros(N, 5, device=DEV)),
                      (torch.zeros(5, N, dtype=torch.int32, device=DEV).T, torch.zeros(N, 5, device=DEV))):
        with pytest.raises((TypeError, ValueError)):
            cstr.cstr_top_logprobs(None, x, None, ids, logp)
    with pytest.raises(cstr.CstrError) as e:
        cstr.cstr_top_logprobs(None, x, None, torch.zeros(N, 1025, dtype=torch.int32, device=DEV), torch.zeros(N, 1025, device=DEV))
    assert e.value.code == -2
    cstr.cstr_sample(None, x[:0], None, i[:0], f[:0])


@pytest.mark.parametrize("dtype", [F32, BF])
def test_lists_that_overflow_or_hold_everything(dtype):
    # candidates around the 2,048 that a list holds, by every way that leads there
    N, V = 6, 9001
    rng = np.random.default_rng(12)
    x = logits(12, N, V, dtype, sigma=0.3, peaks=2)
    u = rng.random(N).astype(np.float32)
    x[0] = x[0].round()                                      # few values, thousands of each
    check_sample(x, u, top_k=np.array([2047, 2048, 2049, 2048, 1500, 4096], np.int32))
    check_sample(x, u, top_k=np.array([50, 600, 700, 8999, 9000, 9001], np.int32), top_p=np.full(N, 0.7, np.float32))
    check_sample(x, u, min_p=np.array([1e-3, 1e-2, 0.5, 0.02, 1e-5, 1e-30], np.float32), top_k=np.full(N, 1200, np.int32))
    check_sample(x, u, top_p=np.array([0.1, 0.2, 0.25, 0.3, 0.5, 0.05], np.float32))
    check_top(x, 1024)
    x[1, ::2] = 40.0                                         # 4,501 equal ones at the top
    check_top(x, 1024)
    check_sample(x, u, top_k=np.full(N, 100, np.int32))
    check_sample(x, u, top_p=np.full(N, 0.01, np.float32))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("level,spread", [(-3e38, 0.0), (1e12, 1e6), (-1e12, 1e6), (1e38, 1e37), (1e-30, 1e-31), (5e10, 1.0)])
def test_logits_of_any_size(dtype, level, spread):
    # a common offset that floats resolve coarsely, masks of -infinity beside the lowest values, any temperature
    N, V = 12, 3000
    rng = np.random.default_rng(13)
    x = (level + spread * torch.from_numpy(rng.standard_normal((N, V)))).to(dtype).to(DEV)
    x[:, ::5] = -math.inf
    x[1, 1:] = -math.inf
    x[2, 7] = torch.finfo(dtype).min
    temperature = np.array([1.0, 1.0, 1e6, 1e12, 1e37, 3e38, 1e30, 0.5, 1e-30, 2e5, 7.0, 1e33], np.float32)
    u = rng.random(N).astype(np.float32)
    check_sample(x, u, temperature=temperature)
    check_sample(x, u, temperature=temperature, top_p=np.full(N, 0.6, np.float32))
    check_sample(x, u, temperature=temperature, top_k=np.full(N, 60, np.int32), min_p=np.full(N, 0.3, np.float32))
    check_top(x, 30)
    check_top(x, 30, temperature=1e20)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("step", [0.0, 0.02, 0.5, 3.0])
def test_wide_nuclei_with_many_equal_logits(dtype, step):
    # borders of top_p among thousands of tokens, alone or equal in thousands; odd row length, masked tokens
    N, V = 5, 70001
    rng = np.random.default_rng(14)
    x = logits(14, N, V, F32, sigma=1.0, peaks=3)
    x = (x if step == 0.0 else (x / step).round() * step).to(dtype)
    x[:, 5::11] = -math.inf
    x[0, 9::7] = math.nan
    u = rng.random(N).astype(np.float32)
    check_sample(x, u, top_p=np.array([0.99, 0.9, 0.5, 0.7, 0.999999], np.float32))
    check_sample(x, u, top_p=np.array([0.99, 0.9, 0.5, 0.7, 0.8], np.float32), top_k=np.array([5000, 20000, 60000, 3000, 2049], np.int32),
                 temperature=np.array([1.0, 0.5, 2.0, 30.0, 0.9], np.float32))
    check_sample(x, u, top_p=np.full(N, 0.97, np.float32), min_p=np.array([1e-4, 1e-6, 1e-3, 3e-3, 0.0], np.float32),
                 temperature=np.array([1.0, 2.0, 1.5, 1.0, 50.0], np.float32))


def test_longest_rows():
    # shares of many blocks, counts and masses over millions of tokens; a row that begins inside a vector
    rng = np.random.default_rng(15)
    x = logits(15, 2, 2000003, BF, offset=3)
    u = rng.random(2).astype(np.float32)
    check_sample(x, u)
    check_sample(x, u, top_p=np.array([0.4, 0.9], np.float32), top_k=np.array([0, 100], np.int32))
    top = torch.empty(2, 40, dtype=torch.int32, device=DEV), torch.empty(2, 40, device=DEV)
    cstr.cstr_top_logprobs(None, x, None, *top)
    assert torch.equal(top[0][:, 0].long(), x.float().argmax(1))
    longest = torch.zeros(1, 8388608, device=DEV)
    longest[0, 8388607] = 3.0
    for uniform, want in ((0.0, 0), (0.5, 4194313), (1.0, 8388607)):
        token = torch.empty(1, dtype=torch.int32, device=DEV)
        cstr.cstr_sample(None, longest, None, token, torch.tensor([uniform], device=DEV))
        # half of V - 1 + e^3 lies 9.04 tokens behind the middle
        assert token.item() == want


def test_two_threads_call_at_once():
    # rows of different lengths need different amounts of shared memory and clusters
    import threading
    cases = [(logits(i, 8, V, F32), torch.rand(8, device=DEV)) for i, V in enumerate((700, 300007, 40001, 128256))]
    want = []
    for x, u in cases:
        out = torch.empty(8, dtype=torch.int32, device=DEV)
        cstr.cstr_sample(None, x, None, out, u, top_p=torch.full((8,), 0.9, device=DEV))
        want.append(out)
    torch.cuda.synchronize()
    bad = []

    def work(k):
        stream = torch.cuda.Stream()
        p = torch.full((8,), 0.9, device=DEV)
        torch.cuda.synchronize()
        for i in range(40):
            x, u = cases[(i + k) % 4]
            out = torch.empty(8, dtype=torch.int32, device=DEV)
            stream.wait_stream(torch.cuda.current_stream())
            cstr.cstr_sample(None, x, None, out, u, top_p=p, stream=stream)
            stream.synchronize()
            if not torch.equal(out, want[(i + k) % 4]):
                bad.append((k, i))
    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad
