"""Constrained policy loss and its gradient against the oracle's statement in 64 bits."""
import math

import numpy as np
import pytest
import torch

import oracle
from paper_2407_08103_b200 import cstr
from synth.configs import config_dfas, config_vocab

from gpu_common import gpu_tables
from operator_cases import DEV, check_loss, f8

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def inputs(seed, N, V, dtype, ld=None, sigma=2.0, offset=0):
    rng = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed)
    ld = V if ld is None else ld
    x = torch.randn(N * ld + offset, generator=g).mul_(sigma).to(dtype).to(DEV)[offset:].as_strided(
        (N, V), (ld, 1), offset)
    adv = rng.standard_normal(N).astype(np.float32)
    return rng, x, adv


def old_from(x, allowed, actions, rng, spread=0.3, temperature=1.0):
    from oracle import operators as ref
    lp = ref.policy_loss(f8(x), allowed, actions, np.zeros(len(actions)), np.ones(len(actions)),
                         temperature=temperature)[1]
    lp = np.where(np.isfinite(lp), lp, -3.0)
    return (lp + rng.standard_normal(len(actions)) * spread).astype(np.float32)


@pytest.mark.parametrize("N,V", [(1, 1), (3, 2), (5, 31), (4, 32), (7, 33), (2, 1000), (3, 1024), (2, 8191),
                                 (2, 8200), (3, 32000), (2, 40001), (1, 128256), (1, 300007)])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_unconstrained_shapes(N, V, dtype):
    rng, x, adv = inputs(N * V, N, V, dtype)
    act = rng.integers(0, V, N)
    ok = np.ones((N, V), bool)
    old = old_from(x, ok, act, rng)
    check_loss(x, ok, act, old, adv, ref_logp=old + 0.1, weight=rng.random(N).astype(np.float32), kl_coef=0.1)
    check_loss(x, ok, act, old, adv, gradient=False, clip_low=0.1, clip_high=0.3)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("ld,offset", [(1024, 0), (1031, 0), (1040, 3), (1024, 1), (1008, 8)])
def test_row_strides_and_alignment(dtype, ld, offset):
    V = 1003
    rng, x, adv = inputs(ld + offset, 6, V, dtype, ld, offset=offset)
    act = rng.integers(0, V, 6)
    ok = np.ones((6, V), bool)
    old = old_from(x, ok, act, rng)
    check_loss(x, ok, act, old, adv)
    before = x.clone()
    whole = x.as_strided((6 * ld - (ld - V),), (1,))
    pad = whole.clone()
    check_loss(x, ok, act, old, adv, in_place=True)
    assert not torch.equal(x, before)
    mask = torch.ones(whole.numel(), dtype=torch.bool, device=DEV)
    mask.as_strided((6, V), (ld, 1)).fill_(False)
    assert torch.equal(whole[mask], pad[mask])             # columns past V untouched


def constrained(names, seed, N, dtype):
    """Tables of the named workloads' automata over one vocabulary, random states and actions."""
    dfas = [config_dfas(n)[0] for n in names]
    vb, vo = config_vocab(names[0])
    V = vo.size - 1
    tables = gpu_tables(dfas, vb, vo)
    masks = [oracle.token_table(d[0], d[1], vb, vo)[0] >= 0 for d in dfas]
    rng, x, adv = inputs(seed, N, V, dtype)
    row_table = rng.integers(0, len(names), N).astype(np.int32)
    states = np.array([rng.integers(0, masks[t].shape[0]) for t in row_table], np.int32)
    allowed = np.stack([masks[t][q] for t, q in zip(row_table, states)])
    act = np.array([rng.choice(np.flatnonzero(a)) if a.any() else 0 for a in allowed], np.int32)
    return rng, x, adv, tables, masks, row_table, states, allowed, act


@pytest.mark.parametrize("dtype", [F32, BF])
def test_constrained_mixed_tables_and_invalid_rows(dtype):
    rng, x, adv, tables, masks, row_table, states, allowed, act = constrained(
        ["api_1k", "json_32k"][:1] + ["json_32k"], 3, 40, dtype)
    states[3], states[4], states[5] = -1, 10 ** 6, -7
    row_table[6], row_table[7] = 2, -1
    act[8], act[9] = -1, x.shape[1]
    act[10] = int(np.flatnonzero(~allowed[10])[0])          # a token that the state does not allow
    for i in (3, 4, 5, 6, 7):
        allowed[i] = False
    old = old_from(x, allowed, act, rng)
    kw = dict(tables=tables, states=states, row_table=row_table, ref_logp=old - 0.2, kl_coef=0.2,
              weight=rng.random(40).astype(np.float32), temperature=0.8)
    want = check_loss(x, allowed, act, old, adv, **kw)
    assert np.isneginf(want[1][3:11]).all() and (want[2][3:11] == 0).all()
    check_loss(x, allowed, act, old, adv, in_place=True, **kw)


def test_constrained_large_vocabulary_workload():
    rng, x, adv, tables, _, _, states, allowed, act = constrained(["json_32k"], 4, 24, BF)
    old = old_from(x, allowed, act, rng)
    check_loss(x, allowed, act, old, adv, tables=tables, states=states)


def test_clipping_sides_and_boundaries():
    N, V = 8, 64
    rng, x, _ = inputs(5, N, V, F32)
    ok, act = np.ones((N, V), bool), rng.integers(0, V, N)
    lp = old_from(x, ok, act, rng, spread=0.0)
    shift = np.array([-1, -1, 1, 1, 0, 0, -0.1, 0.1], np.float32)     # ratio e^-shift
    adv = np.array([1, -1, 1, -1, 1, -1, 2, 2], np.float32)
    want = check_loss(x, ok, act, lp + shift, adv)
    moved = np.abs(want[2]).max(1) > 0
    assert moved.tolist() == [False, True, True, False, True, True, True, True]


def test_nonfinite_logits():
    N, V = 8, 2000
    rng, x, adv = inputs(6, N, V, F32)
    adv = np.abs(adv) + 0.5
    ok, act = np.ones((N, V), bool), rng.integers(10, V, N)
    old = np.full(N, -8.0, np.float32)
    x[0, 1] = math.nan
    x[1] = -math.inf                                       # no mass at all
    x[2, int(act[2])] = -math.inf
    x[3, :] = torch.finfo(F32).min                         # uniform over the lowest values
    x[4, 5] = math.inf
    x[5, 7] = -math.inf
    x[6] = math.nan
    weight = np.ones(N, np.float32)
    weight[6] = 0.0                                        # padding: nothing comes of its NaN
    want = check_loss(x, ok, act, old, adv, weight=weight)
    assert np.isnan(want[0][[0, 4]]).all() and want[0][6] == 0 and abs(want[1][3] + math.log(V)) < 1e-9


def test_disallowed_nan_does_not_matter():
    rng, x, adv, tables, _, _, states, allowed, act = constrained(["api_1k"], 7, 16, F32)
    old = old_from(x, allowed, act, rng)
    x[torch.from_numpy(~allowed).to(DEV)] = math.nan
    check_loss(x, allowed, act, old, adv, tables=tables, states=states)


def test_gradient_agrees_with_differences_of_the_loss():
    rng, x, adv, tables, _, _, states, allowed, act = constrained(["api_1k"], 8, 32, F32)
    old = old_from(x, allowed, act, rng)
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    dev = dict(states=t(states), actions=t(act), old_logp=t(old), advantages=t(adv))
    kw = dict(ref_logp=t(old + 0.1), kl_coef=0.3, clip_low=5.0, clip_high=5.0)       # smooth: never clipped

    def loss(at, d=None):
        out, lp = torch.empty(32, device=DEV), torch.empty(32, device=DEV)
        cstr.cstr_policy_loss(tables, at, dev["states"], dev["actions"], dev["old_logp"], dev["advantages"],
                              out, lp, dlogits=d, **kw)
        return out.double()
    d = torch.empty_like(x)
    loss(x, d)
    g = torch.Generator(device=DEV).manual_seed(1)
    way = torch.randn(x.shape, generator=g, device=DEV)
    h = 2.0 ** -7
    slope = (loss(x + h * way) - loss(x - h * way)) / (2 * h)
    want = (d.double() * way.double()).sum(1)
    # third derivative times h^2 / 6 (directions of size up to 4 among few allowed tokens), 32-bit loss / h
    assert ((slope - want).abs() <= 60 * h * h * (1 + want.abs()) + 2.0 ** -18 / h).all()


def test_side_stream_repeatability_empty_batch_and_refusals():
    rng, x, adv = inputs(9, 50, 33000, BF)
    act, ok = rng.integers(0, 33000, 50), np.ones((50, 33000), bool)
    old = old_from(x, ok, act, rng)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    check_loss(x, ok, act, old, adv, stream=side)
    t = lambda a, dt=F32: torch.as_tensor(np.asarray(a)).to(dt).to(DEV)  # noqa: E731
    a = dict(actions=t(act, torch.int32), old_logp=t(old), advantages=t(adv), loss_out=torch.empty(50, device=DEV),
             logp_out=torch.empty(50, device=DEV))
    got = []
    for _ in range(2):
        d = torch.empty_like(x)
        cstr.cstr_policy_loss(None, x, None, *a.values(), dlogits=d)
        got.append((a["loss_out"].clone(), d))
    torch.cuda.synchronize()
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    cstr.cstr_policy_loss(None, x[:0], None, *[v[:0] for v in a.values()])
    for kw in (dict(dlogits=torch.empty(50, 33000, device=DEV)), dict(dlogits=x[:, :5]), dict(states=a["actions"]),
               dict(actions=a["old_logp"]), dict(weight=a["old_logp"][:9]), dict(ref_logp=a["old_logp"].cpu())):
        b = dict(a, states=None)
        b.update({k: v for k, v in kw.items() if k in b})
        more = {k: v for k, v in kw.items() if k not in b}
        with pytest.raises((TypeError, ValueError)):
            cstr.cstr_policy_loss(None, x, b.pop("states"), *b.values(), **more)
    with pytest.raises(TypeError):
        cstr.cstr_policy_loss(None, x.half(), None, *a.values())
    for kw in (dict(temperature=0.0), dict(temperature=math.inf), dict(clip_low=-0.1), dict(kl_coef=math.nan)):
        with pytest.raises(cstr.CstrError) as e:
            cstr.cstr_policy_loss(None, x, None, *a.values(), **kw)
        assert e.value.code == -2
    vb, vo = config_vocab("api_1k")
    table = gpu_tables([config_dfas("api_1k")[0]], vb, vo)
    with pytest.raises(cstr.CstrError) as e:               # another vocabulary's table
        cstr.cstr_policy_loss(table, x, a["actions"], *a.values())
    assert e.value.code == -6
