"""Attention over a shared prompt and per-row caches, and insertion with eviction, against the
oracle's statements in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2407_08103_b200 import cstr

from operator_cases import DEV, AttentionCase, check_insert, f8, random_cache, ranked_ages

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


@pytest.mark.parametrize("B,T,Hq,Hk,D,P,cap", [
    (1, 1, 1, 1, 8, 0, 1), (1, 1, 1, 1, 8, 1, 1), (3, 1, 4, 2, 64, 17, 5), (2, 1, 8, 8, 128, 100, 33),
    (5, 2, 6, 2, 80, 31, 40), (2, 3, 7, 1, 96, 129, 19), (3, 5, 8, 2, 128, 15, 70), (1, 9, 21, 3, 40, 64, 64),
    (2, 4, 64, 2, 64, 0, 50), (1, 1, 128, 1, 128, 200, 10), (4, 1, 2, 2, 72, 16, 1000), (1, 17, 3, 1, 16, 5, 300),
])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_attention_shapes(B, T, Hq, Hk, D, P, cap, dtype):
    for causal in (False, True):
        if causal and cap < T:
            continue
        c = AttentionCase(B * 1000 + P, B, T, Hq, Hk, D, P, cap, dtype, causal=causal,
                          n_query=np.random.default_rng(1).integers(0, T + 1, B) if causal else None)
        c.run()
        c.check()


@pytest.mark.parametrize("layout,pad", [("heads", 0), ("slots", 8), ("heads", 24)])
def test_attention_strides(layout, pad):
    c = AttentionCase(7, 3, 2, 8, 2, 64, 37, 45, BF, causal=True, layout=layout, pad=pad)
    c.run()
    c.check()


def test_attention_output_strides_and_unwritten_padding():
    c = AttentionCase(8, 3, 2, 4, 2, 40, 20, 30, BF)
    whole = torch.full((3, 2, 4, 48), 7.0, dtype=BF, device=DEV)
    c.out = whole[..., :40]
    c.run()
    c.check()
    assert (whole[..., 40:] == 7.0).all()


def test_attention_of_rows_that_see_nothing():
    c = AttentionCase(9, 4, 3, 4, 2, 64, 0, 20, BF, causal=True, lens=[0, 20, 5, 3], n_query=[3, 0, 2, 3])
    c.lens = np.array([0, 20, 5, 3])
    c.pos = np.array([0, 17, -100, 0], np.int32)          # row 2: every slot lies in its future
    c.dev()
    c.run()
    r = c.check()
    assert np.isneginf(r["lse"][2]).all() and (f8(c.out)[[0, 1, 2]] == 0).all()


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_attention_nonfinite_values_reach_only_the_tokens_that_see_them(value, dtype):
    c = AttentionCase(10, 2, 4, 8, 2, 64, 33, 40, dtype, causal=True, lens=[40, 21])
    for b in range(2):                                     # the last token's key and value rows
        for h in range(2):
            j = int(np.argmax(np.where(np.arange(40) < c.lens[b], c.age[b, h], -99)))
            c.cv[b, j, h, 3] = value
            c.cv[b, j, h, 17] = value
    c.w0 = None
    c.dev()
    c.run()
    c.check()
    assert torch.isfinite(c.out[:, :3]).all() and not torch.isfinite(c.out[:, 3, :, 3]).any()
    c.cv.nan_to_num_(nan=1.0, posinf=1.0, neginf=1.0)
    for b in range(2):
        for h in range(2):
            j = int(np.argmax(np.where(np.arange(40) < c.lens[b], c.age[b, h], -99)))
            c.ck[b, j, h] = value
    c.dev()
    c.run()
    torch.cuda.synchronize()
    assert torch.isfinite(c.out[:, :3]).all() and torch.isfinite(c.lse[:, :3]).all()


@pytest.mark.parametrize("B,P,cap", [(1, 0, 900), (2, 100, 40), (3, 700, 50), (40, 700, 5)])
def test_attention_of_a_query_that_is_not_a_number(B, P, cap):
    # its own row is NaN and no other
    c = AttentionCase(18, B, 2, 4, 2, 64, P, cap, BF, causal=True)
    c.w0 = None
    c.dev()
    c.run()
    want, lse = c.out.clone(), c.lse.clone()
    c.q[0, 1, 2] = math.nan
    c.run()
    torch.cuda.synchronize()
    assert torch.isnan(c.out[0, 1, 2]).all() and torch.isnan(c.lse[0, 1, 2])
    c.out[0, 1, 2], c.lse[0, 1, 2] = want[0, 1, 2], lse[0, 1, 2]
    assert torch.equal(c.out, want) and torch.equal(c.lse, lse)


def test_attention_large_scores_and_lowest_values():
    c = AttentionCase(11, 2, 1, 4, 2, 64, 50, 60, BF, lens=[60, 7], sigma=20.0)
    c.ck[0, 3] = torch.finfo(BF).min                       # scores overflow to an infinity of either sign
    c.q.abs_()
    c.dev()
    c.run()
    c.check()
    c = AttentionCase(12, 2, 1, 4, 2, 64, 9, 60, BF, lens=[60, 7], sigma=200.0)
    c.run()
    c.check()


@pytest.mark.parametrize("T,G,cap", [(1, 1, 6000), (3, 4, 5000), (9, 7, 2500)])
def test_attention_long_cache_few_rows(T, G, cap):
    # keys shared among a cluster; with 63 query rows the weights are computed from the keys again
    c = AttentionCase(13, 1, T, G, 1, 128, 100, cap, BF, causal=T > 1, lens=[cap - 3])
    c.run()
    c.check()


def test_attention_accumulates_over_steps_and_repeats_bit_for_bit():
    runs = []
    for _ in range(2):
        c = AttentionCase(14, 3, 2, 8, 2, 64, 200, 90, BF, causal=True)
        c.run()
        first = c.d_w.clone()
        cstr.cstr_cache_attention(c.cache, c.q, c.out, pos=c.d_pos, accumulate=True, lse_out=c.lse)
        cstr.cstr_cache_attention(c.cache, c.q, c.out, pos=c.d_pos)          # no accumulation
        torch.cuda.synchronize()
        assert torch.allclose(c.d_w - first, first - torch.from_numpy(c.w0).to(DEV), rtol=1e-4, atol=1e-6)
        runs.append((c.out.clone(), c.lse.clone(), c.d_w.clone()))
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_attention_on_another_stream_and_in_a_graph():
    c = AttentionCase(15, 4, 1, 8, 2, 128, 300, 64, BF)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.run(stream=side)
    side.synchronize()
    c.check()
    want = c.out.clone()
    graph = torch.cuda.CUDAGraph()
    c.out.zero_()
    with torch.cuda.graph(graph):
        cstr.cstr_cache_attention(c.cache, c.q, c.out)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(c.out, want)


def test_attention_and_insert_with_offsets_past_32_bits():
    row = 1 << 30                                           # elements between rows; three rows
    buf = torch.empty(2 * row + 2 * 40 * 64 + 64, dtype=BF, device=DEV)
    c = AttentionCase(16, 3, 1, 2, 1, 64, 9, 40, BF, lens=[40, 39, 31])
    ck = buf.as_strided((3, 40, 1, 64), (row, 64, 64, 1))
    cv = buf.as_strided((3, 40, 1, 64), (row, 64, 64, 1), 40 * 64)
    ck.copy_(c.ck)
    cv.copy_(c.cv)
    c.ck, c.cv = ck, cv
    c.run()
    c.check()
    rng = np.random.default_rng(3)
    k, v = random_cache(rng, 3, 1, 64, 2, None)
    w = rng.random((3, 1, 40)).astype(np.float32)
    check_insert(rng, ck, cv, w, c.age, np.array([40, 39, 31], np.int32), k, v,
                 np.array([40, 40, 40], np.int32), 40, 4)


def test_default_driver_refusals():
    c = AttentionCase(17, 2, 1, 4, 2, 64, 8, 10, BF)
    c.run()
    q, out = c.q, c.out
    bad = [dict(q=q.float()), dict(q=q[:1]), dict(q=q[..., :32]), dict(out=out.float()), dict(q=q.cpu()),
           dict(pos=torch.zeros(1, dtype=torch.int32, device=DEV)), dict(pos=torch.zeros(2, device=DEV)),
           dict(lse_out=torch.zeros(3, device=DEV)), dict(n_query=torch.zeros(2, dtype=torch.int32))]
    for kw in bad:
        a = dict(q=q, out=out)
        a.update(kw)
        with pytest.raises((TypeError, ValueError)):
            cstr.cstr_cache_attention(c.cache, a.pop("q"), a.pop("out"), **a)
    with pytest.raises(cstr.CstrError) as e:               # more tokens than the handle was made for
        cstr.cstr_cache_attention(c.cache, torch.cat([q, q], 1), torch.cat([out, out], 1))
    assert e.value.code == -2
    with pytest.raises(cstr.CstrError) as e:
        cstr.cstr_cache_attention(c.cache, q, out, scale=math.nan)
    assert e.value.code == -2
    wide = torch.zeros(2, 1, 4, 68, dtype=BF, device=DEV)
    with pytest.raises(cstr.CstrError) as e:               # stride no multiple of 8
        cstr.cstr_cache_attention(c.cache, wide[..., :64], out)
    assert e.value.code == -6
    bare = cstr.cstr_cache_create(c.ck, c.cv, c.d_lens, 4)
    for kw in (dict(accumulate=True), dict(pos=c.d_lens)):
        with pytest.raises(cstr.CstrError) as e:
            cstr.cstr_cache_attention(bare, q, out, **kw)
        assert e.value.code == -1
    with pytest.raises(cstr.CstrError) as e:
        cstr.cstr_cache_insert(bare, c.ck[:, :1], c.cv[:, :1], c.d_lens, 5)
    assert e.value.code == -1
    for budget, recent in ((0, 0), (11, 0), (5, 6), (5, -1)):
        with pytest.raises(cstr.CstrError) as e:
            cstr.cstr_cache_insert(c.cache, c.ck[:, :1], c.cv[:, :1], c.d_lens, budget, recent)
        assert e.value.code == -2
    with pytest.raises(cstr.CstrError):
        cstr.cstr_cache_insert(c.cache, c.ck[:, :2], c.cv[:, :2], c.d_lens, 5)
    for kw in (dict(n_heads=3), dict(n_heads=0), dict(max_tokens=0)):
        a = dict(n_heads=4, max_tokens=1)
        a.update(kw)
        with pytest.raises(cstr.CstrError):
            cstr.cstr_cache_create(c.ck, c.cv, c.d_lens, a["n_heads"], max_tokens=a["max_tokens"])
    with pytest.raises(cstr.CstrError):                    # head size
        cstr.cstr_cache_create(c.ck[..., :12], c.cv[..., :12], c.d_lens, 4)
    with pytest.raises(TypeError):
        cstr.cstr_cache_create(c.ck.float(), c.cv.float(), c.d_lens, 4)
    with pytest.raises(ValueError):
        cstr.cstr_cache_create(c.ck, c.cv, c.d_lens, 4, weight=torch.zeros(2, 2, 9, device=DEV))
    torch.cuda.synchronize()


# -------------------------------------------------------------- insertion

def random_insert(seed, B, Hk, D, cap, T, budget, recent, kind, dtype=BF):
    rng = np.random.default_rng(seed)
    ck, cv = random_cache(rng, B, Hk, D, cap, None, dtype)
    lens = rng.integers(0, cap + 1, B).astype(np.int32)
    lens[0], lens[-1] = cap, 0
    if kind == "full":
        lens[:] = budget
    age = ranked_ages(rng, lens, Hk, cap)
    w = rng.random((B, Hk, cap)).astype(np.float32)
    if kind == "ties":
        w = np.round(w * 3).astype(np.float32)
    if kind == "odd":
        w[rng.random(w.shape) < 0.1] = np.nan
        w[rng.random(w.shape) < 0.1] = np.inf
        w[rng.random(w.shape) < 0.1] = -np.inf
        w[rng.random(w.shape) < 0.1] = -0.0
        w[rng.random(w.shape) < 0.1] = 0.0
        w[rng.random(w.shape) < 0.1] *= -1
    k = v = None
    if T:
        k, v = random_cache(rng, B, Hk, D, T, None, dtype)
    n_new = rng.integers(-1, T + 2, B) if kind != "full" else None
    return rng, ck, cv, w, age, lens, k, v, lens + 3, budget, recent, n_new


@pytest.mark.parametrize("kind", ["full", "ties", "odd", "any"])
@pytest.mark.parametrize("B,Hk,D,cap,T,budget,recent", [
    (1, 1, 8, 1, 1, 1, 0), (3, 2, 64, 7, 1, 7, 3), (3, 2, 64, 40, 1, 33, 8), (2, 3, 80, 300, 17, 280, 100),
    (2, 1, 128, 700, 300, 600, 20), (3, 2, 16, 257, 256, 256, 256), (3, 1, 64, 100, 0, 50, 20),
    (2, 2, 8, 1030, 5, 5, 5), (2, 4, 24, 513, 2, 511, 0),
])
def test_insert(B, Hk, D, cap, T, budget, recent, kind):
    if kind == "full":
        budget = min(budget, cap)
    check_insert(*random_insert(cap * 7 + T, B, Hk, D, cap, T, budget, recent, kind))


def test_insert_half_precision_heads_layout_and_strided_tokens():
    args = list(random_insert(5, 3, 2, 64, 50, 4, 44, 10, "ties", HF))
    for i in (1, 2):                                       # [B][Hk][cap][D] storage
        args[i] = args[i].transpose(1, 2).contiguous().transpose(1, 2)
    both = torch.cat([args[6], args[7]], -1)               # tokens as slices of one projection
    args[6], args[7] = both[..., :64], both[..., 64:]
    check_insert(*args)


def test_insert_beyond_the_shared_memory_size():
    check_insert(*random_insert(6, 2, 1, 8, 24576 + 700, 40, 24576 + 100, 50, "ties"))
    check_insert(*random_insert(7, 2, 1, 8, 24576 + 700, 0, 300, 50, "odd"))


@pytest.mark.parametrize("cap", [2049, 4097, 8192, 8193, 12000])
def test_insert_sizes_at_which_the_kernel_changes(cap):
    check_insert(*random_insert(9, 3, 1, 8, cap, 70, cap - 50, 90, "ties"))
    check_insert(*random_insert(10, 3, 1, 8, cap, 1, cap - 3, 90, "full"))
    check_insert(*random_insert(11, 3, 2, 8, cap, 0, cap // 2, 0, "odd"))


def test_insert_repeated_steps_stay_within_budget():
    rng = np.random.default_rng(8)
    B, Hk, D, cap, budget = 3, 2, 16, 24, 20
    ck, cv = random_cache(rng, B, Hk, D, cap, None)
    lens = np.array([0, 5, 20], np.int32)
    pos = lens.copy()
    age, w = ranked_ages(rng, lens, Hk, cap), rng.random((B, Hk, cap)).astype(np.float32)
    side = torch.cuda.Stream()
    for step in range(30):
        k, v = random_cache(rng, B, Hk, D, 2, None)
        torch.cuda.synchronize()
        _, _, w, age, lens = check_insert(rng, ck, cv, w, age, lens, k, v, pos, budget, 6,
                                          stream=side if step % 2 else None)
        pos = pos + 2
        assert (lens <= budget).all()
        for b in range(B):                                 # the six newest positions are always there
            for h in range(Hk):
                have = set(age[b, h, :lens[b]].tolist())
                assert set(range(max(0, pos[b] - min(6, lens[b])), pos[b])) <= have | set(range(-9, 0))
        w = (w + rng.random(w.shape) * (np.arange(cap) < 9)).astype(np.float32)
