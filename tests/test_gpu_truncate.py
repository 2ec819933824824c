"""Tokens taken back from the rows' caches: the kernel against the oracle, bit for bit, and the driver in a
loop that drafts tokens and keeps some of them."""
import numpy as np
import pytest
import torch

from oracle import operators as ref
from paper_2407_08103_b200 import cstr
from paper_2407_08103_b200.decode import SharedPromptCache

from operator_cases import DEV, random_cache, ranked_ages

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def check_truncate(ck, cv, weight, age, lens, pos, stream=None):
    d_w, d_a, d_l, d_p = (torch.from_numpy(np.ascontiguousarray(x)).to(DEV) for x in (weight, age, lens, pos))
    bits = lambda t: t.contiguous().view(torch.int16).cpu().numpy()  # noqa: E731
    want = ref.truncate(bits(ck), bits(cv), weight, age, lens, pos)
    cache = cstr.cstr_cache_create(ck, cv, d_l, ck.shape[2], weight=d_w, age=d_a)
    torch.cuda.synchronize()
    for _ in range(2):                                     # (once more takes nothing)
        cstr.cstr_cache_truncate(cache, d_p, stream=stream)
        torch.cuda.synchronize()
        assert np.array_equal(d_l.cpu().numpy(), want[4])
        assert np.array_equal(d_a.cpu().numpy(), want[3])
        assert np.array_equal(d_w.cpu().numpy().view(np.int32), want[2].view(np.int32))
        assert np.array_equal(bits(ck), want[0]) and np.array_equal(bits(cv), want[1])
    return want


@pytest.mark.parametrize("B,Hk,D,cap", [(1, 1, 8, 1), (5, 2, 64, 40), (4, 9, 16, 33), (5, 3, 80, 700), (3, 1, 8, 4097), (4, 1, 8, 24576 + 500)])
@pytest.mark.parametrize("take", [0, 1, 2, 7, 10 ** 6])
def test_newest_tokens_leave(B, Hk, D, cap, take):
    rng = np.random.default_rng(cap + take)
    ck, cv = random_cache(rng, B, Hk, D, cap, None)
    lens = rng.integers(0, cap + 1, B).astype(np.int32)
    lens[0] = cap
    if B > 2:
        lens[1], lens[2] = 0, min(1, cap)
    w = rng.random((B, Hk, cap)).astype(np.float32)
    want = check_truncate(ck, cv, w, ranked_ages(rng, lens, Hk, cap), lens, np.maximum(lens - take, -5).astype(np.int32))
    assert np.array_equal(want[4], np.maximum(lens - take, 0))


@pytest.mark.parametrize("cap", [30, 5000])
def test_heads_that_have_lost_some_of_them(cap):
    # ages differ from head to head, as after insertions that evicted; weights with ties, NaN, both zeroes
    rng = np.random.default_rng(cap)
    B, Hk = 6, 4
    ck, cv = random_cache(rng, B, Hk, 16, cap, None)
    lens = rng.integers(cap // 2, cap + 1, B).astype(np.int32)
    age = np.argsort(rng.random((B, Hk, 3 * cap)), -1)[..., :cap].astype(np.int32)
    w = np.round(rng.random((B, Hk, cap)) * 3).astype(np.float32)
    for value in (np.nan, -0.0, -np.inf, np.inf, -2.0):
        w[rng.random(w.shape) < 0.05] = value
    side = torch.cuda.Stream()
    check_truncate(ck, cv, w, age, lens, rng.integers(2 * cap, 3 * cap, B).astype(np.int32), stream=side)


def test_refusals():
    ck = torch.zeros(2, 4, 1, 8, dtype=BF, device=DEV)
    lens = torch.zeros(2, dtype=torch.int32, device=DEV)
    bare = cstr.cstr_cache_create(ck, ck.clone(), lens, 1)
    with pytest.raises(cstr.CstrError) as e:
        cstr.cstr_cache_truncate(bare, lens)
    assert e.value.code == -1
    for pos in (None, lens[:1], lens.float(), lens.cpu()):
        with pytest.raises(ValueError):
            cstr.cstr_cache_truncate(bare, pos)


def test_indices_stay_in_range():
    cstr.use_check_library(True)
    try:
        cstr.cstr_debug_bounds_status(reset=True)
        for take in (1, 7):
            test_newest_tokens_leave(5, 2, 64, 40, take)
            test_newest_tokens_leave(5, 3, 80, 700, take)
        test_heads_that_have_lost_some_of_them(30)
        record = cstr.cstr_debug_bounds_status(reset=True)
        assert record[0] == 0, "out-of-range index: site %d, index %d, extent %d" % record[1:]
    finally:
        cstr.use_check_library(False)


def test_the_driver_drafts_and_takes_rejected_tokens_back():
    # what is kept decides the attention of every later step, as if the rejected drafts had never been there
    g = torch.Generator(device=DEV).manual_seed(1)
    rng = np.random.default_rng(1)
    B, H, K, D, P = 3, 4, 2, 64, 150

    def normal(*s):
        return torch.randn(s, generator=g, device=DEV).bfloat16()
    pk, pv = normal(P, K, D), normal(P, K, D)
    cache = SharedPromptCache(pk, pv, B, H, budget=40, recent=2, max_tokens=4)
    kept_k, kept_v = [[pk] for _ in range(B)], [[pv] for _ in range(B)]
    for step in range(9):
        T = (4, 1, 3)[step % 3]
        q, k, v = normal(B, T, H, D), normal(B, T, K, D), normal(B, T, K, D)
        out = cache.step(q, k, v)
        drop = rng.integers(0, T, B) if T > 1 else np.zeros(B, np.int64)
        for b in range(B):
            for i in range(T):
                kk = torch.cat(kept_k[b] + [k[b, :i + 1]]).double().repeat_interleave(H // K, 1)
                vv = torch.cat(kept_v[b] + [v[b, :i + 1]]).double().repeat_interleave(H // K, 1)
                p = torch.softmax(torch.einsum("hd,xhd->hx", q[b, i].double(), kk) / D ** 0.5, -1)
                want, size = torch.einsum("hx,xhd->hd", p, vv), torch.einsum("hx,xhd->hd", p, vv.abs())
                assert ((out[b, i].double() - want).abs() <= 2.0 ** -8 * (want.abs() + size)).all()
            keep = T - int(drop[b])
            kept_k[b].append(k[b, :keep])
            kept_v[b].append(v[b, :keep])
        if T > 1:
            cache.take_back(torch.from_numpy(drop.astype(np.int32)).to(DEV))
        have = [sum(len(x) for x in kept_k[b][1:]) for b in range(B)]
        assert cache.lens.tolist() == cache.pos.tolist() == have
        for b in range(B):
            assert sorted(cache.age[b, 0, :have[b]].tolist()) == list(range(have[b]))
    cache.take_back(torch.tensor([-1, 0, 10 ** 6], dtype=torch.int32, device=DEV))
    assert cache.lens.tolist() == cache.pos.tolist() == have[:2] + [0]
