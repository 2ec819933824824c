"""Edges of the cache and loss operators at which a call once went wrong."""
import ctypes
import math
import threading

import numpy as np
import pytest
import torch

from oracle import operators as ref
from paper_2407_08103_b200 import cstr

from operator_cases import DEV, AttentionCase, check_insert, check_loss, f8, random_cache, ranked_ages

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


# P: prompt in the row kernel (or none), on the tensor cores with one and with two tiles of query rows
@pytest.mark.parametrize("P,B", [(0, 2), (33, 2), (700, 2), (700, 40)])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_a_single_token_is_not_reached_by_slots_it_does_not_see(dtype, value, P, B):
    c = AttentionCase(51, B, 1, 8, 2, 64, P, 40, dtype, causal=True, lens=[40, 21] * (B // 2))
    for b in range(B):
        for h in range(2):
            j = int(np.argmax(c.age[b, h, :c.lens[b]] == 7))
            c.age[b, h, j] = c.pos[b] + 3                  # younger than the token
            c.ck[b, j, h] = value
            c.cv[b, j, h] = value
    c.dev()
    c.run()
    c.check()
    assert torch.isfinite(c.out).all() and torch.isfinite(c.d_w).all()


# long caches of one row whose weights are computed from the keys again (63 and 8 query rows), and
# one whose scores are kept
@pytest.mark.parametrize("P,cap,T,G,D", [(100, 10000, 9, 7, 128), (600, 10000, 9, 7, 128), (100, 48000, 4, 2, 128),
                                         (0, 300, 9, 7, 64)])
@pytest.mark.parametrize("value", [math.nan, math.inf, 3e38])
def test_queries_past_n_query_do_not_reach_the_weights(value, P, cap, T, G, D):
    c = AttentionCase(52, 1, T, G, 1, D, P, cap, BF, causal=True, lens=[cap - 7], n_query=[2])
    c.q[0, 2:] = value                                     # padding: may hold anything
    c.dev()
    c.run()
    c.check()
    assert torch.isfinite(c.d_w).all()


# rows shared by clusters of 2 to 16 blocks, the last ones with short shares or (narrow rows) none
@pytest.mark.parametrize("N,V", [(1, 8193), (2, 16385), (1, 65537), (40, 32769), (9, 131073), (300, 16390)])
@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_loss_of_rows_shared_by_a_cluster(dtype, N, V):
    g = torch.Generator(device=DEV).manual_seed(V)
    x = torch.randn(N, V, generator=g, device=DEV).to(dtype)
    act = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    adv = torch.ones(N, device=DEV)
    want = torch.log_softmax(x.double(), 1).gather(1, act.long()[:, None])[:, 0]
    runs = []
    for _ in range(20):
        loss, logp, d = torch.empty(N, device=DEV), torch.empty(N, device=DEV), torch.empty_like(x)
        cstr.cstr_policy_loss(None, x, None, act, want.float(), adv, loss, logp, dlogits=d)
        runs.append((loss, logp, d))
    assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(runs[0], r))
    # logits below 8 and log probabilities below 32 in 32 bits, the sum of the exponentials to 2^-18
    assert (runs[0][1].double() - want).abs().max() <= 2.0 ** -21 * 41 + 2.0 ** -18


# logits far from zero: a model's own masks of -1e9 or -1e30 over all that the constraint allows, or a common offset
@pytest.mark.parametrize("offset", [0.0, 1e4, -1e4, 1e6, -1e9, 1e9, -1e30, 1e30])
@pytest.mark.parametrize("temperature", [1.0, 0.25])
@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_loss_of_logits_with_a_large_offset(dtype, temperature, offset):
    N, V = 6, 5000
    g = torch.Generator().manual_seed(5)
    x = (2.0 * torch.randn(N, V, generator=g, dtype=torch.float64) + offset).to(dtype).to(DEV)
    act = x.argmax(1).int()
    soft = torch.log_softmax(x.double() / temperature, 1)
    want = soft.gather(1, act.long()[:, None])[:, 0]
    old, adv = want.float(), torch.ones(N, device=DEV)
    loss, logp, d = torch.empty(N, device=DEV), torch.empty(N, device=DEV), torch.empty_like(x)
    cstr.cstr_policy_loss(None, x, None, act, old, adv, loss, logp, dlogits=d, temperature=temperature)
    # Differences of logits to the maximum that weigh (32 below it at most) in one rounding, scaled in another:
    # 32 x 2^-22 of an exponent, and 2^-21 a step for the exponential, their sum, its logarithm (below 16)
    tol = 2.0 ** -17 + 2.0 ** -18
    assert (logp.double() - want).abs().max() <= tol
    ratio = torch.exp(want - old.double())[:, None]
    hot = torch.zeros_like(soft).scatter_(1, act.long()[:, None], 1.0)
    grad = -ratio * (hot - soft.exp()) / temperature
    size = ratio * (hot + soft.exp()) / temperature
    unit = 2.0 ** -8 if dtype == BF else 2.0 ** -23
    assert ((d.double() - grad).abs() <= unit * grad.abs() + 4 * tol * size + 1e-12).all()
    assert ((loss.double() + ratio[:, 0]).abs() <= 2 * tol).all()


@pytest.mark.parametrize("step", [1e-6, 1e-4, -1e-3, 1e-2, -0.3, 5.0])
def test_kl_term_near_the_reference_policy(step):
    # the term is about d^2 / 2 there, of summands about 1
    N, V = 64, 1000
    g = torch.Generator().manual_seed(6)
    x = torch.randn(N, V, generator=g).to(DEV)
    act = torch.randint(0, V, (N,), generator=g).int().to(DEV)
    lp = torch.log_softmax(x.double(), 1).gather(1, act.long()[:, None])[:, 0]
    loss, logp, d = torch.empty(N, device=DEV), torch.empty(N, device=DEV), torch.empty_like(x)
    near = (lp + step).float()
    cstr.cstr_policy_loss(None, x, None, act, lp.float(), torch.zeros(N, device=DEV), loss, logp, ref_logp=near,
                          kl_coef=1.0, dlogits=d)
    diff = near.double() - logp.double()                    # exact: both have 24 bits
    want = torch.expm1(diff) - diff
    # the difference in 32 bits, then exp(d) - 1 to two units of its last place, then one subtraction
    size = diff.abs() + torch.expm1(diff).abs()
    assert ((loss.double() - want).abs() <= 2.0 ** -21 * size).all()
    hot = d.gather(1, act.long()[:, None])[:, 0].double()
    p = logp.double().exp()
    assert ((hot + torch.expm1(diff) * (1 - p)).abs() <= 2.0 ** -18 * size + 1e-12).all()


def test_handles_of_several_threads_side_by_side():
    # handles of different sizes launch the same kernels, each from its own thread and stream
    cases = [(cap, AttentionCase(60 + i, 2, 1, 4, 2, 64, 33, cap, BF, lens=[cap, cap - 1]))
             for i, cap in enumerate((40, 3000, 9000, 20000))]
    torch.cuda.synchronize()
    failed = []

    def work(c, cap):
        try:
            side = torch.cuda.Stream()
            c.run(stream=side)
            k, v = (torch.zeros(2, 2, 2, 64, dtype=BF, device=DEV) for _ in range(2))
            pos = torch.full((2,), cap, dtype=torch.int32, device=DEV)
            torch.cuda.current_stream().synchronize()
            for _ in range(50):
                cstr.cstr_cache_attention(c.cache, c.q, c.out, stream=side)
            big = cstr.cstr_cache_create(c.ck, c.cv, c.d_lens, 4, weight=c.d_w.clone(), age=c.d_age, max_tokens=2)
            side.synchronize()
            for _ in range(20):
                cstr.cstr_cache_insert(big, k, v, pos, cap, 2, stream=side)
            side.synchronize()
        except Exception as e:                             # (an assertion in a thread would pass unseen)
            failed.append(e)
    for _ in range(3):
        threads = [threading.Thread(target=work, args=(c, cap)) for cap, c in cases]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    assert not failed


def test_a_new_handle_is_ready_on_any_stream():
    # while the default stream is busy, on a stream that does not wait for it
    rng = np.random.default_rng(4)
    side = torch.cuda.Stream()
    for i in range(3):
        B, Hk, cap = 50, 8, 40
        ck, cv = random_cache(rng, B, Hk, 64, cap, None)
        k, v = random_cache(rng, B, Hk, 64, 2, None)
        lens = np.full(B, cap, np.int32)
        age, w = ranked_ages(rng, lens, Hk, cap), rng.random((B, Hk, cap)).astype(np.float32)
        d = [torch.from_numpy(a).to(DEV) for a in (w, age, lens)]
        pos = torch.full((B,), cap, dtype=torch.int32, device=DEV)
        want = ref.insert(f8(ck), f8(cv), w, age, lens, f8(k), f8(v), lens, cap - 3, 5)
        torch.cuda.synchronize()
        torch.cuda._sleep(200_000_000)                     # about 0.1 s
        cache = cstr.cstr_cache_create(ck, cv, d[2], Hk, weight=d[0], age=d[1], max_tokens=2)
        cstr.cstr_cache_insert(cache, k, v, pos, cap - 3, 5, stream=side)
        side.synchronize()
        torch.cuda.synchronize()
        assert np.array_equal(d[2].cpu().numpy(), want[4]) and (want[4] == cap - 3).all()
        assert np.array_equal(d[1].cpu().numpy(), want[3]) and np.array_equal(f8(ck), want[0])


# the row kernel alone, and behind one and two tiles of query rows on the tensor cores
@pytest.mark.parametrize("P,B", [(100, 2), (600, 2), (2000, 40)])
@pytest.mark.parametrize("x", [14.5, 18.3, 20.4, 22.6, 24.3, 26.0])
def test_half_precision_keeps_small_probabilities(x, P, B):
    # one key with nearly all of the weight, which has value 0; all others 2^-x of it each
    c = AttentionCase(53, B, 1, 4, 1, 64, P, 4, HF, lens=[2] * B, weights=False)
    c.q.zero_()
    c.q[..., 0] = 1.0
    c.pk.zero_()
    c.pk[1:, 0, 0] = -x * math.log(2.0)
    c.pv[:] = 64.0
    c.pv[0] = 0.0
    c.ck[:, :2], c.cv[:, :2] = 0.0, 0.0
    c.ck[:, :2, 0, 0] = -30.0
    c.dev()
    c.run(scale=1.0)
    torch.cuda.synchronize()
    e = np.exp(f8(c.pk)[:, 0, 0])
    want = 64.0 * e[1:].sum() / (e.sum() + 2 * math.exp(-30.0))
    # the same rounding in every probability and one of the output, 2^-11 each; probabilities count in
    # multiples of 2^-24 below 2^-14, and enter the product multiplied by 2^7 at least
    tol = want * (2.0 ** -10 + 2.0 ** (x - 32) + 2.0 ** -14)
    assert np.abs(f8(c.out) - want).max() <= tol


# one tile of query rows and two; the waits of the attention over the prompt get no second try
@pytest.mark.parametrize("B,dim", [(3, 64), (70, 128)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_waits_that_run_out_are_counted_and_leave_the_device_usable(dtype, B, dim):
    cstr.use_check_library(True)
    try:
        c = AttentionCase(70, B, 1, 8, 2, dim, 2000, 20, dtype, weights=False)
        c.run()
        want, lse = c.out.clone(), c.lse.clone()
        assert cstr.cstr_cache_status(c.cache) == 0
        cstr.cstr_test_set_wait_limit(0)
        try:
            for _ in range(3):
                cstr.cstr_cache_attention(c.cache, c.q, c.out, lse_out=c.lse)
                assert cstr.cstr_cache_status(c.cache) > 0
        finally:
            cstr.cstr_test_set_wait_limit(-1)
        cstr.cstr_cache_attention(c.cache, c.q, c.out, lse_out=c.lse)
        assert cstr.cstr_cache_status(c.cache) == 0
        assert torch.equal(c.out, want) and torch.equal(c.lse, lse)
    finally:
        cstr.use_check_library(False)


@pytest.mark.parametrize("B,dim", [(3, 64), (70, 128), (300, 64)])
def test_no_answer_comes_of_a_block_that_gave_up(B, dim):
    # what the call before left in the scratch is not taken for this call's parts
    cstr.use_check_library(True)
    try:
        c = AttentionCase(71, B, 1, 8, 2, dim, 2000, 20, BF, weights=False)
        other = c.q.clone().neg_()
        c.run()
        right, right_lse = c.out.clone(), c.lse.clone()
        cstr.cstr_cache_attention(c.cache, other, c.out)   # (its parts are what would be left)
        cstr.cstr_test_set_wait_limit(0)
        try:
            for _ in range(5):
                c.out.zero_()
                c.lse.zero_()
                cstr.cstr_cache_attention(c.cache, c.q, c.out, lse_out=c.lse)
                assert cstr.cstr_cache_status(c.cache) > 0
                lost = c.lse.isnan()
                assert lost.any() and (c.out.isnan().all(-1) == lost).all()
                assert torch.equal(c.out[~lost], right[~lost]) and torch.equal(c.lse[~lost], right_lse[~lost])
        finally:
            cstr.cstr_test_set_wait_limit(-1)
    finally:
        cstr.use_check_library(False)


# one entry to evict or several, by a warp and by a block
@pytest.mark.parametrize("T,budget", [(1, 40), (1, 30), (3, 38), (0, 20), (70, 3000)])
def test_protected_entries_that_have_to_go_do_so_by_slot(T, budget):
    rng = np.random.default_rng(T)
    cap = 3000 if T == 70 else 40
    lens = np.array([cap, cap - 1, budget], np.int32)
    ck, cv = random_cache(rng, 3, 2, 16, cap, None)
    k, v = random_cache(rng, 3, 2, 16, T, None) if T else (None, None)
    age = ranked_ages(rng, lens, 2, cap)
    pos = np.array([5, 0, 8], np.int32)                    # entries at and past it count as recent
    w = rng.random((3, 2, cap)).astype(np.float32)
    check_insert(rng, ck, cv, w, age, lens, k, v, pos, budget, 2)


@pytest.mark.parametrize("cap,scratch", [(2048, True), (2049, False), (24576, False), (24577, True)])
def test_scratch_of_the_insertion_only_where_it_is_used(cap, scratch):
    B, Hk = (64 << 20) // (cap * 4 * 8), 4                 # 64 MB of it
    ck = torch.zeros(8, dtype=BF, device=DEV).expand(B, cap, Hk, 8)      # (not read)
    w, age = torch.zeros(B, Hk, cap, device=DEV), torch.zeros(B, Hk, cap, dtype=torch.int32, device=DEV)
    lens = torch.zeros(B, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    cache = cstr.cstr_cache_create(ck, ck, lens, Hk, weight=w, age=age)
    used = before - torch.cuda.mem_get_info()[0]
    cache.close()
    assert (used > 48 << 20) == scratch, used


# many new tokens at once: several passes of 32 query rows over the slots, tiles of 128 that start within a row
@pytest.mark.parametrize("B,T,Hq,Hk,D,P,cap", [(2, 33, 2, 1, 64, 0, 300), (1, 64, 4, 2, 128, 700, 90), (2, 129, 2, 2, 64, 130, 400),
                                               (1, 256, 4, 1, 128, 600, 1500), (3, 65, 8, 1, 40, 513, 70)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_attention_of_a_long_new_input(dtype, B, T, Hq, Hk, D, P, cap):
    c = AttentionCase(80, B, T, Hq, Hk, D, P, cap, dtype, causal=True, lens=[cap] + [max(T, cap - 5)] * (B - 1),
                      n_query=[T] + [T // 2 + 1] * (B - 1))
    c.run()
    c.check()
    assert cstr.cstr_cache_status(c.cache) == 0


# long prompts of few key / value heads
@pytest.mark.parametrize("B,T,Hq,Hk,D,P", [(1, 1, 8, 1, 128, 30000), (16, 1, 8, 1, 64, 9000), (2, 2, 16, 2, 128, 20001), (40, 1, 8, 2, 64, 6000)])
def test_attention_of_few_heads_over_a_long_prompt(B, T, Hq, Hk, D, P):
    c = AttentionCase(81, B, T, Hq, Hk, D, P, 12, BF, causal=T > 1)
    c.run()
    c.check()
    assert cstr.cstr_cache_status(c.cache) == 0


def test_prompts_that_the_copy_engine_cannot_read():
    # one head's keys for all heads (a stride of 0), and tokens stored last to first (a negative one)
    c = AttentionCase(82, 3, 1, 8, 2, 64, 700, 20, BF)
    c.pk = c.pk[:, :1].expand(700, 2, 64)
    c.run()
    c.check()
    c = AttentionCase(83, 3, 2, 8, 2, 64, 700, 20, HF, causal=True)
    pk, pv = c.pk.flip(0).contiguous(), c.pv.flip(0).contiguous()
    out = ctypes.c_void_p()
    at = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    cstr._check(cstr.lib().cstr_cache_create(
        2, 3, 8, 2, 64, 2, at(pk[-1]), at(pv[-1]), ctypes.c_int64(700), (ctypes.c_int64 * 4)(-128, 64, -128, 64),
        at(c.ck), at(c.cv), 20, (ctypes.c_int64 * 6)(*c.ck.stride()[:3], *c.cv.stride()[:3]),
        at(c.d_w), at(c.d_age), at(c.d_lens), ctypes.byref(out)))
    cache = cstr.Cache(out)
    c.run()                                                # (a handle of the prompt in its usual order)
    c.check()
    cache.batch, cache.n_heads, cache.n_kv_heads, cache.head_dim = 3, 8, 2, 64
    cache.dtype, cache.device, cache.strides = HF, c.ck.device, {}
    c.d_w.copy_(torch.from_numpy(c.w0))
    cstr.cstr_cache_attention(cache, c.q, c.out, pos=c.d_pos, accumulate=True, lse_out=c.lse)
    c.check()


@pytest.mark.parametrize("N,V", [(3, 1003), (5, 32000), (2, 128256)])
def test_scoring_of_bfloat16_logits(N, V):
    rng = np.random.default_rng(V)
    x = torch.randn(N, V, generator=torch.Generator().manual_seed(V)).mul_(3.0).to(BF).to(DEV)
    ok = np.ones((N, V), bool)
    check_loss(x, ok, rng.integers(0, V, N), np.full(N, -9.0, np.float32), rng.standard_normal(N).astype(np.float32), gradient=False)


def test_a_scale_that_overflows_with_log2_e_is_refused():
    c = AttentionCase(84, 2, 1, 4, 2, 64, 8, 10, BF)
    c.run(scale=2.3e38)                                    # the largest ones are not
    for scale in (2.5e38, -3.4e38):
        with pytest.raises(cstr.CstrError) as e:
            cstr.cstr_cache_attention(c.cache, c.q, c.out, scale=scale)
        assert e.value.code == -2
