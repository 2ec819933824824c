"""Inputs and comparisons shared by the tests of the cache and loss operators."""
import math

import numpy as np
import torch

from oracle import operators as ref
from paper_2407_08103_b200 import cstr

DEV = "cuda:0"
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def f8(t):
    return t.detach().to(torch.float64).cpu().numpy()


def ranked_ages(rng, lens, heads, cap):
    """Distinct ages 0..len-1 in random order over each row's slots; garbage past len."""
    age = rng.integers(-50, 50, size=(len(lens), heads, cap))
    for b, n in enumerate(lens):
        for c in range(heads):
            age[b, c, :n] = rng.permutation(n)
    return age.astype(np.int32)


class AttentionCase:
    """Random caches whose unused slots hold NaN; ``layout`` 'heads' keeps slots of a head together."""

    def __init__(self, seed, B, T, Hq, Hk, D, P, cap, dtype, causal=False, lens=None, n_query=None,
                 layout="slots", sigma=1.0, weights=True, pad=0):
        rng = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        self.shape = (B, T, Hq, Hk, D, P, cap)

        def normal(*shape):
            return torch.randn(shape, generator=g).to(dtype).to(DEV)

        self.q = normal(B, T, Hq, D + pad)[..., :D] * sigma
        if pad:
            self.q = torch.cat([self.q, self.q], -1)[..., :D]      # inner stride 1, padded rows
        self.pk, self.pv = normal(P, Hk, D), normal(P, Hk, D)
        self.lens = rng.integers(0, cap + 1, B) if lens is None else np.asarray(lens)
        if causal:
            self.lens = np.maximum(self.lens, min(T, cap))
        if layout == "heads":
            self.ck, self.cv = (normal(B, Hk, cap, D).transpose(1, 2) for _ in range(2))
        else:
            self.ck, self.cv = normal(B, cap, Hk, D), normal(B, cap, Hk, D)
        for b in range(B):
            self.ck[b, self.lens[b]:] = math.nan
            self.cv[b, self.lens[b]:] = math.nan
        self.n_query = None if n_query is None else np.asarray(n_query, np.int32)
        new = T if self.n_query is None else self.n_query
        self.age = ranked_ages(rng, self.lens, Hk, cap)
        self.pos = (self.lens - new).astype(np.int32) if causal else None
        self.w0 = rng.random((B, Hk, cap)).astype(np.float32) if weights else None
        self.dev()

    def dev(self):
        B, T, Hq, Hk, D, P, cap = self.shape
        i32 = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)  # noqa: E731
        self.d_lens, self.d_age, self.d_pos, self.d_nq = map(i32, (self.lens, self.age, self.pos, self.n_query))
        self.d_w = None if self.w0 is None else torch.from_numpy(self.w0).to(DEV)
        self.out = torch.full((B, T, Hq, D), math.nan, dtype=self.q.dtype, device=DEV)
        self.lse = torch.full((B, T, Hq), math.nan, device=DEV)

    def run(self, stream=None, scale=None):
        T, P = self.shape[1], self.shape[5]
        self.cache = cstr.cstr_cache_create(self.ck, self.cv, self.d_lens, self.shape[2],
                                            prefix_k=self.pk if P else None, prefix_v=self.pv if P else None,
                                            weight=self.d_w, age=self.d_age, max_tokens=T)
        cstr.cstr_cache_attention(self.cache, self.q, self.out, scale=scale, pos=self.d_pos,
                                  n_query=self.d_nq, accumulate=self.w0 is not None, lse_out=self.lse,
                                  stream=stream)

    def check(self, scale=None):
        torch.cuda.synchronize()
        D = self.shape[4]
        scale = D ** -0.5 if scale is None else scale
        r = ref.attention(f8(self.q), f8(self.pk), f8(self.pv), f8(self.ck), f8(self.cv), self.lens, scale,
                          self.age, self.pos, self.n_query, self.w0)
        u, n = UNIT[self.q.dtype], self.shape[5] + self.shape[6]
        # score: D fp32 additions of exact products, then scale, log2(e) and the exponential
        score = D * 2.0 ** -24 * r["abs_score"] + 2.0 ** -22 * (r["abs_score"] + 1.0)
        lse = f8(self.lse)
        none = np.isneginf(r["lse"])
        assert np.array_equal(np.isneginf(lse), none)
        err = np.abs(lse[~none] - r["lse"][~none])
        tol = (score + 2.0 ** -22 * (np.abs(np.where(none, 0.0, r["lse"])) + n * 2.0 ** -24 + 4.0))[~none]
        assert (err <= tol).all(), "lse off by %g" % (err - tol).max()
        # output: probabilities rounded to the values' type (half of them below 2^-14 to a multiple
        # of 2^-24), one rounding of the result, the scores' own error
        out = f8(self.out)
        finite = np.isfinite(r["out"])
        assert np.array_equal(np.isfinite(out), finite)
        vmax = np.abs(f8(self.pv)).max(initial=0.0) + np.nan_to_num(np.abs(f8(self.cv)), nan=0, posinf=0).max(initial=0.0)
        tiny = n * 2.0 ** -25 * vmax if self.q.dtype == torch.float16 else 0.0
        tol = u * (np.abs(r["out"]) + r["abs_out"]) + 4.0 * score[..., None] * r["abs_out"] + tiny + 1e-30
        bad = np.abs(out - r["out"])[finite] > tol[finite]
        assert not bad.any(), "out off by %g" % (np.abs(out - r["out"]) - tol)[finite].max()
        if self.w0 is not None:
            w = f8(self.d_w)
            heads = r["added"].shape[1]
            per = score.reshape(score.shape[0], score.shape[1], heads, -1).max((1, 3))[:, :, None]
            tol = r["added"] * (4.0 * per + 2.0 ** -18) + 2.0 ** -23 * (np.abs(r["weight"]) + 1e-30)
            assert (np.abs(w - r["weight"]) <= tol).all(), "weight off by %g" % (np.abs(w - r["weight"]) - tol).max()
        return r


def random_cache(rng, B, Hk, D, cap, lens, dtype=torch.bfloat16):
    ck = torch.from_numpy(rng.standard_normal((B, cap, Hk, D)).astype(np.float32)).to(dtype).to(DEV)
    cv = torch.from_numpy(rng.standard_normal((B, cap, Hk, D)).astype(np.float32)).to(dtype).to(DEV)
    return ck, cv


def check_insert(rng, ck, cv, weight, age, lens, k_new, v_new, pos, budget, recent, n_new=None,
                 max_tokens=None, stream=None):
    """One insertion against the oracle, bit for bit; returns the new host arrays."""
    d_w, d_a, d_l, d_p = (torch.from_numpy(np.ascontiguousarray(x)).to(DEV) for x in (weight, age, lens, pos))
    d_n = None if n_new is None else torch.from_numpy(np.asarray(n_new, np.int32)).to(DEV)
    T = 0 if k_new is None else k_new.shape[1]
    bits = lambda t: t.contiguous().view(torch.int16).cpu().numpy()  # noqa: E731
    want = ref.insert(bits(ck), bits(cv), weight, age, lens, None if k_new is None else bits(k_new),
                      None if v_new is None else bits(v_new), pos, budget, recent, n_new)
    cache = cstr.cstr_cache_create(ck, cv, d_l, ck.shape[2], weight=d_w, age=d_a,
                                   max_tokens=max(1, T if max_tokens is None else max_tokens))
    cstr.cstr_cache_insert(cache, k_new, v_new, d_p, budget, recent, n_new=d_n, stream=stream)
    torch.cuda.synchronize()
    assert np.array_equal(d_l.cpu().numpy(), want[4])
    assert np.array_equal(d_a.cpu().numpy(), want[3])
    assert np.array_equal(d_w.cpu().numpy().view(np.int32), want[2].view(np.int32))
    assert np.array_equal(bits(ck), want[0])
    assert np.array_equal(bits(cv), want[1])
    return want


def check_loss(x, allowed, actions, old, adv, tables=None, states=None, row_table=None, ref_logp=None,
               weight=None, gradient=True, in_place=False, stream=None, **kw):
    """``x``: device logits [N][V] (any row stride); compares with the oracle."""
    N, V = x.shape
    t = lambda a, dt=torch.float32: None if a is None else torch.as_tensor(np.asarray(a)).to(dt).to(DEV)  # noqa: E731
    host = f8(x)
    loss, logp = (torch.full((N,), math.nan, device=DEV) for _ in range(2))
    d = None
    if gradient:
        if in_place:
            d = x
        else:
            d = torch.full((max(N, 1) * x.stride(0),), math.nan, dtype=x.dtype, device=DEV)
            d = d.as_strided((N, V), x.stride())
    dev = [t(actions, torch.int32), t(old), t(adv), t(ref_logp), t(weight)]
    cstr.cstr_policy_loss(tables, x, t(states, torch.int32), dev[0], dev[1], dev[2], loss, logp,
                          ref_logp=dev[3], weight=dev[4], dlogits=d, row_table=t(row_table, torch.int32),
                          stream=stream, **kw)
    torch.cuda.synchronize()
    h = [None if y is None else f8(y) for y in dev]
    want = ref.policy_loss(host, allowed, actions, h[1], h[2], h[3], h[4], **kw)
    # logp: logits up to |z| in 32 bits (scaled by log2(e) / temperature and back), the sum of the
    # exponentials to 2^-18; loss and gradient carry the ratio's relative error, which is logp's absolute
    with np.errstate(invalid="ignore"):
        z = np.where(allowed & np.isfinite(host), np.abs(host), 0.0).max(1) / kw.get("temperature", 1.0)
        fine = np.isfinite(want[1])
        e_logp = 2.0 ** -21 * (z + np.abs(np.where(fine, want[1], 0.0)) + 1.0) + 2.0 ** -18
        assert np.array_equal(np.isnan(f8(logp)), np.isnan(want[1]))
        assert np.array_equal(np.isneginf(f8(logp)), np.isneginf(want[1]))
        assert (np.abs(f8(logp) - want[1])[fine] <= e_logp[fine]).all()
        lw = np.ones(N) if weight is None else np.abs(h[4])
        ratio = np.exp(np.where(fine, want[1], 0.0) - h[1])
        k = 0.0 if ref_logp is None else np.exp(h[3] - np.where(fine, want[1], 0.0)) + np.abs(h[3]) + np.abs(np.where(fine, want[1], 0.0)) + 1.0
        size = lw * (ratio * np.abs(h[2]) + kw.get("kl_coef", 0.0) * k + np.abs(h[2]) * (1 + kw.get("clip_high", 0.2)))
        ok = np.isfinite(want[0])
        assert np.array_equal(np.isfinite(f8(loss)), ok)
        assert (np.abs(f8(loss) - want[0])[ok] <= (size * (4 * e_logp + 2.0 ** -20))[ok]).all()
        if gradient:
            got = f8(d)
            gok = np.isfinite(want[2])
            assert np.array_equal(np.isfinite(got), gok)
            soft = np.where(allowed, host / kw.get("temperature", 1.0), -np.inf)
            soft = np.exp(soft - np.maximum(soft.max(1, keepdims=True), -1e300))
            soft = np.nan_to_num(soft / np.maximum(soft.sum(1, keepdims=True), 1e-300))
            soft[np.arange(N), np.clip(h[0].astype(np.int64), 0, V - 1)] += 1.0
            rel = size * (8 * e_logp + 2.0 ** -19) / kw.get("temperature", 1.0)
            tol = UNIT[x.dtype] * np.abs(want[2]) + rel[:, None] * soft + 1e-37
            assert (np.abs(got - want[2])[gok] <= tol[gok]).all()
            assert (got[~allowed & gok] == 0).all()
    return want
