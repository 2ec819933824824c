"""Plain statements in 64 bits of the operators around the constrained step: attention over a
shared prompt and per-row caches, insertion with eviction by accumulated attention weight, and
the clipped policy loss over the constrained distribution.  Test infrastructure only; loops over
rows, no code shared with the GPU path."""

from __future__ import annotations

import math

import numpy as np


def attention(q, prefix_k, prefix_v, cache_k, cache_v, lens, scale, age=None, pos=None,
              n_query=None, weight=None):
    """float64 arrays ``q`` [B][T][Hq][D], prefix [P][Hk][D], caches [B][cap][Hk][D].  Returns a dict
    with ``out``, ``lse``, ``weight`` (None in, None out) and, for error bounds, ``abs_out`` =
    sum p |v|, ``abs_score`` = largest scale * sum |q_d k_d| per query, ``added`` = weight received."""
    B, T, Hq, D = q.shape
    P, Hk = prefix_k.shape[0], cache_k.shape[2]
    G = Hq // Hk
    out, abs_out = np.zeros(q.shape), np.zeros(q.shape)
    lse = np.full((B, T, Hq), -np.inf)
    abs_score = np.zeros((B, T, Hq))
    added = np.zeros((B, Hk, cache_k.shape[1]))
    for b in range(B):
        n = min(max(int(lens[b]), 0), cache_k.shape[1])
        m = T if n_query is None else min(max(int(n_query[b]), 0), T)
        for t in range(m):
            for h in range(Hq):
                c = h // G
                slots = [j for j in range(n) if pos is None or age[b, c, j] <= pos[b] + t]
                k = np.concatenate([prefix_k[:, c], cache_k[b, slots, c]])
                v = np.concatenate([prefix_v[:, c], cache_v[b, slots, c]])
                if not len(k):
                    continue
                with np.errstate(invalid="ignore", over="ignore"):
                    s = scale * (k @ q[b, t, h])
                    top = s.max()
                    if top == -np.inf:
                        continue
                    e = np.exp(s - top)
                    total = e.sum()
                    p = e / total
                    out[b, t, h] = p @ v
                    abs_out[b, t, h] = p @ np.abs(v)
                    lse[b, t, h] = top + np.log(total)
                    abs_score[b, t, h] = abs(scale) * (np.abs(k) @ np.abs(q[b, t, h])).max()
                    added[b, c, slots] += p[P:]
    return {"out": out, "lse": lse, "abs_out": abs_out, "abs_score": abs_score, "added": added,
            "weight": None if weight is None else weight + added}


def insert(cache_k, cache_v, weight, age, lens, k_new, v_new, pos, budget, recent, n_new=None):
    """Copies of (cache_k, cache_v, weight, age, lens) after the insertion; arrays of any dtype."""
    ck, cv, w, a, ln = (np.array(x) for x in (cache_k, cache_v, weight, age, lens))
    B, cap, Hk = ck.shape[:3]
    T = 0 if k_new is None else k_new.shape[1]
    for b in range(B):
        n = T if n_new is None else min(max(int(n_new[b]), 0), T)
        old = min(max(int(lens[b]), 0), cap)
        new_len = min(old + n, budget)
        for c in range(Hk):
            def order(j):
                x = float(weight[b, c, j])
                if age[b, c, j] >= pos[b] + n - recent:
                    return (1, 0.0, j)
                return (0, -math.inf, -1e18 + j) if x != x else (0, x, j)
            # (a NaN weight precedes even -infinity: its third component is negative)
            evicted = set(sorted(range(old), key=order)[:old + n - new_len])
            movers = [("old", j) for j in range(new_len, old) if j not in evicted]
            movers += [("new", t) for t in range(n)]
            free = [j for j in range(new_len) if j in evicted or j >= old]
            assert len(movers) == len(free)
            for (kind, j), dst in zip(movers, free):
                if kind == "old":
                    ck[b, dst, c], cv[b, dst, c] = cache_k[b, j, c], cache_v[b, j, c]
                    w[b, c, dst], a[b, c, dst] = weight[b, c, j], age[b, c, j]
                else:
                    ck[b, dst, c], cv[b, dst, c] = k_new[b, j, c], v_new[b, j, c]
                    w[b, c, dst], a[b, c, dst] = 0.0, pos[b] + j
        ln[b] = new_len
    return ck, cv, w, a, ln


def truncate(cache_k, cache_v, weight, age, lens, pos):
    """Copies of (cache_k, cache_v, weight, age, lens) after the entries of age ``pos`` or more have left."""
    ck, cv, w, a, ln = (np.array(x) for x in (cache_k, cache_v, weight, age, lens))
    B, cap, Hk = ck.shape[:3]
    for b in range(B):
        old = min(max(int(lens[b]), 0), cap)
        gone = max(int((age[b, c, :old] >= pos[b]).sum()) for c in range(Hk))
        for c in range(Hk):
            def order(j):
                x = float(weight[b, c, j])
                if age[b, c, j] >= pos[b]:
                    return (0, 0.0, j)
                return (1, 0.0, j) if x != x else (2, x, j)
            out = set(sorted(range(old), key=order)[:gone])
            movers = [j for j in range(old - gone, old) if j not in out]
            free = [j for j in range(old - gone) if j in out]
            assert len(movers) == len(free)
            for j, dst in zip(movers, free):
                ck[b, dst, c], cv[b, dst, c] = cache_k[b, j, c], cache_v[b, j, c]
                w[b, c, dst], a[b, c, dst] = weight[b, c, j], age[b, c, j]
        ln[b] = old - gone
    return ck, cv, w, a, ln


def policy_loss(logits, allowed, actions, old_logp, advantages, ref_logp=None, weight=None,
                clip_low=0.2, clip_high=0.2, kl_coef=0.0, temperature=1.0):
    """float64 ``logits`` [N][V]; ``allowed`` bool [N][V] (a row of False: inactive).  Returns
    (loss [N], logp [N], dlogits [N][V])."""
    N, V = logits.shape
    loss, logp, grad = np.zeros(N), np.full(N, -np.inf), np.zeros((N, V))
    for i in range(N):
        a = int(actions[i])
        if not 0 <= a < V or not allowed[i, a] or logits[i, a] == -np.inf:
            continue
        with np.errstate(invalid="ignore", over="ignore"):
            z = np.where(allowed[i], logits[i] / temperature, -np.inf)
            top = z.max()
            e = np.where(allowed[i], np.exp(z - top), 0.0)
            p = e / e.sum()
            lp = z[a] - top - np.log(e.sum())
            logp[i] = lp
            w = 1.0 if weight is None else float(weight[i])
            if w == 0.0:
                continue
            r = np.exp(lp - old_logp[i])
            adv = float(advantages[i])
            held = r if r != r else min(max(r, 1.0 - clip_low), 1.0 + clip_high)
            x, g = -min(r * adv, held * adv), -r * adv
            if held * adv < r * adv:
                g = 0.0
            if ref_logp is not None:
                d = ref_logp[i] - lp
                x += kl_coef * (np.exp(d) - d - 1.0)
                g += kl_coef * (1.0 - np.exp(d))
            loss[i] = w * x
            grad[i] = np.where(allowed[i], -w * g / temperature * p, 0.0)
            grad[i, a] += w * g / temperature
    return loss, logp, grad
