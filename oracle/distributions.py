"""Plain statements in 64 bits of the operators over whole constrained distributions: a token under
temperature, top-k, top-p and min-p from one uniform number, the most likely tokens, and the divergence
from a teacher's record.  Test infrastructure only; loops over rows, no code shared with the GPU path."""

from __future__ import annotations

import numpy as np


def order(x, allowed):
    """Allowed ids whose logits are neither NaN nor -infinity, most likely first, equal ones by id."""
    ids = [v for v in np.flatnonzero(allowed) if x[v] == x[v] and x[v] != -np.inf]
    return sorted(ids, key=lambda v: (-x[v], v))


def weights(x, ids, temperature):
    """exp((x - max) / temperature) of the ordered ids; infinite logits share everything."""
    top = x[ids[0]]
    if top == np.inf:
        return np.array([1.0 if x[v] == np.inf else 0.0 for v in ids])
    return np.exp((x[ids] - top) / temperature)


def sample_row(x, allowed, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, logp, kept) of one float64 row."""
    bad = (-1, -np.inf, 0.0)
    if any(np.isnan([u, temperature, top_p, min_p])) or temperature < 0 or np.isinf(temperature) \
            or 0 < temperature < 4.3e-39:
        return bad
    ids = order(x, allowed)
    if not ids:
        low = [v for v in np.flatnonzero(allowed) if x[v] == -np.inf]
        return (int(low[0]), -np.inf, 0.0) if low else bad
    if temperature == 0:
        return int(ids[0]), 0.0, 1.0
    w = weights(x, ids, temperature)
    total = w.sum()
    n = len(ids)
    if top_k > 0:
        n = min(n, top_k)
    if min_p > 0:
        if x[ids[0]] == np.inf:
            n = min(n, int((w > 0).sum()))
        else:
            n = min(n, sum((x[v] - x[ids[0]]) / temperature >= np.log(min_p) for v in ids))
    n = max(n, 1)
    if top_p < 1:
        upto = np.cumsum(w[:n])
        n = max(1, int((np.concatenate([[0.0], upto[:-1]]) < top_p * upto[-1]).sum()))
    kept = sorted(zip(ids[:n], w[:n]))
    upto = np.cumsum([k[1] for k in kept])
    u = min(max(u, 0.0), 1.0 - 2.0 ** -24)
    i = int((upto <= u * upto[-1]).sum())
    token, mass = kept[min(i, len(kept) - 1)]
    return int(token), np.log(mass / total), upto[-1] / total


def sample(x, allowed, uniform, temperature=None, top_k=None, top_p=None, min_p=None):
    """(tokens, logp, kept) of float64 rows; None: the setting is not used."""
    rows = []
    for i in range(x.shape[0]):
        kw = {k: a[i] for k, a in (("temperature", temperature), ("top_k", top_k), ("top_p", top_p), ("min_p", min_p))
              if a is not None}
        rows.append(sample_row(x[i], allowed[i], float(uniform[i]), **kw))
    return tuple(np.array(c) for c in zip(*rows))


def top(x, allowed, n, temperature=1.0):
    """(ids [N][n], logp [N][n], lse [N])."""
    N = x.shape[0]
    ids, logp, lse = np.full((N, n), -1), np.full((N, n), -np.inf), np.full(N, -np.inf)
    for i in range(N):
        mine = order(x[i], allowed[i])
        if not mine:
            continue
        w = weights(x[i], mine, temperature)
        with np.errstate(divide="ignore"):
            lse[i] = x[i][mine[0]] / temperature + np.log(w.sum())
            k = min(n, len(mine))
            ids[i, :k] = mine[:k]
            logp[i, :k] = np.log(w[:k] / w.sum()) if x[i][mine[0]] == np.inf \
                else (x[i][mine[:k]] - x[i][mine[0]]) / temperature - np.log(w.sum())
    return ids, logp, lse


DROP, RENORM, LUMP = 0, 1, 2


def distill(x, allowed, ids, teacher, tail, weight=None, temperature=1.0):
    """(loss [N], dlogits [N][V]) of float64 logits ``x``; ``allowed`` bool (a row of False: inactive);
    ``ids`` / ``teacher`` [N][k].  The gradient comes from the events' probabilities, not from the loss."""
    N, V = x.shape
    loss, grad = np.zeros(N), np.zeros((N, V))
    for i in range(N):
        w = 1.0 if weight is None else float(weight[i])
        z = np.where(allowed[i], x[i] / temperature, -np.inf)
        if w == 0.0 or not allowed[i].any() or (z == -np.inf).all():
            continue
        with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
            top = np.nanmax(np.where(np.isnan(z), -np.inf, z))
            e = np.where(z == -np.inf, 0.0, np.exp(z - top))
            q = e / e.sum()
            logq = z - top - np.log(e.sum())
            real = [(v, g) for v, g in zip(ids[i], teacher[i]) if 0 <= v < V and g != -np.inf]
            entries = [(v, g) for v, g in real if z[v] != -np.inf]
            scale = max([g for _, g in entries], default=0.0) if tail == RENORM else 0.0
            t = np.array([np.exp(g - scale) for _, g in entries])
            logt = np.array([g - scale for _, g in entries])
            if tail == RENORM and len(t):
                logt, t = logt - np.log(t.sum()), t / t.sum()
            value = float(sum(t[j] * (logt[j] - logq[v]) for j, (v, _) in enumerate(entries)))
            wanted = np.zeros(V)
            for j, (v, _) in enumerate(entries):
                wanted[v] += t[j]
            if tail == LUMP:
                inside = np.zeros(V, bool)
                inside[[v for v, _ in real]] = True
                rest = np.where(inside, -np.inf, z)
                r = max(0.0, 1.0 - sum(np.exp(g) for _, g in real)) if not any(np.isnan(g) for _, g in real) else np.nan
                if not (rest == -np.inf).all() and r != 0.0:
                    low = np.nanmax(np.where(np.isnan(rest), -np.inf, rest))
                    er = np.where(rest == -np.inf, 0.0, np.exp(rest - low))
                    value += r * (np.log(r) - (np.log(er.sum() / e.sum()) + (low - top)))
                    wanted += r * er / er.sum()
            loss[i] = w * value
            grad[i] = np.where(z == -np.inf, 0.0, w / temperature * (q * wanted.sum() - wanted))
    return loss, grad
