"""The operators around the constrained decoding step, as measured cases.

Three operators that a batch of constrained rows needs next to ``cstr_step``:

- ``attention``: attention of a batch whose rows share a long prompt, each row with its own
  cache of later tokens (``cstr_cache_attention``);
- ``insert``: the new tokens' keys and values enter the rows' caches, and rows over their
  budget lose the entries with the least accumulated attention weight (``cstr_cache_insert``);
- ``loss``: the clipped policy loss with a KL term over the constrained distribution, with the
  gradient of the logits (``cstr_policy_loss``).

``run`` computes them in plain torch operations, or through the library where ``own`` is true.
"""

import math

import numpy as np
import torch

own = False
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ---------------------------------------------------------------- cases

def _attention(name, batch, tokens, heads, kv_heads, dim, prefix, cap, dtype, masked):
    return {"op": "attention", "name": name, "batch": batch, "tokens": tokens, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "prefix": prefix, "cap": cap, "dtype": dtype,
            "masked": masked}


def _insert(name, batch, tokens, kv_heads, dim, cap, budget, recent, dtype):
    return {"op": "insert", "name": name, "batch": batch, "tokens": tokens, "kv_heads": kv_heads,
            "dim": dim, "cap": cap, "budget": budget, "recent": recent, "dtype": dtype}


def _loss(name, rows, vocab, dtype, gradient, reference, constrained):
    return {"op": "loss", "name": name, "rows": rows, "vocab": vocab, "dtype": dtype,
            "gradient": gradient, "reference": reference, "constrained": constrained}


def listed():
    return [
        # an API-call constraint decoded for four users of one short prompt: launch latency
        _attention("attention 4 rows", 4, 1, 8, 8, 64, 1024, 32, "bf16", False),
        # 64 rows answer in JSON after one few-shot prompt, half-way through their 256 tokens
        _attention("attention 64 rows", 64, 1, 32, 8, 128, 4096, 256, "bf16", False),
        # the same batch verifying four drafted tokens a row: causal among the new tokens, odd prompt
        _attention("attention 64 rows, drafts", 64, 5, 32, 8, 128, 8191, 300, "f16", True),
        # few rows over a very long document: the prompt's keys and values have to be streamed
        _attention("attention 6 rows, long prompt", 6, 1, 16, 4, 128, 65000, 512, "bf16", False),
        # a full serving batch, long prompt and long answers
        _attention("attention 512 rows", 512, 1, 32, 8, 128, 16384, 1024, "bf16", False),
        # the new token of four rows, nothing evicted yet or one entry a row: launch latency
        _insert("insert 4 rows", 4, 1, 8, 64, 64, 48, 16, "bf16"),
        # steady state of a full batch: every row replaces its least used entry
        _insert("insert 512 rows", 512, 1, 8, 128, 1024, 1000, 128, "bf16"),
        # a tool's answer of up to 256 tokens enters each row's cache at once
        _insert("insert 64 rows, long input", 64, 256, 8, 128, 2304, 2048, 300, "bf16"),
        # 32 tokens each of four API calls
        _loss("loss 128 x 1024", 128, 1024, "f32", True, True, True),
        # a batch of flat JSON objects, bf16 logits, trained without a reference model
        _loss("loss 2048 x 32000", 2048, 32000, "bf16", True, False, True),
        # scoring alone (no gradient) of the 128,256-token vocabulary, unconstrained
        _loss("score 300 x 128256", 300, 128256, "f32", False, True, False),
        # one micro-batch over the largest vocabulary
        _loss("loss 512 x 256000", 512, 256000, "f32", True, True, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return w["bytes"] / 6.5e12 + w["flops"] / 1.6e15


def draw(rng):
    kind = rng.choice(["attention", "attention", "insert", "loss"])
    while True:
        if kind == "attention":
            kv_heads, group = rng.choice([(1, 8), (2, 8), (4, 4), (4, 7), (8, 4), (8, 1), (16, 1), (8, 8)])
            tokens = rng.choice([1, 1, 1, _log(rng, 2, 9)])
            case = _attention("", _log(rng, 1, 512), tokens, kv_heads * group, kv_heads,
                              rng.choice([64, 80, 96, 128, 128]), _log(rng, 1, 65536),
                              max(tokens, _log(rng, 1, 2048)), rng.choice(["bf16", "f16"]),
                              tokens > 1 or rng.random() < 0.3)
            top = 3.5e-4
        elif kind == "insert":
            cap = _log(rng, 8, 4096)
            tokens = min(rng.choice([1, 1, _log(rng, 2, 400)]), max(1, cap // 2))
            budget = max(tokens, int(cap * rng.uniform(0.6, 1.0)))
            case = _insert("", _log(rng, 1, 512), tokens, rng.choice([1, 2, 4, 8, 16]),
                           rng.choice([64, 80, 128]), cap, budget,
                           int(budget * rng.uniform(0.0, 0.5)), rng.choice(["bf16", "f16"]))
            top = 1.1e-5
        else:
            case = _loss("", _log(rng, 1, 4096), _log(rng, 600, 256000), rng.choice(["f32", "bf16"]),
                         rng.random() < 0.7, rng.random() < 0.6, rng.random() < 0.7)
            top = 1.6e-4
        if _cost(case) <= top:
            del case["name"]
            return case


def work(case):
    """Each input read once, each output written once (expected lengths)."""
    if case["op"] == "attention":
        b, t, hq, hk, d = (case[k] for k in ("batch", "tokens", "heads", "kv_heads", "dim"))
        slots = 0.75 * b * case["cap"]
        kv = (case["prefix"] + slots) * hk * d * 2 * 2
        rows = b * t * hq
        return {"bytes": kv + rows * d * 2 * 2 + rows * 4 + slots * hk * (12 if case["masked"] else 8),
                "flops": 4.0 * d * hq * t * (b * case["prefix"] + slots)}
    if case["op"] == "insert":
        b, t, hk, d = (case[k] for k in ("batch", "tokens", "kv_heads", "dim"))
        new = b * (t + 1) / 2
        old = b * 0.9 * case["budget"]
        return {"bytes": old * hk * 8 + new * hk * (d * 2 * 2 * 2 + 8), "flops": 0.0}
    n, v = case["rows"], case["vocab"]
    e = 4 if case["dtype"] == "f32" else 2
    return {"bytes": float(n) * v * (e * (2 if case["gradient"] else 1)
                                     + (0.125 if case["constrained"] else 0.0)) + 32.0 * n,
            "flops": float(n) * v * 4}


# --------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 2 + 1)
    return g


def _normal(g, shape, dtype, sigma=1.0):
    out = torch.empty(shape, dtype=dtype, device=DEV)
    return out.normal_(0.0, sigma, generator=g)


def _ranks(g, lens, heads, cap):
    """Ages 0..len-1 in a seeded order over each row's slots: a cache that has evicted before."""
    b = lens.numel()
    key = torch.rand((b, heads, cap), device=DEV, generator=g)
    slot = torch.arange(cap, device=DEV)
    key = torch.where(slot < lens.view(b, 1, 1), key, 2.0)
    order = key.argsort(dim=-1)
    return torch.empty_like(order).scatter_(-1, order, slot.expand_as(order)).to(torch.int32)


def _weights(g, shape):
    """Accumulated attention weights: a few heavy entries, many light ones, some untouched."""
    u = torch.rand(shape, device=DEV, generator=g)
    return torch.where(u < 0.03, 0.0, 2.0 * u ** 8 + 0.01 * u)


def _prepare_attention(case, g):
    b, t, hq, hk, d = (case[k] for k in ("batch", "tokens", "heads", "kv_heads", "dim"))
    p, cap, dt = case["prefix"], case["cap"], TYPES[case["dtype"]]
    n_query = torch.randint(1, t + 1, (b,), device=DEV, generator=g, dtype=torch.int32)
    n_query[0] = t
    lens = torch.randint(cap // 2, cap + 1, (b,), device=DEV, generator=g, dtype=torch.int32)
    lens = torch.maximum(lens, n_query)
    s = {
        "q": _normal(g, (b, t, hq, d), dt, 1.5),
        "prefix_k": _normal(g, (p, hk, d), dt), "prefix_v": _normal(g, (p, hk, d), dt),
        "cache_k": _normal(g, (b, cap, hk, d), dt), "cache_v": _normal(g, (b, cap, hk, d), dt),
        "weight": _weights(g, (b, hk, cap)), "lens": lens, "age": _ranks(g, lens, hk, cap),
        "pos": lens - n_query if case["masked"] else None,
        "n_query": n_query if t > 1 else None,
        "out": torch.empty((b, t, hq, d), dtype=dt, device=DEV),
        "lse": torch.empty((b, t, hq), dtype=torch.float32, device=DEV),
    }
    return s


def _prepare_insert(case, g):
    b, t, hk, d = (case[k] for k in ("batch", "tokens", "kv_heads", "dim"))
    cap, budget, dt = case["cap"], case["budget"], TYPES[case["dtype"]]
    full = torch.rand((b,), device=DEV, generator=g) < 0.8
    some = torch.randint(budget // 4, budget + 1, (b,), device=DEV, generator=g)
    lens = torch.where(full, budget, some).to(torch.int32)
    pos = lens + torch.randint(0, 500, (b,), device=DEV, generator=g, dtype=torch.int32)
    return {
        "cache_k": _normal(g, (b, cap, hk, d), dt), "cache_v": _normal(g, (b, cap, hk, d), dt),
        "weight": _weights(g, (b, hk, cap)), "lens": lens, "pos": pos,
        "age": _ranks(g, lens, hk, cap) + (pos - lens).view(b, 1, 1),
        "k_new": _normal(g, (b, t, hk, d), dt), "v_new": _normal(g, (b, t, hk, d), dt),
        "n_new": torch.randint(1, t + 1, (b,), device=DEV, generator=g, dtype=torch.int32)
        if t > 1 else None,
    }


def _automaton(case, seed):
    """A byte DFA in which most states allow most bytes (free text) and some few (keywords),
    and a vocabulary of strings of one to four bytes; the first 256 are the single bytes."""
    rng = np.random.default_rng(seed)
    states, v = 48, case["vocab"]
    trans = rng.integers(0, states, (states, 256)).astype(np.int32)
    keep = np.where(np.arange(states) % 4 == 3, 0.05, 0.9)[:, None]
    trans[rng.random((states, 256)) >= keep] = -1
    trans[:, 65] = rng.integers(0, states, states)
    length = rng.integers(1, 5, v)
    text = rng.integers(0, 256, (v, 4)).astype(np.uint8)
    length[:256] = 1
    text[:256, 0] = np.arange(256)
    return trans, length, text


def _allowed(trans, length, text):
    """Tokens that each state allows, by walking every token's bytes: bool [states][vocab]."""
    states, v = trans.shape[0], length.size
    t = torch.from_numpy(np.vstack([trans, np.full((1, 256), -1, np.int32)])).to(DEV).long()
    t[t < 0] = states
    byte = torch.from_numpy(text).to(DEV).long()
    last = torch.from_numpy(length).to(DEV)
    at = torch.arange(states, device=DEV)[:, None].expand(states, v)
    for i in range(text.shape[1]):
        at = torch.where(last > i, t[at, byte[:, i]], at)
    return at < states


def _prepare_loss(case, g, seed):
    n, v, dt = case["rows"], case["vocab"], TYPES[case["dtype"]]
    s = {"logits": _normal(g, (n, v), dt, 2.0), "tables": None, "states": None, "allowed": None}
    if case["constrained"]:
        trans, length, text = _automaton(case, seed)
        s["allowed"] = _allowed(trans, length, text)
        s["states"] = torch.randint(0, trans.shape[0], (n,), device=DEV, generator=g, dtype=torch.int32)
        s["states"][torch.rand((n,), device=DEV, generator=g) < 0.03] = -1     # finished rows
    if own:
        from paper_2407_08103_b200 import cstr
        if case["constrained"]:
            offsets = np.concatenate([[0], np.cumsum(length)])
            flat = text[np.arange(4)[None, :] < length[:, None]]
            dfa = cstr.cstr_load_dfa(trans, np.ones(trans.shape[0], np.uint8), 0)
            s["tables"] = [cstr.cstr_build_token_table(dfa, flat, offsets)]
    # the sampled tokens, and their log probabilities under the policy that sampled them
    action, logp = [], []
    for lo in range(0, n, 256):
        x = s["logits"][lo:lo + 256].float()
        if s["allowed"] is not None:
            x = x.masked_fill(~s["allowed"][s["states"][lo:lo + 256].clamp(min=0).long()], -math.inf)
        u = torch.rand(x.shape, device=DEV, generator=g).clamp_(min=1e-20)
        a = (x - torch.log(-torch.log(u))).argmax(dim=1)
        action.append(a)
        logp.append(x.gather(1, a[:, None])[:, 0] - x.logsumexp(dim=1))
    logp = torch.cat(logp)
    s["actions"] = torch.cat(action).to(torch.int32)
    s["old_logp"] = logp + _normal(g, (n,), torch.float32, 0.2)
    s["ref_logp"] = logp + _normal(g, (n,), torch.float32, 0.3) if case["reference"] else None
    s["advantages"] = _normal(g, (n,), torch.float32)
    s["weight"] = torch.where(torch.rand((n,), device=DEV, generator=g) < 0.1, 0.0, 1.0 / n)
    s["kl_coef"] = 0.05 if case["reference"] else 0.0
    s["loss"] = torch.empty(n, dtype=torch.float32, device=DEV)
    s["logp"] = torch.empty(n, dtype=torch.float32, device=DEV)
    s["dlogits"] = torch.empty_like(s["logits"]) if case["gradient"] else None
    return s


def prepare(case, seed):
    g = _gen(seed)
    if case["op"] == "loss":
        s = _prepare_loss(case, g, seed)
    else:
        s = _prepare_attention(case, g) if case["op"] == "attention" else _prepare_insert(case, g)
        if own:
            from paper_2407_08103_b200 import cstr
            s["cache"] = cstr.cstr_cache_create(
                s["cache_k"], s["cache_v"], s["lens"], case.get("heads", case["kv_heads"]),
                prefix_k=s.get("prefix_k"), prefix_v=s.get("prefix_v"), weight=s["weight"],
                age=s["age"], max_tokens=case["tokens"])
    s["case"] = case
    return s


# ------------------------------------------------------------------ run

def _run_attention(s, case):
    if own:
        from paper_2407_08103_b200 import cstr
        cstr.cstr_cache_attention(s["cache"], s["q"], s["out"], pos=s["pos"], n_query=s["n_query"],
                                  lse_out=s["lse"], accumulate=True)
        return s["out"], s["lse"], s["weight"]
    b, t, hq, hk, d = (case[k] for k in ("batch", "tokens", "heads", "kv_heads", "dim"))
    p, cap, group = case["prefix"], case["cap"], hq // hk
    q = s["q"].float().view(b, t, hk, group, d) / math.sqrt(d)
    shared = q.permute(2, 0, 1, 3, 4).reshape(hk, b * t * group, d)
    sp = shared @ s["prefix_k"].float().permute(1, 2, 0)                     # [hk][b t g][p]
    sp = sp.view(hk, b, t * group, p).transpose(0, 1)
    each = q.permute(0, 2, 1, 3, 4).reshape(b, hk, t * group, d)
    sc = each @ s["cache_k"].float().permute(0, 2, 3, 1)                     # [b][hk][t g][cap]
    slot, at = torch.arange(cap, device=DEV), torch.arange(t, device=DEV)
    seen = (slot < s["lens"].view(b, 1, 1, 1)).expand(b, hk, t, cap)
    if s["pos"] is not None:
        seen = seen & (s["age"].view(b, hk, 1, cap) <= (s["pos"].view(b, 1) + at).view(b, 1, t, 1))
    sc = sc.view(b, hk, t, group, cap).masked_fill(~seen.unsqueeze(3), -math.inf)
    sc = sc.view(b, hk, t * group, cap)
    top = torch.maximum(sp.amax(-1), sc.amax(-1)).unsqueeze(-1)
    sp, sc = torch.exp(sp - top), torch.exp(sc - top)
    total = sp.sum(-1, keepdim=True) + sc.sum(-1, keepdim=True)
    pv = sp.transpose(0, 1).reshape(hk, b * t * group, p) @ s["prefix_v"].float().transpose(0, 1)
    out = pv.view(hk, b, t * group, d).transpose(0, 1) + sc @ s["cache_v"].float().transpose(1, 2)
    out = (out / total).view(b, hk, t, group, d).transpose(1, 2).reshape(b, t, hq, d)
    lse = (top + torch.log(total)).view(b, hk, t, group).transpose(1, 2).reshape(b, t, hq)
    add = (sc / total).view(b, hk, t, group, cap)
    if s["n_query"] is not None:
        real = at < s["n_query"].view(b, 1)
        out = out.masked_fill(~real.view(b, t, 1, 1), 0.0)
        lse = lse.masked_fill(~real.view(b, t, 1), -math.inf)
        add = add.masked_fill(~real.view(b, 1, t, 1, 1), 0.0)
    s["weight"].add_(add.sum((2, 3)))
    return out.to(s["q"].dtype), lse, s["weight"]


def _run_insert(s, case):
    if own:
        from paper_2407_08103_b200 import cstr
        cstr.cstr_cache_insert(s["cache"], s["k_new"], s["v_new"], s["pos"], case["budget"],
                               case["recent"], n_new=s["n_new"])
        return s["cache_k"], s["cache_v"], s["weight"], s["age"], s["lens"]
    b, t, hk, d = (case[k] for k in ("batch", "tokens", "kv_heads", "dim"))
    cap, budget = case["cap"], case["budget"]
    n = s["n_new"] if s["n_new"] is not None else torch.full_like(s["lens"], t)
    n, old, pos = (x.view(b, 1, 1).long() for x in (n, s["lens"], s["pos"]))
    new_len = (old + n).clamp(max=budget)
    slot = torch.arange(cap, device=DEV).expand(b, hk, cap)
    # eviction order of the old entries: (protected, weight, slot); equal values by slot
    bits = s["weight"].view(torch.int32).long()
    key = torch.where(bits < 0, -(bits & 0x7fffffff), bits)
    key = torch.where(s["weight"].isnan(), -(1 << 31), key)
    key = key + ((s["age"] >= pos + n - case["recent"]).long() << 33)
    key = key.masked_fill(slot >= old, 1 << 40)
    order = key.argsort(dim=-1, stable=True)
    rank = torch.empty_like(order).scatter_(-1, order, slot)
    gone = rank < old + n - budget
    # entries 0..cap-1 are the old slots, cap.. the new tokens.  Old entries that stay but lie past
    # the new length, then the new tokens, take the free slots (evicted or past the old length) in
    # ascending order
    entry = torch.arange(cap + t, device=DEV).expand(b, hk, cap + t)
    live = torch.where(entry < cap, entry < old, entry - cap < n)
    live[..., :cap] &= ~gone
    moving = live & ((entry >= cap) | (entry >= new_len))
    free = (slot < new_len) & (gone | (slot >= old))
    pick = torch.sort((~moving).to(torch.uint8), dim=-1, stable=True).indices[..., :cap]
    place = torch.sort((~free).to(torch.uint8), dim=-1, stable=True).indices
    m = min(pick.shape[-1], place.shape[-1])
    fill = slot[..., :m] < free.sum(-1, keepdim=True)
    pick, place = pick[..., :m], place[..., :m]
    row, head = (x.expand(b, hk, m)[fill] for x in
                 (torch.arange(b, device=DEV).view(b, 1, 1), torch.arange(hk, device=DEV).view(1, hk, 1)))
    src, dst = pick[fill], place[fill]
    is_new = src >= cap
    token, kept = (src - cap).clamp(min=0), src.clamp(max=cap - 1)
    for_k = torch.where(is_new[:, None], s["k_new"][row, token, head], s["cache_k"][row, kept, head])
    for_v = torch.where(is_new[:, None], s["v_new"][row, token, head], s["cache_v"][row, kept, head])
    weight = torch.where(is_new, 0.0, s["weight"][row, head, kept])
    age = torch.where(is_new, (pos[row, 0, 0] + token).to(torch.int32), s["age"][row, head, kept])
    s["cache_k"][row, dst, head], s["cache_v"][row, dst, head] = for_k, for_v
    s["weight"][row, head, dst], s["age"][row, head, dst] = weight, age
    s["lens"].copy_(new_len.view(b))
    return s["cache_k"], s["cache_v"], s["weight"], s["age"], s["lens"]


def _run_loss(s, case):
    if own:
        from paper_2407_08103_b200 import cstr
        cstr.cstr_policy_loss(s["tables"], s["logits"], s["states"], s["actions"], s["old_logp"],
                              s["advantages"], s["loss"], s["logp"], ref_logp=s["ref_logp"],
                              weight=s["weight"], dlogits=s["dlogits"], clip_low=0.2,
                              clip_high=0.28, kl_coef=s["kl_coef"])
        return [s["loss"], s["logp"]] + ([s["dlogits"]] if case["gradient"] else [])
    x = s["logits"].float()
    valid = torch.ones_like(s["actions"], dtype=torch.bool)
    if s["allowed"] is not None:
        valid = s["states"] >= 0
        x = torch.where(s["allowed"][s["states"].clamp(min=0).long()], x, -math.inf)
    action = s["actions"].long()[:, None]
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(1, keepdim=True)
    logp = (x.gather(1, action) - top - torch.log(total))[:, 0]
    valid = valid & (logp > -math.inf)
    ratio, adv = torch.exp(logp - s["old_logp"]), s["advantages"]
    plain, clipped = ratio * adv, ratio.clamp(1.0 - 0.2, 1.0 + 0.28) * adv
    loss, g = -torch.minimum(plain, clipped), -torch.where(plain <= clipped, plain, 0.0)
    if s["ref_logp"] is not None:
        diff = s["ref_logp"] - logp
        loss = loss + s["kl_coef"] * (torch.exp(diff) - diff - 1.0)
        g = g + s["kl_coef"] * (1.0 - torch.exp(diff))
    loss = torch.where(valid, s["weight"] * loss, 0.0)
    g = torch.where(valid, s["weight"] * g, 0.0)
    logp = torch.where(valid, logp, -math.inf)
    if not case["gradient"]:
        return [loss, logp]
    grad = torch.where(valid[:, None], e * (-g[:, None] / total), 0.0)
    grad.scatter_add_(1, action, g[:, None])
    return [loss, logp, grad.to(s["logits"].dtype)]


def run(state):
    case = state["case"]
    return {"attention": _run_attention, "insert": _run_insert, "loss": _run_loss}[case["op"]](state, case)


# ---------------------------------------------------------------- exact

def _exact_attention(s, case):
    """One (row, kv head) at a time over its own list of visible keys, in 64 bits."""
    b, t, hq, hk, d = (case[k] for k in ("batch", "tokens", "heads", "kv_heads", "dim"))
    group, p, cap = hq // hk, case["prefix"], case["cap"]
    if 4.0 * b * t * hq * (p + cap) * d > 4e11:
        return None
    f8 = torch.float64
    out = torch.zeros((b, t, hq, d), dtype=f8, device=DEV)
    lse = torch.full((b, t, hq), -math.inf, dtype=f8, device=DEV)
    weight = s["weight"].to(f8)
    lens = s["lens"].tolist()
    queries = s["n_query"].tolist() if s["n_query"] is not None else [t] * b
    for c in range(hk):
        kp, vp = s["prefix_k"][:, c].to(f8), s["prefix_v"][:, c].to(f8)
        for r in range(b):
            n, m = lens[r], queries[r]
            k = torch.cat([kp, s["cache_k"][r, :n, c].to(f8)])
            v = torch.cat([vp, s["cache_v"][r, :n, c].to(f8)])
            q = s["q"][r, :m, c * group:(c + 1) * group].to(f8)
            z = torch.einsum("tgd,xd->tgx", q, k) * d ** -0.5
            if s["pos"] is not None:
                late = s["age"][r, c, :n][None] > s["pos"][r] + torch.arange(m, device=DEV)[:, None]
                z[:, :, p:] = z[:, :, p:].masked_fill(late[:, None], -math.inf)
            l = torch.logsumexp(z, dim=-1)
            w = torch.exp(z - l[..., None])
            out[r, :m, c * group:(c + 1) * group] = torch.einsum("tgx,xd->tgd", w, v)
            lse[r, :m, c * group:(c + 1) * group] = l
            weight[r, c, :n] += w[:, :, p:].sum((0, 1))
    return out, lse, weight


def _exact_loss(s, case):
    """A few rows at a time in 64 bits, the gradient from the softmax's derivative."""
    n, v = case["rows"], case["vocab"]
    f8 = torch.float64
    loss = torch.zeros(n, dtype=f8, device=DEV)
    logps = torch.full((n,), -math.inf, dtype=f8, device=DEV)
    grad = torch.zeros((n, v), dtype=f8, device=DEV) if case["gradient"] else None
    for lo in range(0, n, 64):
        at = slice(lo, min(n, lo + 64))
        x = s["logits"][at].to(f8)
        ok = torch.ones(x.shape[0], dtype=torch.bool, device=DEV)
        if s["states"] is not None:
            ok = s["states"][at] >= 0
            x = x.masked_fill(~s["allowed"][s["states"][at].clamp(min=0).long()], -math.inf)
        logq = torch.log_softmax(x, dim=1)
        a = s["actions"][at].long()
        lp = logq[torch.arange(x.shape[0], device=DEV), a]
        ok &= lp > -math.inf
        adv, w = s["advantages"][at].to(f8), s["weight"][at].to(f8)
        r = torch.exp(lp - s["old_logp"][at].to(f8))
        c = torch.clamp(r, 0.8, 1.28)
        inside = ~(((adv > 0) & (r > 1.28)) | ((adv < 0) & (r < 0.8)))
        one = -torch.minimum(r * adv, c * adv)
        d = torch.where(inside, -r * adv, 0.0)
        if s["ref_logp"] is not None:
            k = torch.exp(s["ref_logp"][at].to(f8) - lp)
            one = one + s["kl_coef"] * (k - torch.log(k) - 1.0)
            d = d + s["kl_coef"] * (1.0 - k)
        loss[at] = torch.where(ok, one * w, 0.0)
        logps[at] = torch.where(ok, lp, -math.inf)
        if grad is not None:
            d = torch.where(ok, d * w, 0.0)[:, None]
            hot = torch.zeros_like(x).scatter_(1, a[:, None], 1.0)
            grad[at] = torch.where(ok[:, None], d * (hot - torch.exp(logq)), 0.0)
    return [loss, logps] + ([grad] if grad is not None else [])


def exact(case, seed):
    global own
    before, own = own, False
    try:
        if case["op"] == "insert":
            return None                 # copies and whole numbers: nothing is computed
        g = _gen(seed)
        if case["op"] == "attention":
            return _exact_attention(_prepare_attention(case, g), case)
        return _exact_loss(_prepare_loss(case, g, seed), case)
    finally:
        own = before
