"""Sampling and distillation around the constrained decoding step, as measured cases.

Three operators that a batch of constrained rows needs next to ``cstr_step`` and ``cstr_policy_loss``:

- ``sample``: a token of each row's constrained distribution with temperature, top-k, top-p and min-p
  from one uniform number a row, and the row's next automaton state (``cstr_sample``);
- ``top``: the n most likely allowed tokens of each row with their log probabilities, what an answer's
  ``logprobs`` field or a teacher model's record of a position holds (``cstr_top_logprobs``);
- ``distill``: the divergence of a student's constrained distribution from such records, with the
  gradient of the logits (``cstr_distill_loss``).

``run`` computes them in plain torch operations, or through the library where ``own`` is true.
"""

import math

import numpy as np
import torch

own = False
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
STATES = 48
TAILS = {"drop": 0, "renorm": 1, "lump": 2}


# ---------------------------------------------------------------- cases

def _sample(name, rows, vocab, dtype, cut, constrained):
    return {"op": "sample", "name": name, "rows": rows, "vocab": vocab, "dtype": dtype, "cut": cut,
            "constrained": constrained}


def _top(name, rows, vocab, dtype, n, constrained):
    return {"op": "top", "name": name, "rows": rows, "vocab": vocab, "dtype": dtype, "n": n,
            "constrained": constrained}


def _distill(name, rows, vocab, dtype, n, tail, gradient, constrained):
    return {"op": "distill", "name": name, "rows": rows, "vocab": vocab, "dtype": dtype, "n": n, "tail": tail,
            "gradient": gradient, "constrained": constrained}


def listed():
    return [
        # an API-call constraint decoded for four users: launch latency
        _sample("sample 4 x 1024", 4, 1024, "f32", "k+p", True),
        # a serving batch of JSON answers in which every request brings its own settings, greedy ones among them
        _sample("sample 64 x 32000, mixed", 64, 32000, "bf16", "mixed", True),
        # free text in a nucleus of 0.95, some rows confident, some nearly flat
        _sample("sample 300 x 128256, top-p", 300, 128256, "f32", "p", False),
        # a rollout for training: the whole constrained distribution, temperature alone
        _sample("sample 128 x 128256, plain", 128, 128256, "bf16", "plain", True),
        # a full batch over the largest vocabulary with every cut at once
        _sample("sample 512 x 256000", 512, 256000, "f32", "all", True),
        # the five alternatives that an answer's log probabilities show, for four users
        _top("top 5 of 4 x 1024", 4, 1024, "f32", 5, True),
        # a teacher's record of 2,048 positions, 64 tokens each
        _top("top 64 of 2048 x 32000", 2048, 32000, "bf16", 64, True),
        # the same over the largest vocabulary, longer records
        _top("top 256 of 512 x 256000", 512, 256000, "f32", 256, False),
        # 32 tokens each of four API calls
        _distill("distill 128 x 1024", 128, 1024, "f32", 16, "lump", True, True),
        # a batch of flat JSON objects, bf16 logits, records of 64 with their tail in one bucket
        _distill("distill 2048 x 32000", 2048, 32000, "bf16", 64, "lump", True, True),
        # validation: the loss alone
        _distill("distill value 300 x 128256", 300, 128256, "f32", 100, "drop", False, True),
        # one micro-batch over the largest vocabulary, records of an unconstrained teacher
        _distill("distill 512 x 256000", 512, 256000, "f32", 256, "renorm", True, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["sample", "sample", "top", "distill"])
    while True:
        rows, vocab = _log(rng, 1, 4096), _log(rng, 600, 256000)
        dtype, constrained = rng.choice(["bf16", "f32"]), rng.random() < 0.7
        if op == "sample":
            case = _sample("", rows, vocab, dtype, rng.choice(["k", "p", "min", "k+p", "all", "mixed", "plain"]), constrained)
        elif op == "top":
            case = _top("", rows, vocab, dtype, _log(rng, 1, 256), constrained)
        else:
            case = _distill("", rows, vocab, dtype, _log(rng, 1, 256), rng.choice(list(TAILS)), rng.random() < 0.7, constrained)
        if work(case)["bytes"] <= (1.04e9 if op == "distill" else 5.2e8):
            del case["name"]
            return case


def work(case):
    """Each input read once, each output written once."""
    n, v = case["rows"], case["vocab"]
    e = 4 if case["dtype"] == "f32" else 2
    b = float(n) * v * e + 32.0 * n
    if case["constrained"]:
        b += min(n, STATES) * v / 8
    if case["op"] != "sample":
        b += 8.0 * n * case["n"]
    if case["op"] == "distill" and case["gradient"]:
        b += float(n) * v * e
    return {"bytes": b, "flops": 4.0 * n * v}


# --------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 2 + 1)
    return g


def _normal(g, shape, sigma=1.0):
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(0.0, sigma, generator=g)


def _uniform(g, shape, lo=0.0, hi=1.0):
    return torch.rand(shape, device=DEV, generator=g) * (hi - lo) + lo


def _automaton(case, seed):
    """A byte DFA in which most states allow most bytes (free text) and some few (keywords),
    and a vocabulary of strings of one to four bytes; the first 256 are the single bytes."""
    rng = np.random.default_rng(seed)
    v = case["vocab"]
    trans = rng.integers(0, STATES, (STATES, 256)).astype(np.int32)
    keep = np.where(np.arange(STATES) % 4 == 3, 0.05, 0.9)[:, None]
    trans[rng.random((STATES, 256)) >= keep] = -1
    trans[:, 65] = rng.integers(0, STATES, STATES)
    length = rng.integers(1, 5, v)
    text = rng.integers(0, 256, (v, 4)).astype(np.uint8)
    length[:256] = 1
    text[:256, 0] = np.arange(256)
    return trans, length, text


def _next_states(trans, length, text):
    """State after each token from each state, by walking the tokens' bytes: int32 [states][vocab], -1: none."""
    v = length.size
    t = torch.from_numpy(np.vstack([trans, np.full((1, 256), -1, np.int32)])).to(DEV).long()
    t[t < 0] = STATES
    byte = torch.from_numpy(text).to(DEV).long()
    last = torch.from_numpy(length).to(DEV)
    at = torch.arange(STATES, device=DEV)[:, None].expand(STATES, v)
    for i in range(text.shape[1]):
        at = torch.where(last > i, t[at, byte[:, i]], at)
    return torch.where(at < STATES, at, -1).to(torch.int32)


def _logits(g, n, v):
    """A bulk of unlikely tokens, and 24 likely ones that hold from nearly half to nearly all of the probability."""
    x = _normal(g, (n, v), 1.5)
    top = math.log(v) + 1.125 + _uniform(g, (n, 1), -1.0, 7.0) - 0.35 * torch.arange(24, device=DEV)
    part = v // 24                           # each in a part of the vocabulary of its own
    at = torch.randint(0, part, (n, 24), device=DEV, generator=g) + part * (7 * torch.arange(24, device=DEV) % 24)
    return x.scatter_(1, at, top + _normal(g, (n, 24), 0.3))


def _settings(case, g):
    """Per-row temperature, top_k, top_p, min_p (None: not used)."""
    n, cut = case["rows"], case["cut"]

    def pick(values, dtype):
        t = torch.tensor(values, dtype=dtype, device=DEV)
        return t[torch.randint(0, len(values), (n,), device=DEV, generator=g)]
    f = torch.float32
    if cut == "mixed":
        return dict(temperature=pick([0.0, 0.7, 1.0, 1.0, 1.3], f), top_k=pick([0, 0, 1, 20, 50, 400], torch.int32),
                    top_p=pick([1.0, 1.0, 0.5, 0.9, 0.95], f), min_p=pick([0.0, 0.0, 0.02, 0.1], f))
    return dict(temperature=_uniform(g, (n,), 0.7, 1.2),
                top_k=pick([50], torch.int32) if cut in ("k", "k+p", "all") else None,
                top_p=pick([0.95], f) if cut in ("p", "k+p", "all") else None,
                min_p=pick([0.02], f) if cut in ("min", "all") else None)


def _prepare(case, seed):
    """Inputs, without the library's handles."""
    g = _gen(seed)
    n, v, dt = case["rows"], case["vocab"], TYPES[case["dtype"]]
    s = {"logits": _logits(g, n, v).to(dt), "tables": None, "states": None, "next": None, "case": case}
    if case["constrained"]:
        s["automaton"] = _automaton(case, seed)
        s["next"] = _next_states(*s["automaton"])
        s["states"] = torch.randint(0, STATES, (n,), device=DEV, generator=g, dtype=torch.int32)
        s["states"][torch.rand((n,), device=DEV, generator=g) < 0.03] = -1         # finished rows
    if case["op"] == "sample":
        s.update(_settings(case, g))
        s["uniform"] = torch.rand((n,), device=DEV, generator=g)
        s["states_out"] = torch.empty(n, dtype=torch.int32, device=DEV) if case["constrained"] else None
        s["tokens"] = torch.empty(n, dtype=torch.int32, device=DEV)
        s["logp"], s["kept"] = (torch.empty(n, dtype=torch.float32, device=DEV) for _ in range(2))
    elif case["op"] == "top":
        s["ids"] = torch.empty((n, case["n"]), dtype=torch.int32, device=DEV)
        s["logp"] = torch.empty((n, case["n"]), dtype=torch.float32, device=DEV)
        s["lse"] = torch.empty(n, dtype=torch.float32, device=DEV)
    else:
        ids, logp = [], []
        for lo in range(0, n, 256):          # the teacher agrees with the student up to some noise
            x = s["logits"][lo:lo + 256].float()
            x = x + _normal(g, x.shape, 0.7)
            if case["constrained"] and case["tail"] != "renorm":
                x = x.masked_fill(~_allowed(s, slice(lo, lo + 256)), -math.inf)
            value, at = x.topk(min(case["n"], v), dim=1)
            value = value - torch.logsumexp(x, 1, keepdim=True)
            real = value > -math.inf
            ids.append(torch.where(real, at, -1).to(torch.int32))
            logp.append(torch.where(real, value, -math.inf))
        s["ids"], s["teacher"] = torch.cat(ids), torch.cat(logp)
        s["weight"] = torch.where(torch.rand((n,), device=DEV, generator=g) < 0.1, 0.0, 1.0 / n)
        s["loss"] = torch.empty(n, dtype=torch.float32, device=DEV)
        s["dlogits"] = torch.empty_like(s["logits"]) if case["gradient"] else None
    return s


def prepare(case, seed):
    s = _prepare(case, seed)
    if own and case["constrained"]:
        from paper_2407_08103_b200 import cstr
        trans, length, text = s["automaton"]
        offsets = np.concatenate([[0], np.cumsum(length)])
        flat = text[np.arange(4)[None, :] < length[:, None]]
        dfa = cstr.cstr_load_dfa(trans, np.ones(STATES, np.uint8), 0)
        s["tables"] = [cstr.cstr_build_token_table(dfa, flat, offsets)]
    return s


# ------------------------------------------------------------------ run

def _allowed(s, at=slice(None)):
    """bool [rows][vocab]: what the rows' states allow (finished rows: nothing)."""
    states = s["states"][at]
    return (s["next"][states.clamp(min=0).long()] >= 0) & (states >= 0)[:, None]


def _masked(s):
    x = s["logits"].float()
    return x if s["next"] is None else x.masked_fill(~_allowed(s), -math.inf)


def _run_sample(s, case):
    if own:
        from paper_2407_08103_b200 import cstr
        cstr.cstr_sample(s["tables"], s["logits"], s["states"], s["tokens"], s["uniform"],
                         temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
                         logp_out=s["logp"], kept_out=s["kept"], states_out=s["states_out"])
        return [s["tokens"], s["logp"], s["kept"]] + ([s["states_out"]] if case["constrained"] else [])
    # borders between tokens lie close to each other where many are likely: weights and sums in 64 bits
    value, order = torch.sort(_masked(s), dim=1, descending=True, stable=True)
    v = case["vocab"]
    some = value[:, :1] > -math.inf
    greedy = (s["temperature"] == 0)[:, None]
    t = torch.where(greedy, 1.0, s["temperature"][:, None]).double()
    z = (value.double() - torch.where(some, value[:, :1], 0.0).double()) / t
    rank = torch.arange(v, device=DEV)
    keep = torch.where(greedy, rank < 1, z > -math.inf)
    w = torch.where(greedy, keep.double(), torch.exp(z))
    total = w.sum(1, keepdim=True)
    if s["top_k"] is not None:
        k = s["top_k"][:, None]
        keep = keep & ((rank < k) | (k <= 0))
    if s["min_p"] is not None:
        keep = keep & ((z >= torch.log(s["min_p"][:, None].double())) | (rank < 1))
    if s["top_p"] is not None:
        kept = torch.where(keep, w, 0.0)
        before = torch.nn.functional.pad(kept.cumsum(1), (1, 0))
        p = s["top_p"][:, None].double()
        keep = keep & ((before[:, :-1] < p * before[:, -1:]) | (p >= 1) | (rank < 1))
    mass = torch.zeros_like(w).scatter_(1, order, torch.where(keep, w, 0.0))      # by token again
    upto = mass.cumsum(1)
    token = (upto <= s["uniform"][:, None].double() * upto[:, -1:]).sum(1, keepdim=True).clamp(max=v - 1)
    own_mass = mass.gather(1, token)
    some = some[:, 0]
    logp = torch.where(some, torch.log(own_mass / total)[:, 0], -math.inf).float()
    kept = torch.where(some, (upto[:, -1:] / total)[:, 0], 0.0).float()
    tokens = torch.where(some, token[:, 0], -1).to(torch.int32)
    if not case["constrained"]:
        return [tokens, logp, kept]
    after = s["next"][s["states"].clamp(min=0).long(), token[:, 0]]
    return [tokens, logp, kept, torch.where(some, after, -1)]


def _run_top(s, case):
    if own:
        from paper_2407_08103_b200 import cstr
        cstr.cstr_top_logprobs(s["tables"], s["logits"], s["states"], s["ids"], s["logp"], lse_out=s["lse"])
        return [s["ids"], s["logp"], s["lse"]]
    x = _masked(s)
    value, order = torch.sort(x, dim=1, descending=True, stable=True)
    top, n = value[:, :1], min(case["n"], case["vocab"])
    top = torch.where(top > -math.inf, top, 0.0)
    lse = top + torch.log(torch.exp(x - top).sum(1, keepdim=True))
    ids = torch.where(value[:, :n] > -math.inf, order[:, :n], -1).to(torch.int32)
    return [ids, torch.where(ids >= 0, value[:, :n] - lse, -math.inf), lse[:, 0]]


def _run_distill(s, case):
    if own:
        from paper_2407_08103_b200 import cstr
        cstr.cstr_distill_loss(s["tables"], s["logits"], s["states"], s["ids"], s["teacher"], s["loss"],
                               weight=s["weight"], dlogits=s["dlogits"], tail=TAILS[case["tail"]])
        return [s["loss"]] + ([s["dlogits"]] if case["gradient"] else [])
    # the rest's probability is what is left of 1, and a divergence a small difference: records in 64 bits
    x = _masked(s)
    at = s["ids"].clamp(min=0).long()
    mine = x.gather(1, at)
    in_both = (s["ids"] >= 0) & (mine > -math.inf) & (s["teacher"] > -math.inf)
    t = torch.where(in_both, torch.exp(s["teacher"].double()), 0.0)
    if case["tail"] == "renorm":
        t = t / t.sum(1, keepdim=True).clamp(min=1e-300)
    top = x.amax(1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    e = torch.exp(x - top)
    v, real = case["vocab"], s["ids"] >= 0
    spot = torch.where(real, s["ids"], v).long()         # what is no token goes to a column of its own
    total = e.sum(1, keepdim=True, dtype=torch.float64)
    logs = (mine - top).double() - torch.log(total)
    term = torch.where(t > 0, t * (torch.log(t) - logs), 0.0).sum(1)
    all_t = t.sum(1, keepdim=True)
    coef = all_t
    if case["tail"] == "lump":
        left = torch.nn.functional.pad(e, (0, 1)).scatter_(1, spot, 0.0)[:, :v].sum(1, keepdim=True, dtype=torch.float64)
        given = torch.where(real, torch.exp(s["teacher"].double()), 0.0).sum(1, keepdim=True)
        rest = torch.where(left > 0, (1.0 - given).clamp(min=0.0), 0.0)
        share = left / total
        term = term + torch.where(rest > 0, rest * torch.log(rest / share), 0.0)[:, 0]
        all_t = all_t + rest
        coef = all_t - torch.where(rest > 0, rest / share, 0.0)
    valid = (total > 0)[:, 0]
    w = s["weight"].double()
    loss = torch.where(valid, w * term, 0.0).float()
    if not case["gradient"]:
        return [loss]
    scale = torch.where(valid, w, 0.0)[:, None]
    grad = torch.nn.functional.pad(e * (scale * coef / total).float(), (0, 1))
    exactly = scale * (all_t * torch.exp(logs) - t)
    grad = grad.scatter_(1, spot, exactly.float())[:, :v]
    return [loss, torch.where(valid[:, None], grad, 0.0).to(s["logits"].dtype)]


def run(state):
    case = state["case"]
    return {"sample": _run_sample, "top": _run_top, "distill": _run_distill}[case["op"]](state, case)


# ---------------------------------------------------------------- exact

def _exact_sample(s, case):
    """One row at a time over the list of its own tokens: nothing is sorted but what can be kept."""
    n = case["rows"]
    logp = torch.full((n,), -math.inf, dtype=torch.float64, device=DEV)
    kept = torch.zeros(n, dtype=torch.float64, device=DEV)
    u, temps = s["uniform"].tolist(), s["temperature"].tolist()
    ks, ps, ms = (None if s[k] is None else s[k].tolist() for k in ("top_k", "top_p", "min_p"))
    states = None if s["states"] is None else s["states"].tolist()
    for r in range(n):
        if states is not None and states[r] < 0:
            continue
        ids = torch.arange(case["vocab"], device=DEV) if states is None else (s["next"][states[r]] >= 0).nonzero()[:, 0]
        if ids.numel() == 0:
            continue
        x = s["logits"][r, ids].to(torch.float64)
        if temps[r] == 0.0:
            logp[r], kept[r] = 0.0, 1.0
            continue
        p = torch.softmax(x / temps[r], 0)
        mine = torch.argsort(-x, stable=True)
        if ks is not None and ks[r] > 0:
            mine = mine[:ks[r]]
        if ms is not None and ms[r] > 0:
            mine = mine[:max(1, int((x[mine] >= x.max() + temps[r] * math.log(ms[r])).sum()))]
        if ps is not None and ps[r] < 1.0:
            share = torch.cumsum(p[mine], 0)
            mine = mine[:int(torch.searchsorted(share, ps[r] * share[-1])) + 1]
        mine = mine.sort().values
        share = torch.cumsum(p[mine], 0)
        i = int(torch.searchsorted(share, u[r] * share[-1], right=True))
        logp[r], kept[r] = torch.log(p[mine[min(i, mine.numel() - 1)]]), share[-1]
    return [None, logp, kept] + ([None] if case["constrained"] else [])


def _exact_rows(s, lo, hi):
    x = s["logits"][lo:hi].to(torch.float64)
    return x if s["next"] is None else torch.where(_allowed(s, slice(lo, hi)), x, -math.inf)


def _exact_top(s, case):
    out, lses = [], []
    for lo in range(0, case["rows"], 64):
        x = _exact_rows(s, lo, lo + 64)
        lse = torch.logsumexp(x, 1)
        value = x.topk(min(case["n"], case["vocab"]), dim=1).values
        out.append(torch.where(value > -math.inf, value - lse[:, None], -math.inf))
        lses.append(lse)
    return [None, torch.cat(out), torch.cat(lses)]


def _exact_distill(s, case):
    """The rows' distributions over all tokens and, with a lumped tail, over the records' tokens and one more."""
    n, v = case["rows"], case["vocab"]
    loss = torch.zeros(n, dtype=torch.float64, device=DEV)
    grad = torch.zeros((n, v), dtype=torch.float64, device=DEV) if case["gradient"] else None
    for lo in range(0, n, 64):
        x = _exact_rows(s, lo, lo + 64)
        m = x.shape[0]
        ids, given = s["ids"][lo:lo + 64], torch.exp(s["teacher"][lo:lo + 64].to(torch.float64))
        teacher = torch.zeros((m, v + 1), dtype=torch.float64, device=DEV)
        teacher.scatter_(1, torch.where(ids < 0, v, ids).long(), given)      # the last column takes what is not real
        teacher = teacher[:, :v]
        logq = torch.log_softmax(x, 1)
        in_record = teacher > 0
        rest = (1.0 - teacher.sum(1)).clamp(min=0.0)
        teacher = torch.where(x > -math.inf, teacher, 0.0)
        if case["tail"] == "renorm":
            teacher = teacher / teacher.sum(1, keepdim=True).clamp(min=1e-300)
        value = torch.where(teacher > 0, torch.xlogy(teacher, teacher) - teacher * logq, 0.0).sum(1)
        q = torch.exp(logq)
        wanted = teacher
        if case["tail"] == "lump":
            others = torch.where(in_record, 0.0, q)
            share = others.sum(1)
            rest = torch.where(share > 0, rest, 0.0)
            value = value + torch.where(rest > 0, torch.xlogy(rest, rest) - rest * torch.log(share), 0.0)
            wanted = teacher + others * torch.where(share > 0, rest / share, 0.0)[:, None]
        ok = (x > -math.inf).any(1)
        w = torch.where(ok, s["weight"][lo:lo + 64].to(torch.float64), 0.0)
        loss[lo:lo + 64] = torch.where(ok, w * value, 0.0)
        if grad is not None:
            d = w[:, None] * (q * wanted.sum(1, keepdim=True) - wanted)
            grad[lo:lo + 64] = torch.where(ok[:, None], d, 0.0)
    return [loss] + ([grad] if grad is not None else [])


def exact(case, seed):
    s = _prepare(case, seed)
    return {"sample": _exact_sample, "top": _exact_top, "distill": _exact_distill}[case["op"]](s, case)
