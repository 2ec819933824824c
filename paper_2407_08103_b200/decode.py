"""Batched constrained decoding driver over the libcstr binding.

Holds the per-batch device state (one automaton state per row, Algorithm 2's
``q``) and the step workspace; every step is one ``cstr_step`` call.  The LM
that produces the logits is outside this package; ``SharedPromptCache`` is the
attention of one of its layers for a batch that answers one prompt.
"""

from __future__ import annotations

import torch

from . import cstr


def _capturing(stream):
    """Whether the current stream or the one that was passed is being captured."""
    if torch.cuda.is_current_stream_capturing():
        return True
    if stream is None:
        return False
    with torch.cuda.stream(stream):
        return torch.cuda.is_current_stream_capturing()


class ConstrainedDecoder:
    """``tables``: one built Table, or several for a mixed-constraint batch with
    ``row_table`` (int32 per row) choosing each row's table."""

    def __init__(self, tables, batch: int, row_table=None, device="cuda:0"):
        self.tables = [tables] if isinstance(tables, cstr.Table) else list(tables)
        self.batch = batch
        self.device = torch.device(device)
        self.infos = [cstr.cstr_table_info(t) for t in self.tables]
        self.vocab_size = self.infos[0]["vocab_size"]
        self.ws = cstr.cstr_workspace_create(batch)
        self.row_table = None
        if row_table is not None:
            self.row_table = torch.as_tensor(row_table, dtype=torch.int32).to(self.device)
        self.states = torch.empty(batch, dtype=torch.int32, device=self.device)
        self.tokens = torch.empty(batch, dtype=torch.int32, device=self.device)
        self.accept = torch.empty(batch, dtype=torch.uint8, device=self.device)
        self.logp = torch.empty(batch, dtype=torch.float32, device=self.device)
        self.kept = torch.empty(batch, dtype=torch.float32, device=self.device)
        self._settings = {}                       # per-row tensors of settings given as numbers, and the streams that read them
        self._captured = {}                       # ... those that captured steps read
        self._fills = None                        # the stream that fills them
        self._start = self._start_states()
        self.reset()

    def _start_states(self):
        starts = torch.tensor([i["start_state"] for i in self.infos], dtype=torch.int32,
                              device=self.device)
        if self.row_table is None:
            return starts[0].expand(self.batch).contiguous()
        return starts[self.row_table.long()].contiguous()

    def reset(self):
        """All rows back to their automaton's start state (Algorithm 2: q <- I)."""
        self.states.copy_(self._start)

    def step(self, logits, noise=None, masked_out=None, stream=None):
        """One decoding step; returns ``(tokens, masked_logits)`` (device tensors;
        ``tokens`` is reused by the next call)."""
        if masked_out is None:
            masked_out = torch.empty_like(logits)
        cstr.cstr_step(self.tables, logits, self.states, self.tokens, masked_out, self.ws,
                       noise=noise, row_table=self.row_table, accept_out=self.accept,
                       stream=stream)
        return self.tokens, masked_out

    def sample(self, logits, uniform, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, stream=None):
        """One decoding step that draws each row's token from one uniform number (float32 ``[B]``) under
        ``cstr_sample``'s cuts; returns ``(tokens, logp)`` (device tensors, reused by the next call), and
        ``self.kept`` holds the probability that the cuts left.  A setting is a number, or a tensor with one
        entry per row.  A number is held as a tensor of the decoder's: under capture it has to have been used
        before, and the decoder keeps it from then on; a tensor is the caller's to keep."""
        reader = (_capturing(stream), cstr._raw_stream(stream, logits.device), stream)
        cstr.cstr_sample(self.tables, logits, self.states, self.tokens, uniform,
                         temperature=self._setting("temperature", temperature, 1.0, torch.float32, reader),
                         top_k=self._setting("top_k", top_k, 0, torch.int32, reader),
                         top_p=self._setting("top_p", top_p, 1.0, torch.float32, reader),
                         min_p=self._setting("min_p", min_p, 0.0, torch.float32, reader),
                         logp_out=self.logp, kept_out=self.kept, row_table=self.row_table,
                         accept_out=self.accept, stream=stream)
        return self.tokens, self.logp

    def _setting(self, name, value, off, dtype, reader):
        """``reader``: whether a capture is under way, the stream's address, the stream (None: the current one)."""
        if torch.is_tensor(value):
            return value
        if value == off:
            return None
        at, (capturing, raw, stream) = (name, value), reader
        entry = self._settings.get(at) or self._captured.get(at)
        if entry is None:                         # a program has a few: filled once, read by every step
            entry = self._filled(name, value, dtype, capturing)
        row, streams = entry
        if capturing:                             # replays read it as long as the graph lives: it is not dropped any more
            self._captured[at] = entry
        elif raw not in streams:                  # its memory is not handed out again before that stream's steps are done
            row.record_stream(stream or torch.cuda.current_stream(row.device))
            streams.add(raw)
        return row

    def _filled(self, name, value, dtype, capturing):
        if value != value:
            raise ValueError("%s is not a number" % name)
        if dtype == torch.int32 and value % 1 != 0:
            raise ValueError("%s = %r is not a whole number" % (name, value))
        if capturing:
            raise RuntimeError("%s = %r: take one step with it before the capture" % (name, value))
        if len(self._settings) >= 64:             # (an annealed setting; what steps under way still read is recorded)
            self._settings.clear()
        self._fills = self._fills or torch.cuda.Stream(self.device)
        with torch.cuda.stream(self._fills):
            entry = (torch.full((self.batch,), value, dtype=dtype, device=self.device), set())
        self._fills.synchronize()                 # the filling alone: every stream and capture may read it from now on
        self._settings[name, value] = entry
        return entry

    def top_logprobs(self, logits, n: int, temperature: float = 1.0, stream=None):
        """The ``n`` most likely tokens in the rows' present states: ``(ids, logp)`` ``[B][n]``.  A record of what
        ``sample`` (or ``step``) draws from these logits is taken before it: that call moves the states on."""
        with torch.cuda.stream(stream or torch.cuda.current_stream(self.device)):      # (their memory, too)
            ids = torch.empty((self.batch, n), dtype=torch.int32, device=self.device)
            logp = torch.empty((self.batch, n), dtype=torch.float32, device=self.device)
        cstr.cstr_top_logprobs(self.tables, logits, self.states, ids, logp, temperature=temperature,
                               row_table=self.row_table, stream=stream)
        return ids, logp

    def status(self, stream=None):
        """(rows with an out-of-range state, active rows without any allowed token) since last call."""
        return cstr.cstr_step_status(self.ws, stream)


class PushdownDecoder:
    """Per-batch state of Algorithm 3: one PDA state, one stack (``stack_cap``
    symbols) and its depth per row; every step is one ``cstr_pda_step`` call."""

    def __init__(self, table, batch: int, stack_cap: int = 64, device="cuda:0"):
        self.table = table
        self.batch = batch
        self.device = torch.device(device)
        self.info = cstr.cstr_pda_table_info(table)
        self.vocab_size = self.info["vocab_size"]
        self.ws = cstr.cstr_pda_workspace_create(table, batch)
        self.states = torch.empty(batch, dtype=torch.int32, device=self.device)
        self.stacks = torch.zeros((batch, stack_cap), dtype=torch.int32, device=self.device)
        self.depths = torch.empty(batch, dtype=torch.int32, device=self.device)
        self.tokens = torch.empty(batch, dtype=torch.int32, device=self.device)
        self.accept = torch.empty(batch, dtype=torch.uint8, device=self.device)
        self.reset()

    def reset(self):
        """All rows back to the start state with an empty stack (Algorithm 3: q <- I, s <- empty)."""
        self.states.fill_(self.info["start_state"])
        self.depths.zero_()

    def restart_finished(self):
        """Replace every finished row (state -1) by a fresh sequence."""
        done = self.states < 0
        self.states.masked_fill_(done, self.info["start_state"])
        self.depths.masked_fill_(done, 0)

    def step(self, logits, noise=None, masked_out=None, stream=None):
        if masked_out is None:
            masked_out = torch.empty_like(logits)
        cstr.cstr_pda_step(self.table, logits, self.states, self.stacks, self.depths, self.tokens,
                           masked_out, self.ws, noise=noise, accept_out=self.accept, stream=stream)
        return self.tokens, masked_out

    def status(self, stream=None):
        """(inactive rows other than finished ones, rows without an allowed token,
        rows whose stack outgrew ``stack_cap``) since the last call."""
        return cstr.cstr_pda_step_status(self.ws, stream)


class SharedPromptCache:
    """Keys, values and attention of one layer for ``batch`` rows that answer one prompt.

    ``prefix_k`` / ``prefix_v`` ``[P][n_kv_heads][D]`` (bfloat16 or float16) are the prompt's, held
    once; every row has ``budget`` slots for its own tokens.  A row that would exceed its budget
    loses the tokens that have received the least attention, its last ``recent`` ones excepted."""

    def __init__(self, prefix_k, prefix_v, batch: int, n_heads: int, budget: int, recent: int = 0,
                 max_tokens: int = 1):
        heads, dim = prefix_k.shape[1:]
        dev = prefix_k.device
        self.batch, self.budget, self.recent = batch, budget, recent
        self.k = torch.empty((batch, budget, heads, dim), dtype=prefix_k.dtype, device=dev)
        self.v = torch.empty_like(self.k)
        self.weight = torch.empty((batch, heads, budget), dtype=torch.float32, device=dev)
        self.age = torch.empty((batch, heads, budget), dtype=torch.int32, device=dev)
        self.lens = torch.zeros(batch, dtype=torch.int32, device=dev)
        self.pos = torch.zeros(batch, dtype=torch.int32, device=dev)
        self.handle = cstr.cstr_cache_create(self.k, self.v, self.lens, n_heads, prefix_k=prefix_k,
                                             prefix_v=prefix_v, weight=self.weight, age=self.age,
                                             max_tokens=max_tokens)

    def reset(self):
        """Forget every row's own tokens; the prompt stays."""
        self.lens.zero_()
        self.pos.zero_()

    def take_back(self, n, stream=None):
        """Forget each row's newest ``n`` tokens (int32 ``[B]``): drafts that verification rejected.
        Entries that were evicted for them do not come back."""
        with torch.cuda.stream(stream or torch.cuda.current_stream(self.pos.device)):
            self.pos.copy_((self.pos - n.flatten()[:self.batch].clamp(min=0)).clamp(min=0))
            cstr.cstr_cache_truncate(self.handle, self.pos, stream=stream)

    def _check_step(self, q, k, v, scale):
        """What the attention would refuse only after the insertion has taken place."""
        if not q.dim() == k.dim() == v.dim() == 4 or not 1 <= q.shape[1] == k.shape[1] == v.shape[1]:
            raise ValueError("q, k and v must be [B][T][heads][D] of the same T >= 1")
        address, strides = cstr._tokens_arg("q", q, self.handle, q.shape[1], self.handle.n_heads)
        if address % 16 or any(s % 8 or abs(s) > 1 << 33 for s in strides[:3]):
            raise ValueError("q must start on 16 bytes, with strides that are multiples of 8 up to 2^33")
        scale = self.handle.head_dim ** -0.5 if scale is None else float(scale)
        if not abs(scale) < 2.358e38:             # (times log2(e) a float)
            raise ValueError("scale is not finite or too large")
        return scale

    def step(self, q, k, v, n_new=None, scale=None, stream=None):
        """Put the new tokens' ``k`` / ``v`` ``[B][T][n_kv_heads][D]`` into the rows' caches and return
        the attention of ``q`` ``[B][T][n_heads][D]`` over the prompt and the caches.  ``n_new`` int32
        ``[B]``: tokens that a row really has (a finished row has 0); None: all ``T``."""
        scale = self._check_step(q, k, v, scale)
        tokens = q.shape[1]
        with torch.cuda.stream(stream or torch.cuda.current_stream(self.pos.device)):   # (its memory, too)
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
            cstr.cstr_cache_insert(self.handle, k, v, self.pos, self.budget, self.recent, n_new=n_new,
                                   stream=stream)
            cstr.cstr_cache_attention(self.handle, q, out, scale=scale, n_query=n_new, accumulate=True,
                                      pos=self.pos if tokens > 1 else None, stream=stream)
            # (n_new as the kernels take it)
            self.pos += tokens if n_new is None else n_new.flatten()[:self.batch].clamp(0, tokens)
        return out
