"""The README's lines on draws, records and distillation, run as they stand there."""
import os

import numpy as np
import pytest
import torch

import oracle
from helpers import ROOT
from oracle import distributions as ref
from paper_2407_08103_b200 import cstr
from paper_2407_08103_b200.decode import ConstrainedDecoder
from synth.configs import config_dfas, config_vocab

from distribution_cases import F32, logits
from gpu_common import gpu_tables
from operator_cases import DEV, f8

pytestmark = pytest.mark.gpu


def test_the_lines_as_they_stand():
    with open(os.path.join(ROOT, "README.md")) as f:
        text = f.read()
    lines = text[text.index("# every request with its own settings"):]
    lines = lines[:lines.index("```")]
    dfa = config_dfas("api_1k")[0]
    vb, vo = config_vocab("api_1k")
    table = gpu_tables([dfa], vb, vo)[0]
    dec, B, V = ConstrainedDecoder(table, 512), 512, vo.size - 1
    x = logits(1, B, V, F32)
    dec.states.copy_(torch.arange(B, device=DEV) % dec.infos[0]["n_states"])
    q = dec.states.cpu().numpy()
    names = dict(torch=torch, cstr=cstr, dec=dec, table=table, logits=x, student_logits=logits(2, B, V, F32))
    exec(lines, names)
    allowed = oracle.token_table(dfa[0], dfa[1], vb, vo)[0][q] >= 0
    ids, logps, tokens = (names[k].cpu().numpy() for k in ("ids", "logps", "tokens"))
    want = ref.top(f8(x), allowed, 64, float(np.float32(0.8)))
    assert np.array_equal(ids, want[0])                      # of the states before the draw
    some = tokens >= 0
    assert np.array_equal(some, allowed.any(1)) and some.sum() > B // 2
    drawn = (ids == tokens[:, None]) & some[:, None]
    # the draw's log probability is its entry's: two sums over the row in 32 and in 64 bits, and two roundings
    pick = drawn.any(1)
    assert pick.sum() > B // 4
    err = np.abs(logps[drawn].astype(np.float64) - names["logp"].cpu().numpy()[pick].astype(np.float64))
    assert err.max() <= 2 * 2.0 ** -24 * (2.1 * 10 + 36 + 30)
    loss = ref.distill(f8(names["student_logits"]), allowed, ids, logps.astype(np.float64), ref.RENORM)[0]
    assert np.abs(f8(names["loss"]) - loss).max() <= 2.0 ** -24 * 1000
