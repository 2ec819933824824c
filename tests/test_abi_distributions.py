"""Argument checks of the operators over whole distributions that precede every CUDA call."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2407_08103_b200 import build, cstr


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return cstr.lib()


P = ctypes.c_void_p(np.zeros(64, dtype=np.int64).ctypes.data & ~15)


def test_sample_arguments(lib):
    def sample(tables=None, n_tables=0, states=None, states_out=None, logits=P, dtype=0, ld=8, v=8, uniform=P, tokens=P, rows=2):
        return lib.cstr_sample(tables, n_tables, None, states, states_out, logits, dtype, ld, v, uniform, None, None, None,
                               None, tokens, None, None, None, rows, None)
    assert sample(n_tables=-1) == -2 and sample(n_tables=17) == -2 and sample(rows=-1) == -2 and sample(v=0) == -2
    assert sample(v=8388609, ld=8388609) == -2 and sample(dtype=2) == -5 and sample(ld=7) == -6
    assert sample(logits=None) == -1 and sample(uniform=None) == -1 and sample(tokens=None) == -1
    assert sample(n_tables=1) == -1 and sample(n_tables=1, tables=P, states=P) == -1
    assert sample(n_tables=1, tables=P, states_out=P) == -1
    assert sample(logits=ctypes.c_void_p(P.value + 2)) == -6
    assert sample(logits=ctypes.c_void_p(P.value + 1), dtype=1) == -6
    assert sample(rows=0, logits=None, uniform=None, tokens=None) == 0


def test_top_arguments(lib):
    def top(n_tables=0, states=None, logits=P, dtype=0, ld=8, v=8, temperature=1.0, n=4, ids=P, logp=P, rows=2):
        return lib.cstr_top_logprobs(None, n_tables, None, states, logits, dtype, ld, v, temperature, n, ids, logp, None,
                                     rows, None)
    assert top(n_tables=17) == -2 and top(rows=-1) == -2 and top(v=0) == -2 and top(dtype=3) == -5 and top(ld=7) == -6
    assert top(n=0) == -2 and top(n=1025) == -2
    for t in (0.0, -1.0, float("nan"), float("inf"), 1e-39):
        assert top(temperature=t) == -2, t
    assert top(logits=None) == -1 and top(ids=None) == -1 and top(logp=None) == -1
    assert top(n_tables=1) == -1 and top(n_tables=1, states=P) == -1
    assert top(rows=0) == 0


def test_binding_refuses_before_the_library(monkeypatch):
    def no_library():
        raise AssertionError("the library was reached")
    monkeypatch.setattr(cstr, "lib", no_library)
    x, v = torch.zeros(3, 8), torch.zeros(3)
    with pytest.raises(TypeError):
        cstr.cstr_sample(None, x.double(), None, v.int(), v)
    with pytest.raises(ValueError, match="unit inner stride"):
        cstr.cstr_sample(None, x.T, None, v.int(), v)
    for call in (lambda: cstr.cstr_sample(None, x, None, v.int(), v),
                 lambda: cstr.cstr_top_logprobs(None, x, None, torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 2))):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()


def test_distill_arguments(lib):
    def loss(n_tables=0, states=None, logits=P, dtype=0, ld=8, v=8, temperature=1.0, ids=P, logp=P, k=4, tail=0, out=P, d=None,
             rows=2):
        return lib.cstr_distill_loss(None, n_tables, None, states, logits, dtype, ld, v, temperature, ids, logp, k, tail,
                                     None, out, d, rows, None)
    assert loss(n_tables=-1) == -2 and loss(rows=-1) == -2 and loss(v=0) == -2 and loss(v=8388609, ld=8388609) == -2
    assert loss(dtype=2) == -5 and loss(ld=7) == -6 and loss(k=0) == -2 and loss(k=1025) == -2
    assert loss(tail=-1) == -2 and loss(tail=3) == -2
    for t in (0.0, -1.0, float("nan"), float("inf"), 1e-39):
        assert loss(temperature=t) == -2, t
    assert loss(logits=None) == -1 and loss(ids=None) == -1 and loss(logp=None) == -1 and loss(out=None) == -1
    assert loss(n_tables=1) == -1 and loss(n_tables=1, states=P) == -1
    assert loss(logits=ctypes.c_void_p(P.value + 2)) == -6 and loss(d=ctypes.c_void_p(P.value + 1), dtype=1) == -6
    assert loss(rows=0, logits=None) == 0
