"""The decoder's settings given as numbers: their memory under capture, on other streams, and after many others."""
import math
import weakref

import pytest
import torch

from paper_2407_08103_b200 import cstr
from paper_2407_08103_b200.decode import ConstrainedDecoder
from synth.configs import config_dfas, config_vocab

from distribution_cases import F32, logits
from gpu_common import gpu_tables
from operator_cases import DEV

pytestmark = pytest.mark.gpu
B = 8


def decoder():
    vb, vo = config_vocab("api_1k")
    dec = ConstrainedDecoder(gpu_tables([config_dfas("api_1k")[0]], vb, vo), B)
    return dec, logits(3, B, vo.size - 1, F32), torch.rand(B, device=DEV)


@pytest.fixture
def given(monkeypatch):
    """References to what the last call was given as its settings."""
    refs, call = {}, cstr.cstr_sample

    def watched(*a, **kw):
        refs.update({k: weakref.ref(kw[k]) for k in ("temperature", "top_k", "top_p", "min_p") if kw[k] is not None})
        return call(*a, **kw)
    monkeypatch.setattr(cstr, "cstr_sample", watched)
    return refs


def poison():
    """Takes what the allocator has to give for a decoder's settings and fills it."""
    return [torch.full((B,), math.nan, device=DEV) for _ in range(200)]


def test_a_captured_number_outlives_all_others(given):
    dec, x, u = decoder()
    kw = dict(temperature=0.7, top_k=30, top_p=0.9, min_p=0.01)
    want = dec.sample(x, u, **kw)[0].clone()
    dec.reset()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dec.sample(x, u, **kw)
    captured = dict(given)
    assert len(captured) == 4
    for i in range(100):
        dec.sample(x, u, temperature=0.5 + i / 128, top_p=0.5 + i / 256)
    assert len(dec._settings) <= 64
    held = poison()
    assert all(r() is not None for r in captured.values()), "a captured step's setting was freed"
    for _ in range(3):
        dec.reset()
        dec.tokens.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dec.tokens, want)
    dec.reset()                                              # the same numbers outside the graph
    assert torch.equal(dec.sample(x, u, **kw)[0], want)
    assert len(held) == 200


def test_numbers_dropped_within_a_call_on_another_stream():
    dec, x, u = decoder()
    want = dec.sample(x, u, temperature=0.25, top_p=0.75)[0].clone()
    side = torch.cuda.Stream()
    for new in (0.8, 0.85):
        dec._settings.clear()
        dec.sample(x, u, temperature=0.25)
        for i in range(63):                                  # full: the next new number drops the temperature's tensor
            dec.sample(x, u, min_p=(i + 1) / 1024)
        assert len(dec._settings) == 64
        dec.reset()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(200_000_000)                   # a tenth of a second
        dec.sample(x, u, temperature=0.25, top_p=new, stream=side)
        held = poison()
        side.synchronize()
        twin = dec.tokens.clone()
        dec.reset()
        again = dec.sample(x, u, temperature=torch.full((B,), 0.25, device=DEV), top_p=torch.full((B,), new, device=DEV))[0]
        assert torch.equal(twin, again) and len(held) == 200
    dec.reset()
    assert torch.equal(dec.sample(x, u, temperature=0.25, top_p=0.75)[0], want)


def test_a_capture_on_the_stream_that_is_passed():
    dec, x, u = decoder()
    want = dec.sample(x, u, temperature=0.7)[0].clone()
    dec.reset()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        graph.capture_begin()
    try:
        with pytest.raises(RuntimeError, match="before the capture"):
            dec.sample(x, u, temperature=0.123, stream=side)
        dec.sample(x, u, temperature=0.7, stream=side)
    finally:
        with torch.cuda.stream(side):
            graph.capture_end()
    assert ("temperature", 0.7) in dec._captured
    for i in range(70):
        dec.sample(x, u, temperature=0.5 + i / 128)
    dec.reset()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(dec.tokens, want)


def test_a_new_number_does_not_wait_for_other_streams():
    dec, x, u = decoder()
    for i in range(70):
        dec.sample(x, u, temperature=0.5 + i / 128)
    side, done = torch.cuda.Stream(), torch.cuda.Event()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(1_000_000_000)                     # half a second
        done.record()
    for i in range(70):
        dec.sample(x, u, temperature=0.75 + i / 1024)
    assert not done.query()
    torch.cuda.synchronize()
