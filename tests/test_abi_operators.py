"""Argument checks of the cache and loss entry points that precede every CUDA call, and of their
binding before the library is reached."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2407_08103_b200 import build, cstr


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return cstr.lib()


def test_null_range_and_type_errors(lib):
    out = ctypes.c_void_p()
    z = np.zeros(64, dtype=np.int64)
    p = ctypes.c_void_p(z.ctypes.data & ~15)
    s4, s6, s3 = ((ctypes.c_int64 * n)(*[8] * n) for n in (4, 6, 3))

    def create(dtype=1, batch=2, heads=4, kv=2, dim=64, tokens=1, pk=p, pv=p, plen=8, ps=s4, ck=p, cv=p,
               cap=4, cs=s6, w=p, age=p, lens=p):
        return lib.cstr_cache_create(dtype, batch, heads, kv, dim, tokens, pk, pv, ctypes.c_int64(plen), ps,
                                     ck, cv, cap, cs, w, age, lens, ctypes.byref(out))
    for kw in (dict(ck=None), dict(cv=None), dict(cs=None), dict(lens=None), dict(pk=None), dict(pv=None), dict(ps=None)):
        assert create(**kw) == -1, kw
    assert lib.cstr_cache_create(1, 1, 1, 1, 64, 1, p, p, ctypes.c_int64(0), s4, p, p, 1, s6, p, p, p, None) == -1
    for dtype in (0, 3, -1):
        assert create(dtype=dtype) == -5
    for kw in (dict(batch=0), dict(heads=3), dict(heads=1), dict(kv=0), dict(dim=0), dict(dim=12), dict(dim=136),
               dict(tokens=0), dict(cap=0), dict(plen=-1)):
        assert create(**kw) == -2, kw
    assert create(plen=1 << 31) == -6 and create(batch=1 << 28) == -6 and create(tokens=1 << 24) == -6
    assert create(cs=(ctypes.c_int64 * 6)(8, 8, 8, 8, 8, 12)) == -6
    assert b"multiple of 8" in lib.cstr_last_error()
    assert create(ps=(ctypes.c_int64 * 4)(8, 1, 8, 8)) == -6
    assert create(cv=ctypes.c_void_p(p.value + 8)) == -6 and create(pk=ctypes.c_void_p(p.value + 2)) == -6
    assert out.value is None
    assert lib.cstr_cache_insert(None, p, p, s6, 1, None, p, 4, 0, None) == -1
    assert lib.cstr_cache_attention(None, p, s3, 1, None, None, 1.0, 0, p, s3, None, None) == -1
    lib.cstr_free_cache(None)

    def loss(n_tables=0, dtype=0, ld=8, v=8, temp=1.0, logits=p, act=p, lo=0.2, hi=0.2, kl=0.0, rows=2, states=None):
        return lib.cstr_policy_loss(None, n_tables, None, states, logits, dtype, ld, v, temp, act, p, None, p, None,
                                    lo, hi, kl, p, p, None, rows, None)
    assert loss(n_tables=-1) == -2 and loss(n_tables=17) == -2 and loss(dtype=2) == -5
    assert loss(ld=7) == -6 and loss(v=0) == -2 and loss(rows=-1) == -2 and loss(rows=0) == 0
    for kw in (dict(temp=0.0), dict(temp=-1.0), dict(temp=float("nan")), dict(temp=float("inf")), dict(lo=-1.0),
               dict(hi=float("nan")), dict(kl=float("inf"))):
        assert loss(**kw) == -2, kw
    assert loss(logits=None) == -1 and loss(act=None) == -1
    assert loss(n_tables=1) == -1 and loss(n_tables=1, states=p) == -1
    assert loss(logits=ctypes.c_void_p(p.value + 2)) == -6 and loss(logits=ctypes.c_void_p(p.value + 1), dtype=1) == -6


def test_binding_refuses_before_the_library(monkeypatch):
    def no_library():
        raise AssertionError("the library was reached")
    monkeypatch.setattr(cstr, "lib", no_library)
    bf = torch.bfloat16
    k = torch.zeros(2, 4, 2, 64, dtype=bf)
    lens = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        cstr.cstr_cache_create(k.float(), k.float(), lens, 4)
    with pytest.raises(TypeError):
        cstr.cstr_cache_create(k, k.half(), lens, 4)
    with pytest.raises(ValueError):
        cstr.cstr_cache_create(k, k[:, :3], lens, 4)
    with pytest.raises(ValueError):
        cstr.cstr_cache_create(k, k, lens.long(), 4)
    with pytest.raises(ValueError, match="go together"):
        cstr.cstr_cache_create(k, k, lens, 4, prefix_k=k[0])
    with pytest.raises(ValueError, match="CUDA tensor"):
        cstr.cstr_cache_create(k, k, lens, 4)
    x = torch.zeros(3, 8)
    v = torch.zeros(3)
    with pytest.raises(TypeError):
        cstr.cstr_policy_loss(None, x.double(), None, v.int(), v, v, v, v)
    with pytest.raises(ValueError, match="CUDA tensor"):
        cstr.cstr_policy_loss(None, x, None, v.int(), v, v, v, v)
