"""Refusals of the cache and loss entry points at the ends of their ranges; no GPU."""
import ctypes

import numpy as np
import pytest

from paper_2407_08103_b200 import build, cstr


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return cstr.lib()


@pytest.mark.parametrize("temperature", [1e-39, 4e-39])
def test_temperature_whose_reciprocal_overflows(lib, temperature):
    z = np.zeros(64, dtype=np.int64)
    p = ctypes.c_void_p(z.ctypes.data)
    assert lib.cstr_policy_loss(None, 0, None, None, p, 0, 8, 8, temperature, p, p, None, p, None, 0.2, 0.2, 0.0,
                                p, p, None, 2, None) == -2
    assert b"temperature" in lib.cstr_last_error()


def test_truncation_of_nothing(lib):
    p = ctypes.c_void_p(np.zeros(8, dtype=np.int64).ctypes.data)
    assert lib.cstr_cache_truncate(None, p, None) == -1
