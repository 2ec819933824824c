"""Sampling at temperatures that stand for greedy decoding, and at the largest: exponents far below what a double holds."""
import math

import numpy as np
import pytest
import torch

from distribution_cases import BF, F32, check_sample
from operator_cases import DEV

pytestmark = pytest.mark.gpu

ROWS = 61
TEMPERATURES = [1e-9, 5e-9, 1e-8, 2e-8, 4e-8, 6e-7, 1.5e-6, 1e-5]


def rows(seed, V, dtype, equal=1):
    """Rows with maxima from 0.5 to about 2,000, five in each octave (the negative of every third); ``equal``:
    places of the maximum in the odd rows."""
    rng = np.random.default_rng(seed)
    top = 0.505 * 2.0 ** (np.arange(ROWS) / 5)
    top[::3] *= -1
    x = top[:, None] - np.abs(top)[:, None] * (0.01 + np.abs(rng.standard_normal((ROWS, V))))
    for i in range(ROWS):
        x[i, rng.choice(V, equal if i % 2 else 1, replace=False)] = top[i]
    return rng, torch.from_numpy(x).to(dtype).to(DEV)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("temperature", TEMPERATURES)
def test_no_cut(dtype, temperature):
    # three equal maxima lie in chunks of their own mostly
    for V in (1024, 5003):
        rng, x = rows(1, V, dtype, 3)
        want = check_sample(x, rng.random(ROWS).astype(np.float32), temperature=np.full(ROWS, temperature, np.float32))
        assert np.isfinite(want[1]).all()


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("temperature", TEMPERATURES)
def test_top_p_alone_and_mixed_settings(dtype, temperature):
    rng, x = rows(2, 1100, dtype, 3)
    x[5, ::2] = -math.inf
    u, t = rng.random(ROWS).astype(np.float32), np.full(ROWS, temperature, np.float32)
    check_sample(x, u, temperature=t, top_p=np.full(ROWS, 0.9, np.float32))
    pick = lambda v, d: rng.choice(np.array(v, d), ROWS)  # noqa: E731
    check_sample(x, u, temperature=t, top_p=pick([0.5, 0.95, 1.0], np.float32), top_k=pick([0, 0, 2, 40], np.int32),
                 min_p=pick([0.0, 0.0, 0.1], np.float32))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("temperature", TEMPERATURES)
def test_nuclei_of_thousands_of_equal_maxima(dtype, temperature):
    rng, x = rows(3, 9001, dtype, 5000)
    u, t = rng.random(ROWS).astype(np.float32), np.full(ROWS, temperature, np.float32)
    check_sample(x, u, temperature=t, top_p=np.full(ROWS, 0.6, np.float32))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("temperature", [1e30, 5e31, 1e34, 1.4e34, 1e35])
def test_lowest_values_at_the_largest_temperatures(dtype, temperature):
    N, V = 4, 9001
    rng = np.random.default_rng(4)
    x = torch.full((N, V), torch.finfo(dtype).min, dtype=dtype, device=DEV)
    x[:, ::3] = -math.inf
    x[1:, 1::9] = -3e38
    x[2, 1::18] = 1.0
    u, t = rng.random(N).astype(np.float32), np.full(N, temperature, np.float32)
    check_sample(x, u, temperature=t)
    check_sample(x, u, temperature=t, top_p=np.array([0.6, 0.9, 0.5, 0.99], np.float32))
