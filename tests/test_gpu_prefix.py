"""Attention over prompts that are long enough for the tensor cores, against the oracle's statement in
64 bits: ends within a tile, one to several groups of query rows, head sizes, layouts, scales."""
import math

import numpy as np
import pytest
import torch

from paper_2407_08103_b200 import cstr

from operator_cases import AttentionCase

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def run(c, scale=None):
    c.run(scale=scale)
    r = c.check(scale=scale)
    assert cstr.cstr_cache_status(c.cache) == 0
    return r


@pytest.mark.parametrize("B,T,Hq,Hk,D,P,cap", [
    (1, 1, 1, 1, 8, 512, 1), (1, 1, 1, 1, 128, 513, 3), (3, 1, 4, 2, 64, 639, 5), (2, 1, 8, 8, 72, 640, 33),
    (4, 2, 12, 3, 40, 641, 40), (127, 1, 1, 1, 64, 520, 4), (32, 1, 4, 1, 128, 700, 9), (43, 1, 3, 1, 16, 1025, 7),
    (64, 1, 4, 1, 64, 530, 6), (257, 1, 1, 1, 128, 512, 2), (20, 3, 8, 2, 128, 900, 30), (60, 1, 16, 2, 80, 1300, 8),
    (1, 5, 40, 1, 120, 4100, 20), (2, 1, 2, 2, 64, 9001, 12), (100, 2, 8, 2, 64, 128, 10), (300, 1, 8, 4, 128, 200, 4),
])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_shapes(B, T, Hq, Hk, D, P, cap, dtype):
    causal = cap >= T > 1
    run(AttentionCase(B * 1000 + P, B, T, Hq, Hk, D, P, cap, dtype, causal=causal,
                      n_query=np.random.default_rng(2).integers(0, T + 1, B) if causal else None))


@pytest.mark.parametrize("scale", [-0.125, 0.0, 2.0])
@pytest.mark.parametrize("B", [3, 50])
def test_scales(scale, B):
    run(AttentionCase(31, B, 1, 8, 2, 64, 800, 20, BF), scale)


@pytest.mark.parametrize("sigma", [20.0, 200.0])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_maxima_that_grow_along_the_prompt(sigma, dtype):
    c = AttentionCase(32, 40, 1, 8, 2, 64, 1000, 12, dtype, sigma=sigma)
    c.pk *= torch.linspace(0.05, 1.0, 1000, device=c.pk.device).to(dtype)[:, None, None]
    run(c)


def test_prompt_layouts():
    c = AttentionCase(33, 5, 2, 8, 2, 64, 777, 30, BF, causal=True)
    c.pk = c.pk.transpose(0, 1).contiguous().transpose(0, 1)            # [heads][tokens][dim] storage
    both = torch.zeros(777, 2, 144, dtype=BF, device=c.pv.device)       # rows with padding
    both[..., 16:80] = c.pv
    c.pv = both[..., 16:80]
    run(c)


def test_lowest_keys_and_nonfinite_values():
    c = AttentionCase(34, 6, 1, 8, 2, 64, 700, 20, BF)
    c.pk[100] = torch.finfo(BF).min                                     # scores of -infinity in 32 bits
    c.q.abs_()
    run(c)
    c = AttentionCase(35, 6, 1, 8, 2, 64, 700, 20, BF)
    c.pv[650, 1, 5] = math.inf                                          # seen by the heads of the second
    r = run(c)
    assert np.isfinite(r["out"][:, :, :4]).all() and not np.isfinite(r["out"][:, :, 4:, 5]).any()


def test_one_row_is_not_changed_by_the_others():
    # a query of NaN stays in its own row, and tokens past n_query get nothing
    c = AttentionCase(36, 33, 2, 4, 1, 128, 600, 16, BF, causal=True, n_query=[1] * 32 + [2])
    c.run()
    c.check()
    want = c.out.clone()
    assert (want[:32, 1] == 0).all()
    c.w0 = None
    c.dev()
    c.q[7] = math.nan
    c.run()
    torch.cuda.synchronize()
    keep = [b for b in range(33) if b != 7]
    assert torch.equal(c.out[keep], want[keep]) and torch.isnan(c.out[7, 0]).all()


def test_repeats_bit_for_bit():
    runs = []
    for _ in range(3):
        c = AttentionCase(37, 70, 1, 8, 2, 128, 2000, 40, BF)
        c.run()
        torch.cuda.synchronize()
        runs.append((c.out.clone(), c.lse.clone(), c.d_w.clone()))
    assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(runs[0], r))


@pytest.mark.parametrize("shape", [(3, 1, 4, 2, 64, 639, 5), (43, 1, 3, 1, 16, 1025, 7), (20, 3, 8, 2, 128, 900, 30)])
def test_no_index_out_of_range(shape):
    cstr.use_check_library(True)
    try:
        cstr.cstr_debug_bounds_status(reset=True)
        test_shapes(*shape, BF)
        record = cstr.cstr_debug_bounds_status(reset=True)
        assert record[0] == 0, "out-of-range index: site %d, index %d, extent %d" % record[1:]
    finally:
        cstr.use_check_library(False)
