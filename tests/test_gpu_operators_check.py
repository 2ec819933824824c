"""Small cases of the cache and loss operators once more against the checking build: the record of
out-of-range indices stays at zero."""
import pytest
import torch

from paper_2407_08103_b200 import cstr

import test_gpu_cache as cache_cases
import test_gpu_loss as loss_cases

pytestmark = pytest.mark.gpu


@pytest.fixture
def checked():
    cstr.use_check_library(True)
    try:
        cstr.cstr_debug_bounds_status(reset=True)
        yield
        torch.cuda.synchronize()
        record = cstr.cstr_debug_bounds_status(reset=True)
        assert record[0] == 0, "out-of-range index: site %d, index %d, extent %d" % record[1:]
    finally:
        cstr.use_check_library(False)


@pytest.mark.parametrize("shape", [(3, 1, 4, 2, 64, 17, 5), (2, 3, 7, 1, 96, 129, 19), (1, 17, 3, 1, 16, 5, 300),
                                   (2, 4, 64, 2, 64, 0, 50)])
def test_attention(checked, shape):
    cache_cases.test_attention_shapes(*shape, torch.bfloat16)


@pytest.mark.parametrize("kind", ["full", "ties", "odd", "any"])
@pytest.mark.parametrize("shape", [(1, 1, 8, 1, 1, 1, 0), (3, 2, 64, 40, 1, 33, 8), (2, 1, 128, 700, 300, 600, 20),
                                   (3, 1, 64, 100, 0, 50, 20)])
def test_insert(checked, shape, kind):
    cache_cases.test_insert(*shape, kind)


def test_loss(checked):
    loss_cases.test_constrained_mixed_tables_and_invalid_rows(torch.float32)
    loss_cases.test_row_strides_and_alignment(torch.bfloat16, 1031, 0)
