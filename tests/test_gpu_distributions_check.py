"""Small cases of the operators over whole distributions once more against the checking build: the record of
out-of-range indices stays at zero."""
import numpy as np
import pytest
import torch

from paper_2407_08103_b200 import cstr

import test_gpu_distill as distill_cases
import test_gpu_sample as sample_cases
from distribution_cases import BF, F32, check_sample, logits

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


@pytest.mark.parametrize("dtype", [F32, BF])
def test_sampling(checked, dtype):
    sample_cases.test_constrained_rows(dtype, ("api_1k",))
    sample_cases.test_row_strides_and_alignment(dtype, 1031, 0)
    sample_cases.test_lists_that_overflow_or_hold_everything(dtype)


def test_wide_nuclei_over_a_cluster(checked):
    x = logits(3, 2, 60001, F32, sigma=0.7, peaks=1)
    check_sample(x, np.array([0.3, 0.9], np.float32), top_p=np.array([0.9, 0.99], np.float32))


@pytest.mark.parametrize("tail", distill_cases.TAILS)
def test_distillation(checked, tail):
    distill_cases.test_ids_twice_out_of_range_and_missing(tail)
    distill_cases.test_constrained_rows_and_foreign_records(F32, tail)
    distill_cases.test_shapes(1, 128256, 1024, BF, tail)
