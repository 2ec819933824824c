"""Numbers that are no settings are refused before anything reaches the GPU."""
import math

import pytest
import torch

from paper_2407_08103_b200.decode import ConstrainedDecoder


@pytest.mark.parametrize("value", [0.5, 2.5, -0.5, math.nan, math.inf])
def test_top_k_counts_tokens(value):
    dec = ConstrainedDecoder.__new__(ConstrainedDecoder)     # (a decoder's tables live on a GPU)
    dec._settings, dec._captured = {}, {}
    with pytest.raises(ValueError, match="top_k"):
        dec._setting("top_k", value, 0, torch.int32, (False, 0, None))
    assert dec._setting("top_k", 0.0, 0, torch.int32, (False, 0, None)) is None
