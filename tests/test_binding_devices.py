"""Tensors of another device than the current one do not reach the library: it would run on the current one."""
import types

import pytest
import torch

from paper_2407_08103_b200 import cstr


class OnDevice:
    """What the binding asks of a CUDA tensor, without one."""
    is_cuda = True

    def __init__(self, index, shape, dtype):
        self.device, self.shape, self.dtype = torch.device("cuda", index), torch.Size(shape), dtype

    def stride(self, i=None):
        return (self.shape[1], 1) if i is None else (self.shape[1], 1)[i]

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096


@pytest.mark.parametrize("index,current", [(1, 0), (0, 1), (0, 0)])
def test_operators_over_whole_rows(monkeypatch, index, current):
    reached = []

    def library():
        return types.SimpleNamespace(**{name: lambda *a: reached.append(name) or 0 for name in
                                        ("cstr_sample", "cstr_top_logprobs", "cstr_distill_loss", "cstr_policy_loss")})
    monkeypatch.setattr(cstr, "lib", library)
    monkeypatch.setattr(cstr, "_raw_stream", lambda stream, device: 0)
    cstr._load_types()
    monkeypatch.setattr(cstr, "_get_device", lambda: current)
    x, f, i = OnDevice(index, (3, 8), torch.float32), OnDevice(index, (3,), torch.float32), OnDevice(index, (3,), torch.int32)
    ids, logp = OnDevice(index, (3, 2), torch.int32), OnDevice(index, (3, 2), torch.float32)
    calls = (lambda: cstr.cstr_sample(None, x, None, i, f),
             lambda: cstr.cstr_top_logprobs(None, x, None, ids, logp),
             lambda: cstr.cstr_distill_loss(None, x, None, ids, logp, f),
             lambda: cstr.cstr_policy_loss(None, x, None, i, f, f, f, f))
    for call in calls:
        if index == current:
            call()
        else:
            with pytest.raises(ValueError, match="device %d is current" % current):
                call()
    assert len(reached) == (4 if index == current else 0)
