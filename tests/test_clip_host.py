"""What the clipping calls of the binding refuse before the library is asked, and what the clipper keeps (no GPU)."""
import types

import pytest
import torch

from paper_2603_01501_b200 import binding as gb
from paper_2603_01501_b200 import packed


class Fake:
    """What the checks look at of a tensor on some device."""

    def __init__(self, device, dtype):
        self.device, self.dtype, self.is_cuda = torch.device(device), dtype, True

    def numel(self):
        return 1

    def data_ptr(self):
        return 4096


class Library:
    def __getattr__(self, name):
        def call(*_):
            raise AssertionError(f"{name} was called")
        return call


def test_results_on_another_device_than_the_list_are_refused(monkeypatch):
    monkeypatch.setattr(gb, "load_library", Library)
    monkeypatch.setattr(gb, "_on", lambda stream, device: (0, None))
    ctx = types.SimpleNamespace(handle=None, device=torch.device("cuda", 0))
    here, there = Fake("cuda:0", torch.float64), Fake("cuda:1", torch.float64)
    norm = Fake("cuda:1", torch.float32)
    for call in (lambda: gb.gac_clip_grad_norm(ctx, 1.0, norm_out=norm), lambda: gb.gac_clip_sumsq(ctx, there),
                 lambda: gb.gac_clip_apply(ctx, there, 1.0), lambda: gb.gac_clip_apply(ctx, here, 1.0, norm_out=norm)):
        with pytest.raises(ValueError):
            call()
