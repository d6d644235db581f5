"""Checks of the dense operators' bindings that need more than one GPU, on stand-ins for tensors (no GPU)."""
import types

import pytest
import torch

from paper_2010_11305_amd import mx4


def stand_in(shape, index):
    return types.SimpleNamespace(shape=shape, dtype=torch.uint8, is_cuda=True, is_contiguous=lambda: True,
                                 device=torch.device("cuda", index), data_ptr=lambda: 0)


def test_codes_and_scales_on_two_devices(monkeypatch):
    called = []
    monkeypatch.setattr(mx4, "_target", lambda out, rows, cols, device, what: types.SimpleNamespace(data=stand_in((1,), 0), device=device))
    monkeypatch.setattr(mx4.lib, "call", lambda *a: called.append(a))
    with pytest.raises(ValueError, match="one device"):
        mx4.from_codes(stand_in((4, 20), 0), stand_in((4, 2), 1), 40)
    assert not called
    mx4.from_codes(stand_in((4, 20), 1), stand_in((4, 2), 1), 40)
    assert len(called) == 1
