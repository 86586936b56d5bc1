"""A tensor on another device than the current one is refused before a launch (on the host: a device number is all that is
looked at)."""
import pytest
import torch

import paper_2609_15039_amd as sp


class Far(torch.Tensor):
    """Says that it is on device 1."""
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 1


def test_tile_experts(monkeypatch):
    launched = []
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(sp, "splitee_tile_weights", lambda *a, **k: launched.append(a))
    W = torch.zeros(2, 32, 64, dtype=torch.bfloat16).as_subclass(Far)
    with pytest.raises(ValueError, match="on device 1, the current device is 0"):
        sp.tile_experts(W)
    assert not launched
