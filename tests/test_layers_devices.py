"""A layer's description belongs to the device that its tensors lie on (no GPU: calls that are refused before the library is reached)."""

import pytest
import torch

from paper_2605_21177_amd import binding as B

from test_layers_host import _OnDevice


def test_a_description_of_another_device_is_refused(monkeypatch):
    current = [0]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    monkeypatch.setattr(B, "lib", lambda: pytest.fail("the library is reached"))
    t = lambda *s: _OnDevice(torch.zeros(*s), current[0])  # noqa: E731
    norm, linear = B.make_norm(B.LAYERNORM, t(4, 16), t(16), t(16)), B.make_linear(t(4, 16), t(24, 16))
    current[0] = 1
    y, z = t(4, 16), t(4, 24)
    for call in (lambda: B.chunkft_norm_forward(norm, y), lambda: B.chunkft_norm_backward(norm, t(4, 2), y, y),
                 lambda: B.chunkft_linear_forward(linear, z), lambda: B.chunkft_linear_backward(linear, z, dX=y)):
        with pytest.raises(ValueError, match="current device"):
            call()
