"""Streams that the expert layer's calls are given (on the host)."""
import types

import pytest
import torch

from paper_2103_16716_amd import experts


def test_a_stream_of_another_device_is_refused(monkeypatch):
    """Its kernels would run on a device that the tensors are not on."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="stream is on cuda:1, the current device is cuda:0"):
        experts._on(types.SimpleNamespace(device_index=1, cuda_stream=0))
    experts._on(types.SimpleNamespace(device_index=0, cuda_stream=0))
    assert experts._on(None) is experts._current
