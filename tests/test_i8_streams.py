"""A stream of another device than the current one is refused (no GPU: the devices are
stand-ins, and nothing is called)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2608_23167_amd import api


@pytest.fixture
def on_device_1(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)


@pytest.mark.parametrize("index", [0, 2])
def test_stream_of_another_device(on_device_1, index):
    with pytest.raises(ValueError, match=f"stream must be of the current device.*cuda:1.*cuda:{index}"):
        api._on(SimpleNamespace(cuda_stream=7, device_index=index))


def test_stream_of_the_current_device(on_device_1):
    assert api._on(SimpleNamespace(cuda_stream=7, device_index=1)) == 7


def test_tensor_of_another_device(on_device_1):
    with pytest.raises(ValueError, match="current device"):
        api._on(SimpleNamespace(cuda_stream=7, device_index=1), torch.zeros(1))
