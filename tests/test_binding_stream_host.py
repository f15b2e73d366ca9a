"""Which stream a call without one takes (no GPU: torch's own functions are replaced by ones that name what they were asked)."""
from types import SimpleNamespace

import pytest
import torch

import paper_2402_18789_amd.binding as B


@pytest.fixture
def device_2(monkeypatch):
    """device 2 is the current one; its current stream's handle is 7002"""
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 2)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: SimpleNamespace(cuda_stream=7002 if device is None else 7000 + device))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 2, raising=False)
    return monkeypatch


def test_the_current_devices_current_stream(device_2):
    device_2.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 7000 + i, raising=False)
    assert B._stream(None) == 7002


@pytest.mark.parametrize("gone", ["_cuda_getCurrentRawStream", "_cuda_getDevice"])
def test_without_the_short_way_to_its_handle(device_2, gone):
    """a torch that lacks the names: the public call"""
    device_2.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 7000 + i, raising=False)
    device_2.delattr(torch._C, gone)
    assert B._stream(None) == 7002


def test_before_the_device_is_in_use_and_with_a_stream_of_the_callers(monkeypatch):
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: SimpleNamespace(cuda_stream=41))
    assert B._stream(None) == 41
    assert B._stream(0) == 0 and B._stream(12) == 12 and B._stream(SimpleNamespace(cuda_stream=9)) == 9
