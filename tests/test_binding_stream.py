"""The stream that calls are put on: torch's current one, with or without the functions that give its handle directly."""
import types

import pytest
import torch

from paper_2507_03840_amd import binding as B


@pytest.mark.parametrize("gone", ["_device", "_raw_stream"])
def test_without_the_direct_functions(monkeypatch, gone):
    monkeypatch.setattr(B, gone, None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=1234))
    assert B._stream().value == 1234


def test_before_the_device_is_initialised(monkeypatch):
    """torch.cuda.current_stream() initialises the device (or says why it cannot); the direct functions would not."""
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=77))
    assert B._stream().value == 77


@pytest.mark.gpu
def test_current_stream(monkeypatch):
    torch.zeros(1, device="cuda")
    handle = lambda: (B._stream().value or 0, torch.cuda.current_stream().cuda_stream)
    side = torch.cuda.Stream()
    for _ in range(2):
        assert handle()[0] == handle()[1]
        with torch.cuda.stream(side):
            assert handle()[0] == handle()[1] == side.cuda_stream
        monkeypatch.setattr(B, "_raw_stream", None)
