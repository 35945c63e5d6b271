"""Where calls find the current device and stream: plain numbers of torch's own, or its public names."""
import importlib.util

import pytest
import torch

from paper_2008_01425_amd import device


def loaded():
    spec = importlib.util.spec_from_file_location("paper_2008_01425_amd.device_again", device.__file__)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_a_torch_without_the_plain_numbers(monkeypatch):
    for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
        monkeypatch.delattr(torch._C, name, raising=False)
    module = loaded()
    assert module._current_device is torch.cuda.current_device
    asked = []

    class Stream:
        cuda_stream = 7
    monkeypatch.setattr(torch.cuda, "current_stream", lambda index: asked.append(index) or Stream)
    assert module._current_stream(3) == 7 and asked == [3]


@pytest.mark.gpu
def test_the_plain_numbers_are_those_of_the_public_names():
    side = torch.cuda.Stream()
    for stream in (torch.cuda.default_stream(), side):
        with torch.cuda.stream(stream):
            assert device._current_device() == torch.cuda.current_device()
            assert device._current_stream(torch.cuda.current_device()) == torch.cuda.current_stream().cuda_stream == stream.cuda_stream
