"""The binding's streams are the current device's: tensors of another device are refused."""
from types import SimpleNamespace

import pytest
import torch

from paper_2609_32398_gb300 import doloss as dl


def test_the_stream_of_a_device_that_is_not_current_is_refused(monkeypatch):
    """The default streams of all devices have one handle, which stands for the current device's."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device: SimpleNamespace(cuda_stream=7 + device.index))
    at = lambda i: SimpleNamespace(device=torch.device("cuda", i))  # noqa: E731
    assert dl._stream(at(0)) == 7
    with pytest.raises(ValueError, match="current device"):
        dl._stream(at(1))


@pytest.mark.parametrize("call", ["forward_backward_host", "forward_backward_host_async"])
def test_the_buffer_of_a_host_call_too(monkeypatch, call):
    """The host calls take their stream from the device buffer."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device: SimpleNamespace(cuda_stream=0))

    def launch(*args):
        raise AssertionError("launched")

    monkeypatch.setattr(dl, "lib", lambda: SimpleNamespace(do_forward_backward_host=launch,
                                                           do_forward_backward_host_async=launch))
    z, buffer = torch.zeros(4, 8), SimpleNamespace(device=torch.device("cuda", 1), data_ptr=lambda: 256, numel=lambda: 1)
    with pytest.raises(ValueError, match="current device"):
        if call == "forward_backward_host":
            dl.forward_backward_host(z, 2, device_buffer=buffer)
        else:
            dl.forward_backward_host_async(z, 2, torch.zeros(64), buffer)
