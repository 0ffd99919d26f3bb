"""The linear layers' device status is asked on the device of the stream that is given, whichever device is current."""
import contextlib

import pytest
import torch

from paper_2503_06671_b200 import binding


class Stream:
    cuda_stream = 1234

    def __init__(self, index):
        self.device = torch.device("cuda", index)


class Library:
    """Notes which device was current, and which stream was handed on, at each call."""

    def __init__(self):
        self.calls, self.current = [], 0

    def esc_linear_device_status(self, stream):
        self.calls.append((self.current, stream.value))
        return 0

    esc_linear_selftest_bounded_wait = esc_linear_device_status


@pytest.fixture
def library(monkeypatch):
    fake = Library()

    @contextlib.contextmanager
    def device(d):
        before, fake.current = fake.current, d.index
        yield
        fake.current = before

    monkeypatch.setattr(binding, "lib", lambda: fake)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: fake.current)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream(fake.current))
    return fake


@pytest.mark.parametrize("call", [binding.esc_linear_device_status, binding.esc_linear_selftest_bounded_wait])
def test_status_of_the_streams_device(library, call):
    call()
    call(Stream(0))
    call(Stream(1))
    assert library.calls == [(0, 1234), (0, 1234), (1, 1234)] and library.current == 0
