"""The text operators' objects and streams: what they do on the host around a call, with the
device's part played by stand-ins (no GPU needed)."""
import contextlib

import pytest
import torch

from paper_2607_16074_gb300 import jnx as J
from paper_2607_16074_gb300 import runtime as R


class Status:
    """A status word that kernels still running on some stream report to: what they report
    is there once the device has been waited for, and a reset takes place in its turn."""

    def __init__(self):
        self.value, self.pending, self.log = 0, [], []

    def synchronize(self, device=None):
        self.log.append("wait")
        for change in self.pending:
            self.value = change(self.value)
        self.pending = []

    def report(self, code):
        self.pending.append(lambda v: v or code)

    def item(self):
        return self.value

    def zero_(self):
        self.pending.append(lambda v: 0)


@pytest.fixture
def operator(monkeypatch):
    op = R._TextOperator.__new__(R._TextOperator)
    op.status, op._device = Status(), 0
    monkeypatch.setattr(torch.cuda, "synchronize", op.status.synchronize)
    return op


def test_check_waits_for_what_it_checks(operator):
    operator.status.report(J.JNX_ERR_DEVICE_BOUNDS)
    with pytest.raises(J.JnxError) as e:
        operator.check()
    assert e.value.code == J.JNX_ERR_DEVICE_BOUNDS
    operator.check()


def test_check_wipes_no_later_report(operator):
    operator.status.report(J.JNX_ERR_TIMEOUT)
    with pytest.raises(J.JnxError):
        operator.check()
    assert not operator.status.pending  # the word is cleared before check returns
    operator.status.report(J.JNX_ERR_DEVICE_BOUNDS)
    with pytest.raises(J.JnxError) as e:
        operator.check()
    assert e.value.code == J.JNX_ERR_DEVICE_BOUNDS


class Memory:
    def __init__(self):
        self.streams = []

    def record_stream(self, stream):
        self.streams.append(stream.cuda_stream)


class Stream:
    def __init__(self, handle):
        self.cuda_stream, self.waited = handle, []

    def wait_event(self, event):
        self.waited.append(event)


@pytest.fixture
def made_on_11(monkeypatch):
    op = R._TextOperator.__new__(R._TextOperator)
    op._device, op._held, op._known, op._made = 0, [Memory(), Memory()], {11}, "made"
    op.capturing = False
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: op.capturing)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 11, raising=False)
    return op


def test_memory_is_known_to_every_stream_that_uses_it(made_on_11):
    op, other = made_on_11, Stream(22)
    assert op._on(None) == 11 and op._on(Stream(11)) == 11
    assert not any(m.streams for m in op._held)  # the allocator knows of its own stream
    for _ in range(3):
        assert op._on(other) == 22
    assert all(m.streams == [22] for m in op._held) and other.waited == ["made"]


def test_a_capturing_stream_does_not_wait_for_what_lies_outside(made_on_11):
    op, other = made_on_11, Stream(22)
    op.capturing = True
    assert op._on(other) == 22
    assert all(m.streams == [22] for m in op._held) and not other.waited
    op.capturing = False
    op._on(other)
    assert other.waited == ["made"]
