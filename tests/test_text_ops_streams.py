"""The text operators' objects and streams: what they do on the host around a call, with the
device's part played by stand-ins (no GPU needed)."""
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
