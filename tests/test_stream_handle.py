"""How the binding finds torch's current stream, with a torch of its own making (no GPU)."""
import sys
from types import SimpleNamespace

import pytest

from tests.libqe import need_lib


class Torch:
    """Current device and stream handle, and the raw accessors as `private` gives them."""

    def __init__(self, private):
        self.device, self.handle, self.objects = 0, 0x70, 0
        self.cuda = SimpleNamespace(current_stream=self._stream)
        self._C = private(self)

    def _stream(self):
        self.objects += 1
        return SimpleNamespace(cuda_stream=self.handle)


def renamed(t):
    return SimpleNamespace()


def other_arguments(t):
    return SimpleNamespace(_cuda_getDevice=lambda: t.device, _cuda_getCurrentRawStream=lambda: t.handle)


def other_answer(t):
    return SimpleNamespace(_cuda_getDevice=lambda: t.device, _cuda_getCurrentRawStream=lambda device: (t.handle, device))


def as_known(t):
    return SimpleNamespace(_cuda_getDevice=lambda: t.device, _cuda_getCurrentRawStream=lambda device: t.handle + device)


@pytest.mark.parametrize("private", [renamed, other_arguments, other_answer, as_known])
def test_current_stream(private, monkeypatch):
    qe = need_lib()
    fake = Torch(private)
    monkeypatch.setitem(sys.modules, "torch", fake)
    monkeypatch.setattr(qe, "_current_stream", None)
    for handle in (0x70, 0x80, 0):
        fake.handle = handle
        assert qe.stream_handle(None) == handle
    assert (fake.objects == 1) == (private is as_known)  # no Stream object a call where the raw accessors serve
    assert qe.stream_handle(5) == 5 and qe.stream_handle(SimpleNamespace(cuda_stream=9)) == 9


def test_a_failed_first_use_binds_nothing(monkeypatch):
    qe = need_lib()
    fake = Torch(as_known)
    monkeypatch.setitem(sys.modules, "torch", fake)
    monkeypatch.setattr(qe, "_current_stream", None)

    def none():
        raise RuntimeError("no GPU")
    monkeypatch.setattr(fake.cuda, "current_stream", none)
    with pytest.raises(RuntimeError):
        qe.stream_handle(None)
    monkeypatch.setattr(fake.cuda, "current_stream", fake._stream)
    assert qe.stream_handle(None) == 0x70 and qe.stream_handle(None) == 0x70 and fake.objects == 1
