"""Where the binding of the compact cache takes the current stream and device from: torch's short ways, and the
public ones in a torch that lacks them (no GPU)."""
from types import SimpleNamespace

import pytest

import paper_2607_05061_amd as kv


def _torch(short):
    entered = []

    class Device:
        def __init__(self, dev):
            self.dev = dev

        def __enter__(self):
            entered.append(self.dev)

        def __exit__(self, *a):
            entered.append("left")

    own = SimpleNamespace(_cuda_getCurrentRawStream=lambda d: 100 + d, _cuda_getDevice=lambda: 1) if short else SimpleNamespace()
    cuda = SimpleNamespace(current_stream=lambda d: SimpleNamespace(cuda_stream=100 + d), current_device=lambda: 1, device=Device)
    return SimpleNamespace(_C=own, cuda=cuda), entered


@pytest.mark.parametrize("short", [True, False])
def test_current_stream_and_device(short):
    torch, entered = _torch(short)
    got = []
    f = lambda *a: got.append(a) or 0  # noqa: E731
    kv._call(torch, f, 1, None, "x")
    assert got == [("x", 101)] and entered == []
    kv._call(torch, f, 0, None, "y")  # another device than the current one
    assert got[1:] == [("y", 100)] and entered == [0, "left"]
    kv._call(torch, f, 1, SimpleNamespace(cuda_stream=7))
    assert got[2:] == [(7,)]
