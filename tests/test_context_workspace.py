"""Which workspaces a context keeps and which stream it binds (CPU: torch's allocations
and streams are stand-ins)."""
import gc
import weakref

import pytest

import paper_2608_08751_amd as ivf
from paper_2608_08751_amd import _binding


class Memory:
    """What torch.empty returns here."""

    def __init__(self, size):
        self.size, self.streams = size, []

    def numel(self):
        return self.size

    def data_ptr(self):
        return 0x7F0000000000

    def record_stream(self, stream):
        self.streams.append(stream)


class Device:
    stream, capturing = 1, False


@pytest.fixture()
def device(monkeypatch):
    import torch

    state = Device()
    monkeypatch.setattr(torch, "empty", lambda size, **_: Memory(size))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: state.capturing)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: state.stream)
    monkeypatch.setattr(_binding, "_stream_handle", lambda device=None: state.stream)
    return state


@pytest.fixture()
def vctx():
    ctx = ivf.Context(-1)
    yield ctx
    ctx.close()


def test_a_workspace_of_a_captured_call_is_kept(vctx, device):
    vctx.ensure_workspace(2 << 20)  # before the capture, as a program sizes it
    device.capturing = True
    vctx.ensure_workspace(2 << 20)
    device.capturing = False
    first = weakref.ref(vctx._ws)
    vctx.ensure_workspace(4 << 20)
    second = weakref.ref(vctx._ws)
    device.capturing = True
    vctx.ensure_workspace(8 << 20)  # grows inside a capture
    device.capturing = False
    third = weakref.ref(vctx._ws)
    vctx.ensure_workspace(16 << 20)
    gc.collect()
    assert first() is not None and third() is not None
    assert second() is None  # no capture has used it
    assert vctx._ws.numel() == 16 << 20


def test_a_workspace_without_capture_is_let_go(vctx, device):
    vctx.ensure_workspace(2 << 20)
    first = weakref.ref(vctx._ws)
    vctx.ensure_workspace(1 << 20)
    assert vctx._ws is first()  # large enough
    vctx.ensure_workspace(4 << 20)
    gc.collect()
    assert first() is None


def test_every_stream_that_uses_a_workspace_is_known(vctx, device):
    vctx.ensure_workspace(2 << 20)
    ws = vctx._ws
    assert ws.streams == []  # of its own stream torch knows
    for device.stream in (2, 1, 2, 3):
        vctx.ensure_workspace(1 << 20)
    assert ws.streams == [2, 3]
    vctx.ensure_workspace(4 << 20)  # allocated on stream 3
    ws = vctx._ws
    for device.stream in (3, 1):
        vctx.ensure_workspace(1 << 20)
    assert ws.streams == [1]


def test_bind_follows_torch_after_the_handle_was_given_another_stream(vctx, device):
    class Recorder:
        def __init__(self, lib):
            self.lib, self.stream = lib, None

        def __getattr__(self, name):
            return getattr(self.lib, name)

        def ivf_set_stream(self, handle, stream):
            self.stream = stream
            return self.lib.ivf_set_stream(handle, stream)

    lib = vctx.lib = Recorder(vctx.lib)
    device.stream = 64
    vctx.bind()
    assert lib.stream == 64
    vctx.lib.ivf_set_stream(vctx.handle, 128)
    vctx.bind()
    assert lib.stream == 64
