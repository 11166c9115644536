"""The binding's workspace and streams, on stand-ins for torch's streams and events: the zero-fill is
queued where the call that needs it runs, calls on other streams wait for it once, and
memory in use there is not handed out again."""
import contextlib

import pytest
import torch


class Stream:
    def __init__(self, handle, log):
        self.cuda_stream, self.log = handle, log

    def wait_event(self, e):
        self.log.append(("wait", self.cuda_stream, e.on))


class Buffer:
    def __init__(self, n, log, now):
        self.n, self.log, self.now = n, log, now

    def __getitem__(self, word):
        assert word == slice(None, 4)
        return self

    def copy_(self, other):
        self.log.append(("copy", self.n, other.n, self.now[-1].cuda_stream))

    def data_ptr(self):
        return 4096 * (1 + self.n)

    def numel(self):
        return self.n

    def record_stream(self, s):
        self.log.append(("keep", self.n, s.cuda_stream))


@pytest.fixture
def fake(monkeypatch):
    from paper_2609_15359_gb300 import build
    build.build()
    from paper_2609_15359_gb300 import maps as M
    log, now = [], []
    now.append(Stream(1, log))
    capturing = []

    @contextlib.contextmanager
    def on(s):
        now.append(s)
        yield
        now.pop()

    class Event:
        def record(self, s):
            self.on = s.cuda_stream

    def zeros(n, dtype=None, device=None):
        log.append(("zeros", n, now[-1].cuda_stream))
        return Buffer(n, log, now)

    monkeypatch.setattr(torch, "zeros", zeros)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "Event", Event)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[-1])
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: bool(capturing))
    monkeypatch.setattr(M, "_stream", lambda s: (now[-1] if s is None else s).cuda_stream)
    return M, log, now, capturing


def test_a_call_on_another_stream_waits_for_the_zero_fill(fake):
    M, log, _, _ = fake
    ws, side = M.Workspace(1000), Stream(2, log)
    assert log == [("zeros", 1000, 1)]
    for _ in range(3):
        got, handle = M._scratch(ws, 500, side)
        assert got is ws and handle == 2
    assert log[1:] == [("wait", 2, 1), ("keep", 1000, 2)]
    assert M._scratch(ws, 500, None) == (ws, 1) and len(log) == 3


def test_growth_is_on_the_stream_of_the_call(fake):
    M, log, _, _ = fake
    ws, side = M.Workspace(), Stream(2, log)
    _, handle = M._scratch(ws, 5000, side)
    assert handle == 2 and ws.nbytes == 5000 and ("zeros", 5000, 2) in log
    log.clear()
    M._scratch(ws, 5000, side)
    assert log == []
    M._scratch(ws, 4000, None)  # and now the first stream waits
    assert log == [("wait", 1, 2), ("keep", 5000, 1)]


def test_a_temporary_workspace_belongs_to_the_stream_of_the_call(fake):
    M, log, _, _ = fake
    ws, handle = M._scratch(None, 700, Stream(3, log))
    assert handle == 3 and log == [("zeros", 700, 3)] and ws.known == {3}


def test_a_captured_call_waits_for_nothing_outside_its_graph(fake):
    M, log, now, capturing = fake
    ws = M.Workspace(1000)
    now.append(Stream(5, log))
    capturing.append(1)
    M._scratch(ws, 1000, None)
    assert log[1:] == [("keep", 1000, 5)]


def test_growth_keeps_the_recorded_error(fake):
    """The status that an earlier call recorded is not lost where a later call needs more."""
    M, log, _, _ = fake
    ws, side = M.Workspace(), Stream(2, log)
    M._scratch(ws, 5000, side)
    assert log == [("zeros", 256, 1), ("wait", 2, 1), ("keep", 256, 2), ("zeros", 5000, 2), ("copy", 5000, 256, 2)]


def test_attention_asks_for_its_workspace_on_every_device(fake, monkeypatch):
    """The size grows with a device's multiprocessors: one device's does not serve another."""
    M, _, _, _ = fake
    device, asked = [0], []
    monkeypatch.setattr(torch.cuda, "current_device", lambda: device[0])
    monkeypatch.setattr(M.lib, "maps_kv4_attention_workspace_size", lambda *sizes: 1000 * (1 + device[0]))

    class Enough(Exception):
        pass

    def scratch(ws, nbytes, stream):
        asked.append(nbytes)
        raise Enough

    monkeypatch.setattr(M, "_scratch", scratch)
    q, cache = torch.empty(3, 4, 64), torch.empty(5, 2, 1152, dtype=torch.uint8)
    for device[0] in (0, 1, 0, 1):
        with pytest.raises(Enough):
            M.maps_kv4_attention(q, torch.empty(3), torch.empty(2), torch.empty(2, 4), cache, 16, 0.1, torch.empty(3, 4, 64))
    assert asked == [1000, 2000, 1000, 2000]


def test_the_current_stream_without_the_private_function(monkeypatch):
    """The binding loads and finds the current stream on a PyTorch that lacks the function it prefers."""
    import importlib.util

    from paper_2609_15359_gb300 import maps as M
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    spec = importlib.util.spec_from_file_location("maps_without", M.__file__)
    other = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(other)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream(17, []))
    assert other._stream(None) == 17 and other._stream(Stream(5, [])) == 5


def test_pointer_and_size_are_the_buffers():
    """`ptr` is a pointer for any ctypes call, one without declared arguments too, and follows a buffer that its owner puts in."""
    import ctypes

    from paper_2609_15359_gb300 import maps as M
    ws = M.Workspace(1000, device="cpu")
    assert isinstance(ws.ptr, ctypes.c_void_p) and ws.ptr.value == ws.buf.data_ptr() and ws.nbytes == 1000
    mine = torch.zeros(4096, dtype=torch.uint8)
    ws.buf = mine
    assert ws.buf is mine and ws.ptr.value == mine.data_ptr() and ws.nbytes == 4096
    ws.ensure(5000)
    assert ws.nbytes == 5000 == ws.buf.numel() and ws.ptr.value == ws.buf.data_ptr()
