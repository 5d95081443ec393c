"""A workspace that a call makes for itself on a given stream is that stream's memory, on the host: the allocation happens
while the stream is torch's current one, since memory freed on another stream may still be written there."""
import contextlib

import pytest
import torch

from paper_2609_24456_amd import conduit as cd


class _Log:
    """Stands for the device: the stream that is current at each allocation, and the stream of each clear."""

    def __init__(self, monkeypatch):
        self.current, self.allocated, self.cleared = ["torch's current"], [], []
        empty = torch.empty

        @contextlib.contextmanager
        def stream(s):
            self.current.append(s)
            yield
            self.current.pop()

        def allocate(n, dtype, device):
            self.allocated.append(self.current[-1])
            return empty(n, dtype=dtype)

        monkeypatch.setattr(torch, "empty", allocate)
        monkeypatch.setattr(torch.cuda, "stream", stream)
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: handle)
        monkeypatch.setattr(torch.cuda, "default_stream", lambda: "default")
        monkeypatch.setattr(cd, "_stream", lambda s: s)
        monkeypatch.setattr(cd, "_on_device", lambda t: True)
        monkeypatch.setattr(cd, "lib", lambda: self)

    def conduit_workspace_init(self, p, n, stream):
        self.cleared.append(stream)
        return cd.OK


@pytest.mark.parametrize("stream,current", [(0x7000, 0x7000), (0, "default"), (None, "torch's current")])
def test_a_new_workspace_is_allocated_on_its_stream(monkeypatch, stream, current):
    log = _Log(monkeypatch)
    cd.workspace(1000, stream=stream)
    cd._workspace(None, lambda: 1000, stream)
    assert log.allocated == [current, current] and log.cleared == [stream, stream]
    assert log.current == ["torch's current"]


def test_a_caller_s_workspace_is_taken_as_it_is(monkeypatch):
    log = _Log(monkeypatch)
    ws = torch.zeros(512, dtype=torch.uint8)
    got, p, n = cd._workspace(ws, lambda: pytest.fail("its size is not asked for"), 0x7000)
    assert got is ws and p == ws.data_ptr() and n == 512 and not log.allocated and not log.cleared
