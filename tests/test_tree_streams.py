"""Which stream a handle's calls go to and what they wait for (no GPU: streams that only record)."""
import contextlib

import pytest
import torch

from paper_2403_12900_amd.tree import TreeOps


class Stream:
    def __init__(self, raw):
        self.cuda_stream, self.waited = raw, []

    def wait_stream(self, other):
        self.waited.append(other.cuda_stream)


class World:
    """The current stream, and whether it is being captured; the handle under test and where its library puts work."""

    def __init__(self, monkeypatch):
        self.current, self.capturing, self.target = Stream(0), False, 0
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: self.current.cuda_stream, raising=False)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: self.current)
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: self.capturing)
        monkeypatch.setattr(torch.cuda, "device", lambda device: contextlib.nullcontext())
        world = self

        class Library:
            def spr_tree_ops_workspace_bytes(self):
                return 256

            def spr_tree_ops_init(self, ws, size, stream, out):
                return 0

            def spr_tree_ops_set_stream(self, h, raw):
                world.target = raw
                return 0

        class Workspace:
            def __init__(self):
                self.used = []

            def data_ptr(self):
                return 0

            def numel(self):
                return 256

            def record_stream(self, s):
                self.used.append(s.cuda_stream)

        monkeypatch.setattr("paper_2403_12900_amd.tree.load_library", Library)
        monkeypatch.setattr(torch, "empty", lambda *a, **k: Workspace())
        self.ops = TreeOps(0)

    def call(self, stream, capturing=False):
        """What the stream waited for in this call."""
        self.current, self.capturing = stream, capturing
        before = len(stream.waited)
        self.ops._enter()
        assert self.target == stream.cuda_stream
        return stream.waited[before:]


def test_eager_calls_wait_for_the_last_stream(monkeypatch):
    w = World(monkeypatch)
    a, b, zero = Stream(5), Stream(7), w.current
    assert w.call(zero) == []
    assert w.call(a) == [0] and w.call(a) == []
    assert w.call(b) == [5] and w.call(a) == [7] and w.call(zero) == [5]
    assert w.ops.ws.used == [5, 7, 5, 0]


@pytest.mark.parametrize("after", ["the capture's", "another", "the last eager one's"])
def test_a_capture_between_two_eager_calls(monkeypatch, after):
    """The capture itself waits for nothing; the next eager call waits for the last eager one, not for the captured."""
    w = World(monkeypatch)
    a, b, c = Stream(5), Stream(7), Stream(9)
    w.call(a)
    assert w.call(b, capturing=True) == [] and w.call(b, capturing=True) == []
    if after == "the capture's":
        assert w.call(b) == [5] and w.call(b) == []
    elif after == "another":
        assert w.call(c) == [5] and w.call(c) == [] and w.call(b) == [9]
    else:
        assert w.call(a) == [] and w.call(c) == [5]
