"""The binding's own scratch: one buffer for each stream, none shared with a graph (no GPU needed)."""
import contextlib

import pytest
import torch

import paper_2609_33390_amd as brisk

CPU = torch.device("cpu", 0)


class Stream:
    """A stream as the binding sees it."""

    def __init__(self, handle):
        self.cuda_stream = handle


@pytest.fixture
def streams(monkeypatch):
    """The current stream's handle and whether it is captured, without a GPU."""
    now = {"handle": 1, "capturing": False}

    @contextlib.contextmanager
    def enter(s):
        before, now["handle"] = now["handle"], s.cuda_stream
        yield
        now["handle"] = before

    monkeypatch.setattr(brisk, "_ws", {})
    monkeypatch.setattr(brisk, "_raw_stream", lambda index: now["handle"])
    monkeypatch.setattr(brisk, "_capturing", lambda: now["capturing"])
    monkeypatch.setattr(torch.cuda, "stream", enter)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: Stream(handle))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: Stream(0))
    return now


def _get(nbytes, stream=None, tag="op"):
    return brisk._workspace(CPU, nbytes, tag, stream)


def test_each_stream_has_its_own(streams):
    a = _get(1000)
    streams["handle"] = 2
    b = _get(1000)
    assert a.data_ptr() != b.data_ptr()
    assert _get(1000).data_ptr() == b.data_ptr()
    assert _get(500, Stream(1)).data_ptr() == a.data_ptr()
    assert _get(500, 1).data_ptr() == a.data_ptr()
    assert _get(500, 2).data_ptr() == b.data_ptr()
    c = _get(1000, 0)
    assert c.data_ptr() not in (a.data_ptr(), b.data_ptr())
    assert _get(1000, tag="other").data_ptr() not in (a.data_ptr(), b.data_ptr(), c.data_ptr())


def test_growth_on_one_stream_leaves_the_others(streams):
    a, b = _get(1000), _get(1000, 2)
    grown = _get(5000, 2)
    assert grown.numel() >= 5000 and _get(1000, 2).data_ptr() == grown.data_ptr()
    assert _get(1000).data_ptr() == a.data_ptr() and b.numel() >= 1000


def test_buffers_are_made_on_the_stream_that_uses_them(streams, monkeypatch):
    made, empty = [], torch.empty

    def record(*args, **kw):
        made.append(streams["handle"])
        return empty(*args, **kw)

    monkeypatch.setattr(torch, "empty", record)
    _get(1000)
    _get(1000, 7)
    _get(1000, Stream(8))
    assert made == [1, 7, 8] and streams["handle"] == 1


def test_captured_calls_keep_to_the_graph(streams):
    a = _get(1000)
    streams["capturing"] = True
    g, h = _get(1000), _get(1000)
    assert len({x.data_ptr() for x in (a, g, h)}) == 3
    streams["capturing"] = False
    assert _get(1000).data_ptr() == a.data_ptr()
