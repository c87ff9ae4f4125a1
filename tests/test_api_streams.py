"""Whose memory the tensor-level wrappers allocate, on the host: torch's
streams and the launches are replaced by records, so nothing runs on a GPU."""
import contextlib

import pytest


class Streams:
    """The stack of streams that allocations belong to, and what was asked for."""

    def __init__(self):
        self.stack = ["current"]

    @contextlib.contextmanager
    def use(self, stream):
        self.stack.append(stream)
        yield
        self.stack.pop()


@pytest.fixture
def streams(monkeypatch):
    import torch
    s = Streams()

    def external(handle):
        assert handle != 0, "a zero handle does not name the default stream here: torch takes a stream of its pool"
        return ("external", handle)

    monkeypatch.setattr(torch.cuda, "stream", s.use)
    monkeypatch.setattr(torch.cuda, "ExternalStream", external)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda *a: "default")
    empty = torch.empty
    s.made = []

    def record(*args, **kw):
        t = empty(*args, **kw)
        s.made.append((tuple(t.shape), s.stack[-1]))
        return t

    monkeypatch.setattr(torch, "empty", record)
    return s


@pytest.mark.parametrize("given,owner", [(None, "current"), (0, "default"), (64, ("external", 64)), ("side", "side")])
def test_a_workspace_belongs_to_the_calls_stream(streams, given, owner):
    from paper_2011_11188_amd import api
    api._scratch(48, "cpu", given)
    assert streams.made == [((48,), owner)]
    assert streams.stack == ["current"]
