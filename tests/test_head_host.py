"""How the 4-bit output projection orders streams, with streams and a context that only take notes (no GPU)."""
import contextlib

import pytest
import torch

from paper_2406_11257_amd import head


class Notes:
    def __init__(self, name, log):
        self.name, self.log = name, log

    def wait_stream(self, other):
        self.log.append((self.name, other.name))


class Refuses:
    """A context whose operators are refused from the `after`-th on."""
    device = torch.device("cpu")

    def __init__(self, stream, after):
        self._stream, self.left, self.calls = stream, after, []

    def __getattr__(self, name):
        if not name.startswith("excp_"):
            raise AttributeError(name)

        def call(*a):
            if self.left == 0:
                raise TypeError(name)
            self.left -= 1
            self.calls.append(name)
        return call


@pytest.fixture
def streams(monkeypatch):
    log = []
    own, caller = Notes("own", log), Notes("caller", log)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: caller)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    return own, log


@pytest.mark.parametrize("after", [1, 2])
def test_a_refusal_leaves_the_callers_stream_behind_what_was_queued(streams, after):
    own, log = streams
    ctx = Refuses(own, after)
    hd = head.MxHead(ctx, torch.zeros(6, 4))
    log.clear()
    with pytest.raises(TypeError):
        hd.score(torch.zeros(2, 4), torch.zeros(2, dtype=torch.int32))
    assert log == [("own", "caller"), ("caller", "own")] and len(ctx.calls) == after
