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


def test_scores_give_their_gradients_once(streams):
    """The logits of scores become their gradient: a second call would take that for logits."""
    own, _ = streams
    ctx = Refuses(own, 1000)
    hd = head.MxHead(ctx, torch.zeros(6, 4), train=True)
    hidden, targets, g = torch.zeros(2, 4), torch.zeros(2, dtype=torch.int64), torch.ones(2)
    s = hd.score(hidden, targets)
    hd.gradients(hidden, targets, s, g)
    calls = len(ctx.calls)
    for again in (s, dict(s)):
        with pytest.raises(ValueError, match="score"):
            hd.gradients(hidden, targets, again, g)
    assert len(ctx.calls) == calls
    hd.gradients(hidden, targets, hd.score(hidden, targets), g)
    hd.gradients(hidden, targets, dict(s, logits=s["logits"].clone()), g)      # logits that were kept


@pytest.mark.parametrize("after", range(2, 8))
def test_scores_are_spent_where_their_gradient_was_queued(streams, after):
    own, _ = streams
    ctx = Refuses(own, 3)
    hd = head.MxHead(ctx, torch.zeros(6, 4), train=True)
    hidden, targets, g = torch.zeros(2, 4), torch.zeros(2, dtype=torch.int64), torch.ones(2)
    s = hd.score(hidden, targets)
    for wrong in (torch.zeros(3, 4), torch.zeros(2, 5)):
        with pytest.raises(ValueError, match="hidden"):
            hd.gradients(wrong, targets, s, g)
    assert len(ctx.calls) == 3
    ctx.left = after - 2
    with pytest.raises(TypeError) if after < 7 else contextlib.nullcontext():
        hd.gradients(hidden, targets, s, g)
    queued = "excp_token_logprobs_backward" in ctx.calls
    assert queued == (after > 3)                             # what may be refused of the hidden states comes before
    ctx.left = 1000
    with pytest.raises(ValueError) if queued else contextlib.nullcontext():
        hd.gradients(hidden, targets, s, g)
