"""Whose pool the hidden buffer of a list of gradients comes from, and which streams the allocator is told of.  Needs no GPU: nothing is enqueued."""
import contextlib

import pytest
import torch

from paper_2101_07706_amd import csgs


class Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


CURRENT, SIDE, OTHER = Stream(1), Stream(2), Stream(3)


@pytest.fixture
def seen(monkeypatch):
    """What was allocated under which stream, which streams were recorded on it, and the library's calls with theirs."""
    stack, seen = [CURRENT], {"allocated": [], "recorded": [], "calls": []}

    @contextlib.contextmanager
    def under(stream):
        stack.append(stack[-1] if stream is None else stream)
        yield
        stack.pop()

    empty = torch.empty

    def allocate(*shape, **kw):
        t = empty(*shape, **kw)
        seen["allocated"].append((t.data_ptr(), stack[-1].cuda_stream))
        return t

    monkeypatch.setattr(torch.cuda, "stream", under)
    monkeypatch.setattr(torch, "empty", allocate)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: seen["recorded"].append((t.data_ptr(), s.cuda_stream)))
    monkeypatch.setattr(csgs, "_torch_stream", lambda s: stack[-1] if s is None else s, raising=False)
    monkeypatch.setattr(csgs, "_stream", lambda s: (stack[-1] if s is None else s).cuda_stream)
    monkeypatch.setattr(csgs, "_call", lambda name, *args: seen["calls"].append((name, args[-1])))
    return seen


def calls(l, stream):
    total = torch.zeros(1, dtype=torch.float64)
    csgs.csgs_grad_norm(l, csgs.GRAD_L2, total, stream=stream)
    csgs.csgs_grad_scale(l, csgs.GRAD_L2, total, 1.0, stream=stream)
    csgs.csgs_grad_clip(l, csgs.GRAD_L2, 1.0, stream=stream)


@pytest.mark.parametrize("stream", [None, SIDE])
def test_buffer_belongs_to_the_stream_that_fills_it(seen, stream):
    l = csgs.make_grad_list([torch.ones(4, 3)], stream=stream)
    own = (stream or CURRENT).cuda_stream
    assert seen["allocated"] == [(l.base, own)] and seen["calls"] == [("csgs_grad_list_init", own)]
    calls(l, stream)
    assert [s for _, s in seen["calls"]] == [own] * 4
    assert set(seen["recorded"]) <= {(l.base, own)}      # (nothing needs to be said of a buffer's own stream)


@pytest.mark.parametrize("made_on,used_on", [(None, SIDE), (SIDE, None), (SIDE, OTHER)])
@pytest.mark.parametrize("call", range(3))
def test_other_streams_are_recorded_before_they_use_it(seen, made_on, used_on, call):
    l = csgs.make_grad_list([torch.ones(4, 3)], stream=made_on)
    total = torch.zeros(1, dtype=torch.float64)
    [lambda: csgs.csgs_grad_norm(l, csgs.GRAD_L2, total, stream=used_on), lambda: csgs.csgs_grad_scale(l, csgs.GRAD_L2, total, 1.0, stream=used_on),
     lambda: csgs.csgs_grad_clip(l, csgs.GRAD_MAX, 1.0, stream=used_on)][call]()
    assert seen["recorded"] == [(l.base, (used_on or CURRENT).cuda_stream)]
    calls(l, used_on)
    assert len(seen["recorded"]) == 1                    # once a stream


def test_a_call_that_is_recorded_for_later(seen, monkeypatch):
    """A plan runs on the stream that it was recorded for."""
    l = csgs.make_grad_list([torch.ones(4, 3)])
    monkeypatch.undo()                                   # the plan takes the calls themselves
    monkeypatch.setattr(csgs, "_torch_stream", lambda s: s, raising=False)
    recorded = []
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: recorded.append((t.data_ptr(), s.cuda_stream)))
    with csgs.record() as plan:
        csgs.csgs_grad_clip(l, csgs.GRAD_L2, 1.0, stream=SIDE)
    assert recorded == [(l.base, SIDE.cuda_stream)] and len(plan.calls) == 1
