"""What LossHead gives the library, on the CPU: the entry points are recorded instead of run."""
import contextlib
import warnings
import weakref

import pytest
import torch


@pytest.fixture
def recorded(monkeypatch):
    """(losses, list of the calls' (workspace address, bytes))"""
    from paper_2502_16982_amd import binding, losses
    calls = []
    monkeypatch.setattr(losses, "stream_handle", lambda device: 7)
    monkeypatch.setattr(losses, "on", lambda device: contextlib.nullcontext())
    monkeypatch.setattr(losses, "capturing", lambda: False, raising=False)
    monkeypatch.setattr(losses, "current_stream", lambda device: None, raising=False)
    monkeypatch.setattr(binding, "muon_cross_entropy", lambda *a: calls.append((a[-3], a[-2])))
    monkeypatch.setattr(binding, "muon_distill", lambda *a: calls.append((a[-3], a[-2])))
    return losses, calls


def inputs(tokens, vocab, width, dtype=torch.bfloat16):
    return torch.zeros(tokens, width, dtype=dtype), torch.zeros(vocab, width, dtype=dtype), torch.zeros(tokens, dtype=torch.int64)


def teacher(tokens, top):
    return torch.zeros(tokens, top, dtype=torch.int32), torch.zeros(tokens, top)


def test_a_call_is_cut_alike_whatever_came_before(recorded):
    """The bytes that the library cuts a call by follow from the call, not from what a larger one left."""
    losses, calls = recorded
    args = inputs(9000, 600, 64)
    losses.LossHead(9000, 600, 64, device="cpu").cross_entropy(*args)
    used = losses.LossHead(9000, 600, 64, device="cpu")
    used.cross_entropy(*inputs(9000, 20000, 64))
    used.cross_entropy(*args)
    used.distill(*args[:2], *teacher(9000, 5))
    used.distill(*inputs(9000, 20000, 64)[:2], *teacher(9000, 5))
    used.distill(*args[:2], *teacher(9000, 5))
    assert calls[0][1] == calls[2][1] < calls[1][1]
    assert calls[3][1] == calls[5][1] < calls[4][1]


def test_a_workspace_that_a_captured_call_uses_stays(recorded, monkeypatch):
    """A graph holds the address: a larger call gets other memory, and what the graph writes to is not given back."""
    losses, calls = recorded
    capturing = [False]
    monkeypatch.setattr(losses, "capturing", lambda: capturing[0], raising=False)
    head = losses.LossHead(16, 100, 32, device="cpu")
    head.cross_entropy(*inputs(16, 100, 32))
    capturing[0] = True
    head.cross_entropy(*inputs(16, 100, 32))
    capturing[0] = False
    first, address = weakref.ref(head.workspace), calls[-1][0]
    head.distill(*inputs(16, 5000, 32)[:2], *teacher(16, 500))
    assert calls[-1][0] != address and first() is not None
    second = weakref.ref(head.workspace)
    head.distill(*inputs(16, 50000, 32)[:2], *teacher(16, 500))          # no graph holds the second one
    assert first() is not None and second() is None


def test_a_workspace_makes_room_before_the_next_one(recorded, monkeypatch):
    """Growing never holds two workspaces, and calls of the declared size do not grow it: distillation up to the entries declared."""
    losses, calls = recorded
    head = losses.LossHead(16, 100, 32, device="cpu")
    before = head.workspace.data_ptr()
    head.cross_entropy(*inputs(16, 100, 32))
    head.distill(*inputs(16, 100, 32)[:2], *teacher(16, 64))
    assert [c[0] for c in calls] == [before, before]
    more = losses.LossHead(16, 100, 32, device="cpu", top=300)
    before = more.workspace.data_ptr()
    more.distill(*inputs(16, 100, 32)[:2], *teacher(16, 300))
    assert calls[-1][0] == before

    old, empty, left = weakref.ref(head.workspace), torch.empty, []

    def spy(*size, **kw):
        if kw.get("dtype") == torch.uint8:
            left.append(old())
        return empty(*size, **kw)

    monkeypatch.setattr(torch, "empty", spy)
    head.cross_entropy(*inputs(16, 5000, 32))
    assert left == [None]


class Stream:
    """Stands for a stream: which others it was made to wait for."""

    def __init__(self, handle):
        self.handle, self.waited = handle, []

    def wait_stream(self, other):
        self.waited.append(other.handle)


def test_calls_on_different_streams_wait_for_each_other(recorded, monkeypatch):
    """There is one workspace: a call on another stream than the one before comes after it, and the first one after whatever held the memory on
    the stream where it was allocated."""
    losses, _ = recorded
    now, captures, kept = [Stream(1)], [False], []
    monkeypatch.setattr(losses, "stream_handle", lambda device: now[0].handle)
    monkeypatch.setattr(losses, "current_stream", lambda device: now[0], raising=False)
    monkeypatch.setattr(losses, "capturing", lambda: captures[0])
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device: now[0])
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, stream: kept.append(stream.handle))
    first, second, third = now[0], Stream(2), Stream(3)
    head = losses.LossHead(16, 100, 32, device="cpu")
    head.cross_entropy(*inputs(16, 100, 32))
    assert first.waited == [] and kept == []
    now[0] = second
    head.cross_entropy(*inputs(16, 100, 32))
    head.cross_entropy(*inputs(16, 100, 32))
    assert second.waited == [1] and 2 in kept
    now[0], captures[0] = third, True                       # a capture begins behind everything, and cannot wait for what is outside
    head.cross_entropy(*inputs(16, 100, 32))
    assert third.waited == [] and 3 in kept
    now[0], captures[0] = first, False
    head.cross_entropy(*inputs(16, 5000, 32))               # a new workspace comes from this stream
    assert first.waited == [] or first.waited == [3]
    now[0] = second
    head.cross_entropy(*inputs(16, 5000, 32))
    assert second.waited == [1, 1]


def test_arguments_that_autograd_follows_are_warned_of(recorded):
    losses, _ = recorded
    head = losses.LossHead(16, 100, 32, device="cpu")
    hidden, weight, targets = inputs(16, 100, 32)
    weight.requires_grad_()
    with pytest.warns(UserWarning, match="cross_entropy is not recorded by autograd"):
        head.cross_entropy(hidden, weight, targets)
    with pytest.warns(UserWarning, match="distill is not recorded by autograd"):
        head.distill(hidden, weight, *teacher(16, 3))
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        head.cross_entropy(hidden, weight.detach(), targets)
        with torch.no_grad():
            assert not head.cross_entropy(hidden, weight, targets).loss.requires_grad
