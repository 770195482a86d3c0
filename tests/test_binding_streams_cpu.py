"""Outputs that the binding makes for a call on another stream come from that stream's memory, and are held for the current stream, which
will read them (recorded with stand-ins for torch's calls; no GPU needed)."""
import contextlib
import inspect

import pytest
import torch

from paper_2601_15013_amd import binding


@pytest.fixture
def events(monkeypatch):
    seen, at = [], ["current"]

    @contextlib.contextmanager
    def stream(s):
        before, at[0] = at[0], s
        yield
        at[0] = before

    class Made:
        def record_stream(self, s):
            seen.append(("held for", s))

    def empty(shape, dtype=None, device=None):
        seen.append(("made on", at[0], shape, dtype, device))
        return Made()

    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: at[0])
    monkeypatch.setattr(torch, "empty", empty)
    return seen


def test_an_output_for_another_stream(events):
    binding._new((3, 4), torch.float32, "device", "side")
    assert events == [("made on", "side", (3, 4), torch.float32, "device"), ("held for", "current")]


def test_an_output_for_the_current_stream(events):
    binding._new((3,), torch.int32, "device", None)
    assert events == [("made on", "current", (3,), torch.int32, "device")]


def test_an_output_for_the_current_stream_by_name(events):
    binding._new((3,), torch.int32, "device", "current")
    assert events == [("made on", "current", (3,), torch.int32, "device")]


def test_several_outputs_are_made_at_once(events):
    binding._new_all([((1,), torch.int32), ((2,), torch.float32)], "device", "side")
    assert [e[:2] for e in events] == [("made on", "side")] * 2 + [("held for", "current")] * 2


def test_every_call_with_a_stream_makes_its_outputs_so():
    takes = [f for _, f in inspect.getmembers(binding, inspect.isfunction) if "stream" in inspect.signature(f).parameters]
    assert len(takes) > 15
    assert [f.__name__ for f in takes if "torch.empty" in inspect.getsource(f)] == ["_new", "_new_all"]
