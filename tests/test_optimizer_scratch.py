"""The binding's own scratch, without a device: what it keeps, gives back, and holds on to when there is no memory for a larger one."""
import contextlib

import pytest
import torch

from paper_2104_11125_amd import binding


class _Ctx(binding.ScaleCom):
    def __init__(self):
        self._ctx, self.device, self.stream = None, torch.device("cpu"), "a stream"
        self._ortho_scratch, self._ortho_captured = [], False

    def close(self):
        pass

    __del__ = close


@pytest.fixture
def capturing(monkeypatch):
    state = {"now": False, "current": "a stream", "entered": 0}

    @contextlib.contextmanager
    def stream(s):
        assert s == "a stream"
        state["entered"] += 1
        before, state["current"] = state["current"], s
        yield
        state["current"] = before

    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: state["current"])
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: state["now"] and state["current"] == "a stream")
    return state


@pytest.mark.parametrize("current", ["a stream", "another"])
def test_what_is_kept(capturing, current):
    capturing["current"] = current
    ctx = _Ctx()
    first = ctx._kept_scratch(100)
    assert first.numel() == 100 and ctx._kept_scratch(60) is first
    second = ctx._kept_scratch(200)
    assert ctx._ortho_scratch == [second]                   # (one that no graph holds is given back)
    capturing["now"] = True
    assert ctx._kept_scratch(150) is second
    capturing["now"] = False
    third = ctx._kept_scratch(300)
    fourth = ctx._kept_scratch(400)
    assert len(ctx._ortho_scratch) == 2 and ctx._ortho_scratch[0] is second and ctx._ortho_scratch[1] is fourth and third is not fourth
    capturing["now"] = True
    fifth = ctx._kept_scratch(500)                          # allocated inside a capture
    capturing["now"] = False
    ctx._kept_scratch(600)
    assert [t.numel() for t in ctx._ortho_scratch] == [200, 500, 600] and ctx._ortho_scratch[1] is fifth


def test_no_memory_for_a_larger_one(capturing, monkeypatch):
    ctx = _Ctx()
    capturing["now"] = True
    held = ctx._kept_scratch(100)
    capturing["now"] = False
    empty = torch.empty

    def none(*a, **k):
        raise RuntimeError("out of memory")

    monkeypatch.setattr(torch, "empty", none)
    with pytest.raises(RuntimeError):
        ctx._kept_scratch(1000)
    monkeypatch.setattr(torch, "empty", empty)
    ctx._kept_scratch(200)
    ctx._kept_scratch(300)
    assert [t.numel() for t in ctx._ortho_scratch] == [100, 300] and ctx._ortho_scratch[0] is held
