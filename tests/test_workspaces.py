"""Which buffers HotPath gives its calls as workspaces.  Host logic alone: no context, and the buffers are on the host."""
import types
import weakref

import pytest
import torch

from paper_2103_00686_amd.hotpath import HotPath


@pytest.fixture
def hp():
    h = HotPath.__new__(HotPath)
    h.dev = torch.device("cpu")
    h.ctx = types.SimpleNamespace(stream=5)
    h._ws, h._norm_ws = {}, []
    return h


@pytest.mark.parametrize("name", ["bwd", "bwd_ahead0"])
def test_an_outgrown_workspace_stays(hp, name):
    """A graph may hold its address: it must not go back to the allocator."""
    first = hp._workspace(name, 1000)
    seen = weakref.ref(first)
    del first
    assert hp._workspace(name, 500) is seen()
    second = hp._workspace(name, 1 << 20)
    assert second.numel() >= 1 << 20
    assert seen() is not None and seen().data_ptr() != second.data_ptr()
    assert hp._workspace(name, 1000) is second


def test_growing_step_by_step_holds_a_bounded_sum(hp):
    for n in range(1000, 200_000, 100):
        ws = hp._workspace("bwd", n)
        assert ws.numel() >= n
    held = [w.numel() for w in hp._ws["bwd"]]
    assert sum(held) <= 3 * held[-1] and held[-1] <= 1.5 * 200_000  # a geometric sum of ratio 2/3


def test_workspaces_are_told_apart_by_name(hp):
    assert hp._workspace("bwd", 1000).data_ptr() != hp._workspace("part", 1000).data_ptr()


def test_eager_norms_share_one(hp, monkeypatch):
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    a = hp._norm_workspace(100)
    assert hp._norm_workspace(5000) is a
    b = hp._norm_workspace(1 << 20)
    assert b.numel() >= 1 << 20 and hp._norm_workspace(100) is b


def test_captured_norms_share_none(hp, monkeypatch):
    """Two graphs, or one and an eager call, that run at the same time."""
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    eager = hp._norm_workspace(100)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev=None: types.SimpleNamespace(cuda_stream=5))
    a, b = hp._norm_workspace(100), hp._norm_workspace(100)
    assert min(a.numel(), b.numel()) >= 100
    assert len({t.data_ptr() for t in (eager, a, b)}) == 3


def test_a_captured_norm_on_another_stream_says_so(hp, monkeypatch):
    """The buffer is dropped when the call returns: the allocator has to know which stream reads it."""
    said = []
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev=None: types.SimpleNamespace(cuda_stream=6))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda s, device=None: s)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: said.append(s))
    hp._norm_workspace(100)
    assert said == [5]
