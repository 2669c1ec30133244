"""The binding's kept workspaces, on host memory."""

import pytest

import paper_2608_15531_amd as fq

torch = pytest.importorskip("torch")


@pytest.fixture
def kept(monkeypatch):
    monkeypatch.setattr(fq, "_workspaces", {})
    monkeypatch.setattr(fq, "_captured", {})


def test_calls_in_a_capture_never_share_a_workspace_with_others(kept):
    eager = fq.workspace(1 << 20, "cpu", 7)
    a = fq.workspace(1 << 20, "cpu", 7, capture=1)
    a[:] = 5   # what replays of the first graph leave there
    assert fq.workspace(1 << 19, "cpu", 7, capture=1) is a            # of the same graph
    b = fq.workspace(1 << 19, "cpu", 7, capture=2)                    # another graph, same stream
    assert fq.workspace(1 << 20, "cpu", 7) is eager
    assert len({t.data_ptr() for t in (eager, a, b)}) == 3
    assert (eager == 0).all() and (b[:256 * 1024] == 0).all()
    larger = fq.workspace(1 << 21, "cpu", 7, capture=2)
    assert larger is not b and larger.numel() == 1 << 21 and (larger[:256 * 1024] == 0).all()
    assert fq.workspace(1 << 21, "cpu", 8, capture=2) is not larger   # another stream of the capture
    # an eager call that needs more replaces the kept one alone
    assert fq.workspace(1 << 22, "cpu", 7) is not eager
    assert fq.workspace(1 << 21, "cpu", 7, capture=2) is larger
