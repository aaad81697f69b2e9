"""Workspaces that grow: what they keep alive is bounded by the largest size they were asked for, and can be given back.  No GPU needed."""
import threading

import pytest
import torch

from paper_2501_17116_amd import binding as b


def held(ws):
    return ws.buf.numel() + sum(t.numel() for t in ws._outgrown)


@pytest.mark.parametrize("first,step", [(1000, 1), (1 << 20, 4096), (1, 7), (17, 1000)])
def test_growth_keeps_a_bounded_number_of_bytes(first, step):
    """Each buffer is at least half as large again as the one before: no more than 3 times the last, which is at most 1.5 times what was asked for."""
    ws = b.Workspace("cpu")
    need, grown = first, 0
    for _ in range(3000):
        before = ws.buf
        assert ws.get(need).numel() >= need
        grown += ws.buf is not before
        assert held(ws) <= 4.5 * need + 64
        need += step
    assert grown <= 40
    at = ws.buf.data_ptr()
    ws.release()
    assert held(ws) == ws.buf.numel() and ws.get(1).data_ptr() == at


def test_the_first_size_is_taken_as_it_is():
    ws = b.Workspace("cpu")
    assert ws.get(12345).numel() == 12345 and not ws._outgrown
    assert ws.get(50000).numel() == 50000       # more than half as much again: as it is, too
    assert ws.get(50001).numel() == 75000


def test_memory_that_lacks_only_the_slack_is_enough(monkeypatch):
    ws, real = b.Workspace("cpu"), torch.empty

    def empty(n, **kw):
        if n > 1200:
            raise torch.OutOfMemoryError
        return real(n, **kw)

    monkeypatch.setattr(torch, "empty", empty)
    assert ws.get(1000).numel() == 1000
    assert ws.get(1100).numel() == 1100
    with pytest.raises(torch.OutOfMemoryError):
        ws.get(1300)
    assert ws.buf.numel() == 1100 and len(ws._outgrown) == 1


@pytest.fixture
def host(monkeypatch):
    real, waited = b.Workspace, []
    monkeypatch.setattr(b, "Workspace", lambda device: real("cpu"))
    monkeypatch.setattr(b, "_default_ws", {})
    monkeypatch.setattr(torch.cuda, "synchronize", waited.append)
    return waited


def test_the_calls_own_workspaces_can_be_released(host):
    for device, stream in ((0, 1), (0, 2), (1, 1)):
        for need in (100, 200, 400):
            b._default_workspace(device, stream)._sized(need)
    other = threading.Thread(target=lambda: [b._default_workspace(0, 1)._sized(n) for n in (10, 20)])
    other.start()
    other.join()
    current = {k: ws.buf.data_ptr() for k, ws in b._default_ws.items()}
    assert sum(len(ws._outgrown) for ws in b._default_ws.values()) == 7
    b.release_outgrown()
    assert sorted(host) == [0, 1]               # each device once, before anything is dropped
    assert all(not ws._outgrown for ws in b._default_ws.values())
    assert {k: ws.buf.data_ptr() for k, ws in b._default_ws.items()} == current
    host.clear()
    b.release_outgrown()
    assert not host                             # nothing to wait for


def test_what_is_outgrown_while_release_waits_is_kept(host, monkeypatch):
    """Its kernels were enqueued after the wait began."""
    ws = b._default_workspace(0, 1)
    ws._sized(100)
    ws._sized(200)
    young = ws.buf
    monkeypatch.setattr(torch.cuda, "synchronize", lambda device: ws._sized(400))
    b.release_outgrown()
    assert len(ws._outgrown) == 1 and ws._outgrown[0] is young
