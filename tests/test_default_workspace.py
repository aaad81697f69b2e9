"""The workspaces that calls take for themselves: one a device, stream and thread.  A call is several launches which pass quantized operands
through its workspace, and the interpreter's lock is released inside it, so two threads on one stream would mix them.  No GPU needed."""
import threading

import pytest
import torch

from paper_2501_17116_amd import binding as b


class Like:
    def __init__(self, index):
        self.device = torch.device("cuda", index)


@pytest.fixture
def host(monkeypatch):
    """Buffers in host memory; a stream's handle is what the test says."""
    where = {"device": 0, "stream": 7}
    real = b.Workspace

    class HostWorkspace(real):
        def __init__(self, device="cuda"):
            super().__init__("cpu")

    class Stream:
        @property
        def cuda_stream(self):
            return where["stream"]

    monkeypatch.setattr(b, "Workspace", HostWorkspace)
    monkeypatch.setattr(b, "_default_ws", {})
    monkeypatch.setattr(b, "_stream_of", lambda t: where["stream"])
    monkeypatch.setattr(torch.cuda, "current_device", lambda: where["device"])
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Stream())
    return where


def mx_pointer():
    return b._mx_ws(b.FP4_OP_MX_FWD, 24, 4096, 512, None, Like(0))[0]


def plain_pointer():
    return b._ws(1 << 16, None).data_ptr()


@pytest.mark.parametrize("pointer", [mx_pointer, plain_pointer])
def test_threads_on_one_stream_do_not_share(host, pointer):
    mine, others, meet = pointer(), [], threading.Barrier(3)

    def work():
        others.append(pointer())
        meet.wait()          # neither ends before the other has its own

    threads = [threading.Thread(target=work) for _ in range(2)]
    for t in threads:
        t.start()
    meet.wait()
    for t in threads:
        t.join()
    assert len({mine, *others}) == 3
    assert pointer() == mine      # and a thread keeps its own


@pytest.mark.parametrize("pointer", [mx_pointer, plain_pointer])
def test_streams_do_not_share(host, pointer):
    first = pointer()
    host["stream"] = 8
    assert pointer() != first
    host["stream"] = 7
    assert pointer() == first


def test_both_kinds_of_call_share_a_threads_workspace(host):
    big = b._ws(1 << 24, None).data_ptr()
    assert mx_pointer() == big
    assert len(b._default_ws) == 1


def test_a_callers_workspace_is_taken(host):
    ws = b.Workspace()
    at = b._mx_ws(b.FP4_OP_MX_FWD, 24, 4096, 512, ws, Like(0))[0]
    assert at == ws.buf.data_ptr() and b._ws(16, ws).data_ptr() == at and not b._default_ws
