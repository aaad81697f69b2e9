"""The MX binding tells orientations apart where sizes cannot, before anything reaches the library (stand-ins for tensors, no GPU)."""
import pytest
import torch

from paper_2501_17116_amd import binding as b
from tests.test_other_device import On, Room, mx, reached  # noqa: F401

S = 64


def tensor(transposed, bits=4):
    return mx(0, S, S, transposed, bits)


@pytest.fixture
def weights(monkeypatch, reached):  # noqa: F811
    monkeypatch.setattr(b, "mx_empty", lambda lines, length, bits=4, transposed=False, device=None: mx(0, lines, length, transposed, bits))
    wq = b.mx_prepare_weights(On(0, S, S))
    reached.clear()
    return wq


@pytest.fixture(autouse=True)
def room(monkeypatch):
    monkeypatch.setattr(Room, "get", lambda self, n: On(0, 1, n))


def fwd(W, saved=None):
    return b.mx_linear_fwd(On(0, S, S), W, saved=saved, Y=On(0, S, S), ws=Room())


def dgrad(W):
    return b.mx_linear_bwd_dgrad(On(0, S, S), W, dA=On(0, S, S), ws=Room())


def wgrad(saved):
    return b.mx_linear_bwd_wgrad(On(0, S, S), saved, dW=On(0, S, S, torch.float32), ws=Room())


def both(saved, W):
    return b.mx_linear_bwd(On(0, S, S), saved, W, dA=On(0, S, S), dW=On(0, S, S, torch.float32), ws=Room())


def test_weights(reached, weights):  # noqa: F811
    saved = tensor(True, 8)
    for call, says in ((lambda: fwd(weights.bwd), "MxWeights.fwd"), (lambda: dgrad(weights.fwd), "MxWeights.bwd"), (lambda: both(saved, weights.fwd), "MxWeights.bwd")):
        with pytest.raises(ValueError, match=says):
            call()
    assert not reached
    fwd(weights.fwd), dgrad(weights.bwd), both(saved, weights.bwd)
    for t in (tensor(False), tensor(True)):      # a caller's own, from masters held either way
        fwd(t), dgrad(t), both(saved, t)
    assert reached == ["mx_linear_fwd", "mx_linear_bwd_dgrad", "mx_linear_bwd"] * 3


@pytest.mark.parametrize("axis", [b.FP4_AXIS_ROW, b.FP4_AXIS_COL])
def test_outputs(reached, axis):  # noqa: F811
    with pytest.raises(ValueError, match="transposed"):
        b.mx_quantize(On(0, S, S), axis, out=tensor(axis == b.FP4_AXIS_ROW))
    assert not reached
    b.mx_quantize(On(0, S, S), axis, out=tensor(axis == b.FP4_AXIS_COL))
    assert reached == ["mx_quantize"]


def test_checkpoints(reached, weights):  # noqa: F811
    for call in (lambda: fwd(weights.fwd, tensor(False, 8)), lambda: wgrad(tensor(False, 8)), lambda: both(tensor(False, 8), weights.bwd)):
        with pytest.raises(ValueError, match="transposed"):
            call()
    assert not reached
    fwd(weights.fwd, tensor(True, 8)), wgrad(tensor(True, 8)), both(tensor(True, 4), weights.bwd)
    assert reached == ["mx_linear_fwd", "mx_linear_bwd_wgrad", "mx_linear_bwd"]
