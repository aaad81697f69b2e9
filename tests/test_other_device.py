"""Tensors and workspaces of another GPU than the current one are refused: a launch goes to the current device, where their addresses mean
nothing.  Stand-ins for tensors, no GPU: nothing may reach the library."""
import pytest
import torch

from paper_2501_17116_amd import binding as b


class On:
    """What the binding looks at of a matrix on a GPU."""
    is_cuda = True

    def __init__(self, index, rows, cols, dtype=torch.bfloat16):
        self.device, self.shape, self.dtype = torch.device("cuda", index), (rows, cols), dtype

    def dim(self):
        return 2

    def stride(self):
        return (self.shape[1], 1)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 16

    def numel(self):
        return self.shape[0] * self.shape[1]


class Room:
    def get(self, nbytes):
        return On(1, 1, nbytes)


def mx(index, lines, length, transposed=False, bits=4):
    t = b.MxTensor.__new__(b.MxTensor)
    t._codes = t._scales = t._room = None
    t._set(16, 16, bits, lines, length, transposed, torch.device("cuda", index))
    return t


M, K, N = 8, 64, 32
CALLS = {
    "mx_quantize": lambda i: b.mx_quantize(On(i, M, K), b.FP4_AXIS_ROW, out=mx(i, M, K)),
    "mx_dequantize": lambda i: b.mx_dequantize(mx(i, M, K), out=On(i, M, K)),
    "mx_gemm": lambda i: b.mx_gemm(mx(i, M, K), mx(i, N, K), out=On(i, M, N)),
    "mx_gemm, addend": lambda i: b.mx_gemm(mx(i, M, K), mx(i, N, K), out=On(i, M, N), addend=On(i, M, N, torch.float32)),
    "mx_linear_fwd": lambda i: b.mx_linear_fwd(On(i, M, K), mx(i, N, K, True), Y=On(i, M, N), ws=Room()),
    "mx_linear_bwd_dgrad": lambda i: b.mx_linear_bwd_dgrad(On(i, M, N), mx(i, K, N), dA=On(i, M, K), ws=Room()),
    "mx_linear_bwd_wgrad": lambda i: b.mx_linear_bwd_wgrad(On(i, M, N), mx(i, K, M, True, 8), dW=On(i, K, N, torch.float32), ws=Room()),
    "mx_linear_bwd": lambda i: b.mx_linear_bwd(On(i, M, N), mx(i, K, M, True, 8), mx(i, K, N), dA=On(i, M, K), dW=On(i, K, N, torch.float32), ws=Room()),
}


@pytest.fixture
def reached(monkeypatch):
    """Calls that reach the library, which does nothing; the current device is cuda:0, and every stream the default one."""
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: calls.append(name) or 0

    monkeypatch.setattr(b, "lib", Library)
    monkeypatch.setattr(b, "_mx_room", lambda *shape: 4096)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0)
    return calls


@pytest.mark.parametrize("name", CALLS)
def test_mx_calls(reached, name):
    CALLS[name](0)
    assert reached == [name.split(",")[0]]
    reached.clear()
    with pytest.raises(ValueError, match="current device"):
        CALLS[name](1)
    assert not reached


def test_the_other_calls_arguments(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    b._dev_check(On(0, 4, 8), None, On(0, 8, 8))
    with pytest.raises(ValueError, match="current device"):
        b._dev_check(On(0, 4, 8), On(1, 8, 8))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    b._dev_check(On(1, 4, 8))


def test_workspaces(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    ws = b.Workspace("cpu")
    ws.buf = On(0, 1, 4096)
    assert ws.get(4096) is ws.buf
    ws.buf = On(1, 1, 4096)
    with pytest.raises(ValueError, match="current device"):
        ws.get(4096)
