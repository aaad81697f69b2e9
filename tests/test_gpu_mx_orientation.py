"""Square layers, where sizes cannot tell a tensor's orientation from the other: the wrong one is refused, the right one computes."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as mx
from paper_2501_17116_amd import binding as b
from tests.test_gpu_mx_gemm import bound, close

pytestmark = pytest.mark.gpu
S = 96


@pytest.fixture(scope="module")
def layer():
    g = torch.Generator().manual_seed(8)
    A, W, dY = [torch.randn(S, S, generator=g) for _ in range(3)]
    return A, W, dY, b.mx_prepare_weights(W.cuda())


def test_weights_of_the_other_pass(layer):
    A, W, dY, wq = layer
    with pytest.raises(ValueError, match="MxWeights.fwd"):
        b.mx_linear_fwd(A.cuda(), wq.bwd)
    with pytest.raises(ValueError, match="MxWeights.bwd"):
        b.mx_linear_bwd_dgrad(dY.cuda(), wq.fwd)
    saved = b.mx_checkpoint_save(A.cuda())
    with pytest.raises(ValueError, match="MxWeights.bwd"):
        b.mx_linear_bwd(dY.cuda(), saved, wq.fwd)
    aq, w = mx.through(A.double().numpy(), 4), W.double().numpy()
    w_fwd = mx.through(np.ascontiguousarray(w.T), 4)
    close(b.mx_linear_fwd(A.cuda(), wq.fwd), aq @ w_fwd.T, bound(aq, w_fwd, S))
    # weights held as [outputs, inputs], quantized along their rows, are a forward pass's as they lie
    by_rows = b.mx_quantize(W.t().contiguous().cuda(), b.FP4_AXIS_ROW)
    assert torch.equal(b.mx_linear_fwd(A.cuda(), by_rows), b.mx_linear_fwd(A.cuda(), wq.fwd))


def test_outputs_marked_otherwise(layer):
    x = layer[0].cuda()
    with pytest.raises(ValueError, match="transposed"):
        b.mx_quantize(x, b.FP4_AXIS_COL, out=b.mx_empty(S, S))
    with pytest.raises(ValueError, match="transposed"):
        b.mx_quantize(x, b.FP4_AXIS_ROW, out=b.mx_empty(S, S, transposed=True))
    for axis in (b.FP4_AXIS_ROW, b.FP4_AXIS_COL):
        t = b.mx_empty(S, S, 8, transposed=axis == b.FP4_AXIS_COL)
        assert b.mx_quantize(x, axis, out=t) is t
        assert float((b.mx_dequantize(t, torch.float32) - x).abs().max()) < 0.25     # an element errs by a fourth of its block's scale at most


def test_checkpoints_along_rows(layer):
    A, W, dY, wq = layer
    rows = b.mx_quantize(A.cuda(), b.FP4_AXIS_ROW, 8)
    with pytest.raises(ValueError, match="transposed"):
        b.mx_linear_fwd(A.cuda(), wq.fwd, saved=b.mx_empty(S, S, 8))
    with pytest.raises(ValueError, match="transposed"):
        b.mx_linear_bwd_wgrad(dY.cuda(), rows)
    with pytest.raises(ValueError, match="transposed"):
        b.mx_linear_bwd(dY.cuda(), rows, wq.bwd)
