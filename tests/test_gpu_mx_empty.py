"""Layers with an empty side on the GPU: no outputs, no inputs, no tokens, with a checkpoint and without."""
import pytest
import torch

from paper_2501_17116_amd import binding as b

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("M", [1, 24, 300])
def test_no_outputs(M, bits, dtype):
    K = 520
    A = torch.randn(M, K, device="cuda", dtype=dtype)
    wq = b.mx_prepare_weights(torch.empty(K, 0, device="cuda", dtype=dtype))
    assert b.mx_linear_fwd(A, wq.fwd, act_bits=bits).shape == (M, 0)
    saved = b.mx_checkpoint(M, K)
    assert b.mx_linear_fwd(A, wq.fwd, act_bits=bits, saved=saved).shape == (M, 0)
    alone = b.mx_checkpoint_save(A)
    assert torch.equal(saved.codes, alone.codes) and torch.equal(saved.scales, alone.scales)
    dA, dW = b.mx_linear_bwd(torch.empty(M, 0, device="cuda", dtype=dtype), saved, wq.bwd)
    assert dA.shape == (M, K) and bool((dA == 0).all()) and dW.shape == (K, 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M", [1, 24, 300])
def test_no_inputs(M, dtype):
    N = 136
    A = torch.empty(M, 0, device="cuda", dtype=dtype)
    wq = b.mx_prepare_weights(torch.empty(0, N, device="cuda", dtype=dtype))
    saved = b.mx_checkpoint(M, 0)
    for kept in (None, saved):
        Y = b.mx_linear_fwd(A, wq.fwd, saved=kept)
        assert Y.shape == (M, N) and bool((Y == 0).all())
    dA, dW = b.mx_linear_bwd(torch.randn(M, N, device="cuda", dtype=dtype), saved, wq.bwd)
    assert dA.shape == (M, 0) and dW.shape == (0, N)
