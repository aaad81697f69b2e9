"""The MX layer on the GPU: forward pass with its checkpoint, both gradients, against the oracle in fp64 and against differences."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as mx
from paper_2501_17116_amd import binding as b
from tests.test_gpu_mx_gemm import bound, close

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(M, K, N, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    A = torch.randn(M, K, generator=g)
    A[:, torch.randperm(K, generator=g)[: max(1, K // 200)]] *= 30.0
    return [t.to(DT[dtype]) for t in (A, torch.randn(K, N, generator=g) * 0.02, torch.randn(M, N, generator=g) * 0.01)]


def host(t):
    return t.double().cpu().numpy()


SHAPES = [(1, 64, 48), (1, 1000, 264), (2, 4096, 40), (7, 520, 1048), (16, 513 * 8, 256), (17, 256, 72), (33, 200, 520), (64, 1096, 128), (100, 72, 1096),
          (257, 512, 264), (1055, 392, 136)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_passes(M, K, N, dtype):
    A, W, dY = make(M, K, N, dtype, M + K + N)
    a, w, g = host(A), host(W), host(dY)
    bf16 = dtype == "bf16"
    wq = b.mx_prepare_weights(W.cuda())
    w_fwd, w_bwd = mx.through(w.T, 4), mx.through(w, 4)
    for act in (4, 8):
        aq = mx.through(a, act)
        close(b.mx_linear_fwd(A.cuda(), wq.fwd, act_bits=act), aq @ w_fwd.T, bound(aq, w_fwd, K), bf16)
        for bits in (8, 4):
            saved = b.mx_checkpoint(M, K, bits)
            close(b.mx_linear_fwd(A.cuda(), wq.fwd, act_bits=act, saved=saved), aq @ w_fwd.T, bound(aq, w_fwd, K), bf16)
            alone = b.mx_checkpoint_save(A.cuda(), bits)
            assert torch.equal(saved.codes, alone.codes) and torch.equal(saved.scales, alone.scales)
            assert np.array_equal(host(b.mx_dequantize(saved, torch.float32)), mx.through(a.T, bits).T)
    w8 = b.mx_quantize(W.cuda(), b.FP4_AXIS_COL, 8)      # weights in 8 bits
    w8_fwd = mx.through(w.T, 8)
    for act in (4, 8):
        aq = mx.through(a, act)
        close(b.mx_linear_fwd(A.cuda(), w8, act_bits=act), aq @ w8_fwd.T, bound(aq, w8_fwd, K), bf16)
    saved = b.mx_checkpoint_save(A.cuda())
    kept = mx.through(a.T, 8)
    gq = mx.through(g, 4)
    dA = b.mx_linear_bwd_dgrad(dY.cuda(), wq.bwd)
    close(dA, gq @ w_bwd.T, bound(gq, w_bwd, N), bf16)
    for bits in (4, 8):
        gt = mx.through(g.T, bits)
        dW = b.mx_linear_bwd_wgrad(dY.cuda(), saved, grad_bits=bits)
        close(dW, kept @ gt.T, bound(kept, gt, M))
        dA2, dW2 = b.mx_linear_bwd(dY.cuda(), saved, wq.bwd, grad_bits=bits)
        assert torch.equal(dA2, dA) and torch.equal(dW2, dW)
        acc = dW.clone()
        b.mx_linear_bwd(dY.cuda(), saved, wq.bwd, grad_bits=bits, dW=acc, accumulate=True)
        close(acc, 2 * (kept @ gt.T), 2 * bound(kept, gt, M) + 2.0 ** -22 * np.abs(kept @ gt.T))


def test_gradients_are_those_of_the_products_by_differences():
    """The products are linear in the weights and in the activations, so a difference along a direction is the derivative there."""
    M, K, N = 70, 96, 40
    A, W, dY = make(M, K, N, "f32", 5)
    wq = b.mx_prepare_weights(W.cuda())
    saved = b.mx_checkpoint(M, K)
    b.mx_linear_fwd(A.cuda(), wq.fwd, saved=saved)
    dA, dW = b.mx_linear_bwd(dY.cuda(), saved, wq.bwd)
    kept = host(b.mx_dequantize(saved, torch.float32))                       # what the backward pass knows of A
    w_bwd = host(b.mx_dequantize(wq.bwd, torch.float32))
    gt = host(b.mx_dequantize(b.mx_quantize(dY.cuda(), b.FP4_AXIS_COL), torch.float32))
    gr = host(b.mx_dequantize(b.mx_quantize(dY.cuda(), b.FP4_AXIS_ROW), torch.float32))
    rng = np.random.default_rng(6)
    for _ in range(4):
        E, F = rng.normal(size=(K, N)), rng.normal(size=(M, K))
        h = 0.5
        along_w = (np.sum(gt * (kept @ (host(W) + h * E))) - np.sum(gt * (kept @ (host(W) - h * E)))) / (2 * h)
        along_a = (np.sum(gr * ((kept + h * F) @ w_bwd)) - np.sum(gr * ((kept - h * F) @ w_bwd))) / (2 * h)
        tol_w = np.sum(bound(kept.T, gt.T, M) * np.abs(E)) + 1e-9
        tol_a = np.sum(bound(gr, w_bwd, N) * np.abs(F)) + 1e-9
        assert abs(np.sum(host(dW) * E) - along_w) <= tol_w
        assert abs(np.sum(host(dA) * F) - along_a) <= tol_a


def test_rows_apart_other_streams_and_graphs():
    M, K, N = 24, 520, 136
    A, W, dY = make(M, K, N, "bf16", 9)
    wide = torch.full((M, K + 16), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 8:8 + K] = A.cuda()
    wq = b.mx_prepare_weights(W.cuda())
    ref_saved = b.mx_checkpoint(M, K)
    ref = b.mx_linear_fwd(A.cuda(), wq.fwd, saved=ref_saved)
    ref_dA, ref_dW = b.mx_linear_bwd(dY.cuda(), ref_saved, wq.bwd)
    saved = b.mx_checkpoint(M, K)
    assert torch.equal(b.mx_linear_fwd(wide[:, 8:8 + K], wq.fwd, saved=saved), ref)
    assert torch.equal(saved.codes, ref_saved.codes)
    dYd = dY.cuda()
    Y, dA, dW = torch.empty_like(ref), torch.empty_like(ref_dA), torch.empty_like(ref_dW)
    ws = b.Workspace()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def step():
        b.mx_linear_fwd(wide[:, 8:8 + K], wq.fwd, saved=saved, Y=Y, ws=ws)
        b.mx_linear_bwd(dYd, saved, wq.bwd, dA=dA, dW=dW, ws=ws)

    with torch.cuda.stream(s):
        step()
    s.synchronize()
    assert torch.equal(Y, ref) and torch.equal(dA, ref_dA) and torch.equal(dW, ref_dW)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    for k in range(3):
        for t in (Y, dA, dW):
            t.fill_(-1.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, ref) and torch.equal(dA, ref_dA) and torch.equal(dW, ref_dW), k
        torch.ones(1000, device="cuda").sum().item()


def test_no_tokens_and_empty_sides():
    W = torch.randn(64, 32, device="cuda")
    wq = b.mx_prepare_weights(W)
    A = torch.empty(0, 64, device="cuda")
    saved = b.mx_checkpoint(0, 64)
    assert b.mx_linear_fwd(A, wq.fwd, saved=saved).shape == (0, 32)
    dA, dW = b.mx_linear_bwd(torch.empty(0, 32, device="cuda"), saved, wq.bwd)
    assert dA.shape == (0, 64) and bool((dW == 0).all())
    keep = torch.randn(64, 32, device="cuda")
    was = keep.clone()
    b.mx_linear_bwd_wgrad(torch.empty(0, 32, device="cuda"), saved, dW=keep, accumulate=True)
    assert torch.equal(keep, was)


def test_refusals():
    A, W, dY = [t.cuda() for t in make(8, 64, 32, "bf16", 1)]
    wq = b.mx_prepare_weights(W)
    with pytest.raises(ValueError):
        b.mx_linear_fwd(A, wq.bwd)
    with pytest.raises(ValueError):
        b.mx_linear_fwd(A, wq.fwd, saved=b.mx_checkpoint(9, 64))
    with pytest.raises(ValueError):
        b.mx_linear_fwd(A, wq.fwd, Y=torch.empty(8, 32, device="cuda"))
    with pytest.raises(ValueError):
        b.mx_linear_bwd(dY, b.mx_checkpoint(8, 63), wq.bwd)
    with pytest.raises(ValueError):
        b.mx_linear_bwd_wgrad(dY, b.mx_checkpoint(8, 64), accumulate=True)
    with pytest.raises(b.Fp4Error):
        b.mx_linear_fwd(A, wq.fwd, act_bits=7)
