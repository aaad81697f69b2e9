"""The product of few tokens where a workgroup takes 16, 32 or 64 columns, from codes and from tokens that it quantizes itself: what serving
runs.  On 256 compute units a workgroup takes 16 columns up to 4096 of them, 32 up to 8192, 64 beyond (with at most 32 tokens)."""
import pytest
import torch

from oracle import mx_oracle as mx
from paper_2501_17116_amd import binding as b
from tests.mx_exact import operand, product, same, values
from tests.test_gpu_mx_gemm import bound, close

pytestmark = pytest.mark.gpu
BITS = [(4, 4), (8, 4), (4, 8), (8, 8)]
COLUMNS = [4093, 5003, 8195, 9005, 11008]


@pytest.mark.parametrize("bl,br", BITS)
@pytest.mark.parametrize("Kc", [72, 520])
@pytest.mark.parametrize("Q", COLUMNS)
@pytest.mark.parametrize("P", [1, 16, 17, 32, 40, 64, 100])
def test_from_codes(P, Q, Kc, bl, br):
    l, r = operand(P, Kc, bl, P + Kc, 2), operand(Q, Kc, br, Q + Kc, 2)
    want = product(l, r)
    assert same(b.mx_gemm_by_tile(l, r, 16), want)
    assert same(b.mx_gemm_by_tile(l, r, 16, torch.bfloat16), want)
    held = torch.randint(-64, 64, (P, (Q + 7) // 8 * 8), device="cuda").float()
    add = held[:, :Q]
    total = want + add.double()
    assert same(b.mx_gemm_by_tile(l, r, 16, addend=add), total)
    if P <= 32:
        assert b.mx_gemm_tile(P, Q, Kc, bl, br)[0] == 16
        assert same(b.mx_gemm(l, r, addend=add, out=add), total)     # in place: every column once


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N", [5003, 9005])
@pytest.mark.parametrize("M,K", [(1, 72), (1, 4096), (16, 520), (17, 520), (32, 72), (32, 1000), (24, 4096)])
def test_from_tokens(M, K, N, dtype):
    g = torch.Generator().manual_seed(M + K + N)
    A, W = torch.randn(M, K, generator=g).to(dtype), (torch.randn(K, N, generator=g) * 0.02).to(dtype)
    room = torch.zeros(K, (N + 7) // 8 * 8, dtype=dtype, device="cuda")
    room[:, :N] = W.cuda()
    a = A.double().numpy()
    held = torch.zeros(M, (K + 7) // 8 * 8, dtype=dtype, device="cuda")
    held[:, :K] = A.cuda()
    for wbits in (4, 8):
        wq = b.mx_quantize(room[:, :N], b.FP4_AXIS_COL, wbits)
        w_fwd = values(wq).cpu().numpy()
        for act in (4, 8):
            aq = mx.through(a, act)
            Y = b.mx_linear_fwd(held[:, :K], wq, act_bits=act)
            close(Y, aq @ w_fwd.T, bound(aq, w_fwd, K), dtype == torch.bfloat16)
            apart = b.mx_gemm(b.mx_quantize(held[:, :K], b.FP4_AXIS_ROW, act), wq, dtype)   # the same kernel from codes: the same sums
            assert torch.equal(Y, apart)
