"""MX tensors whose codes pass 2^32 bytes: the far end as if it were a tensor of its own."""
import pytest
import torch

from paper_2501_17116_amd import binding as b

pytestmark = pytest.mark.gpu


def tail(t, first):
    """Lines from `first` on as an MX tensor."""
    codes = t.codes[first:] if t.bits == 4 else t.codes[:, first:]
    return b.MxTensor(codes.contiguous(), t.scales[first:].contiguous(), t.length, t.transposed)


def test_product_of_many_lines():
    """Scales of 1: sums are multiples of 1/4 below 2^22, exact in fp32, whichever kernel forms them."""
    lines, length = (1 << 21) - 3, 4200
    g = torch.Generator(device="cuda").manual_seed(1)
    big = b.mx_empty(lines, length)
    assert big.codes.numel() > 1 << 32
    big.codes.random_(0, 256, generator=g)
    big.codes[:, length // 2:] = 0
    big.scales.fill_(127)
    few = b.mx_empty(40, length)
    few.codes.random_(0, 256, generator=g)
    few.codes[:, length // 2:] = 0
    few.scales.fill_(127)
    for first in (0, lines - 700):
        part = b.MxTensor(big.codes[first:first + 700].contiguous(), big.scales[first:first + 700].contiguous(), length)
        want = b.mx_dequantize(part, torch.float32).double() @ b.mx_dequantize(few, torch.float32).double().t()
        assert torch.equal(b.mx_gemm(big, few)[first:first + 700].double(), want)
        assert torch.equal(b.mx_gemm(few, big)[:, first:first + 700].double(), want.t())


@pytest.mark.parametrize("bits", [4, 8])
def test_quantization_of_many_rows(bits):
    rows, cols = (1 << 21) - 32, 1104
    x = torch.randn(1 << 16, cols, device="cuda", dtype=torch.bfloat16).repeat(32, 1)[:rows]
    x[-500:].mul_(3.0)
    assert x.numel() * 2 > 1 << 32
    r, c = b.mx_quantize_both(x, bits, bits)
    first = rows - 512 - 32 * 3
    sub_r, sub_c = b.mx_quantize_both(x[first:], bits, bits)
    end = tail(r, first)
    assert torch.equal(end.codes, sub_r.codes) and torch.equal(end.scales, sub_r.scales)
    n = rows - first
    for p in range(bits // 4):
        big, small = (c.codes, sub_c.codes) if bits == 4 else (c.codes[p], sub_c.codes[p])
        assert torch.equal(big[:, first // 2:first // 2 + n // 2], small[:, :n // 2])
    assert torch.equal(c.scales[:, first // 32:first // 32 + n // 32], sub_c.scales[:, :n // 32])
    back = b.mx_dequantize(r)
    assert torch.equal(back[first:], b.mx_dequantize(sub_r))
    back = b.mx_dequantize(c)
    assert torch.equal(back[first:], b.mx_dequantize(sub_c))
