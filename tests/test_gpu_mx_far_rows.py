"""MX quantization of matrices whose rows lie so far apart that a tile's 32 rows no longer lie within 2^32 bytes: the codes of a copy
whose rows lie together.  Rows just within, too."""
import pytest
import torch

from paper_2501_17116_amd import binding as b

pytestmark = pytest.mark.gpu

# bytes from row to row: the last and the first on either side of 2^32 / 32, where row 31 alone passes 2^32, and far past it
STEPS = [(1 << 27) - 32, 1 << 27, ((1 << 32) // 31 // 32 + 1) * 32, (1 << 28) + 96]


@pytest.fixture(scope="module")
def room():
    t = torch.empty(71 * ((1 << 28) + 96) + 4096, dtype=torch.uint8, device="cuda")
    yield t
    del t
    torch.cuda.empty_cache()


@pytest.mark.parametrize("step", STEPS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(32, 128), (70, 392)])
def test_codes_are_those_of_rows_that_lie_together(room, rows, cols, dtype, step):
    held = room.view(dtype)
    g = torch.Generator(device="cuda").manual_seed(rows + step % 1000)
    x = torch.randn(rows, cols, generator=g, device="cuda").to(dtype)
    far = held.as_strided((rows, cols), (step // held.element_size(), 1), 64)
    far.copy_(x)
    for bits in (4, 8):
        want_r, want_c = b.mx_quantize_both(x, bits, bits)
        r, c = b.mx_quantize_both(far, bits, bits)
        alone_r, alone_c = b.mx_quantize(far, b.FP4_AXIS_ROW, bits), b.mx_quantize(far, b.FP4_AXIS_COL, bits)
        for got, want in ((r, want_r), (c, want_c), (alone_r, want_r), (alone_c, want_c)):
            assert torch.equal(got.codes, want.codes) and torch.equal(got.scales, want.scales)
    back = b.mx_dequantize(want_c, dtype)
    far.fill_(7)
    b.mx_dequantize(want_c, dtype, out=far)
    assert torch.equal(far, back)
    far.fill_(7)
    b.mx_dequantize(want_r, dtype, out=far)
    assert torch.equal(far, b.mx_dequantize(want_r, dtype))
