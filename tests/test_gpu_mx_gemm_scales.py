"""Scales and passes in the larger tiles, bit for bit: blocks under different scales, operands in 8 bits (two and four passes), several tiles a
workgroup, NaN blocks in every tile."""
import pytest
import torch

from paper_2501_17116_amd import binding as b
from tests.mx_exact import operand, product, same

pytestmark = pytest.mark.gpu
BITS = [(4, 4), (8, 4), (4, 8), (8, 8)]


@pytest.mark.parametrize("bl,br", BITS)
@pytest.mark.parametrize("tile", [64, 128, 192, 256])
@pytest.mark.parametrize("P,Q,Kc", [(4352, 4352, 40), (4100, 4360, 512), (4353, 4225, 1100)])
def test_scales_of_several_tiles_a_workgroup(P, Q, Kc, tile, bl, br):
    l, r = operand(P, Kc, bl, P + Kc), operand(Q, Kc, br, Q + Kc)
    want = product(l, r)
    got = b.mx_gemm_by_tile(l, r, tile)
    assert same(got, want)
    assert same(b.mx_gemm_by_tile(l, r, tile, torch.bfloat16), want)
    ld = (Q + 7) // 8 * 8
    add = torch.randint(-64, 64, (P, ld), device="cuda").float()[:, :Q]
    assert same(b.mx_gemm_by_tile(l, r, tile, addend=add), want + add.double())


@pytest.mark.parametrize("bl,br", BITS)
@pytest.mark.parametrize("tile", [16, 32, 64, 128, 192, 256])
@pytest.mark.parametrize("P,Q,Kc", [(300, 264, 200), (520, 1000, 1100)])
def test_nan_blocks(P, Q, Kc, tile, bl, br):
    l, r = operand(P, Kc, bl, 1), operand(Q, Kc, br, 2)
    blocks = (Kc + 31) // 32
    for line, block in ((5, 3), (130, 0), (P - 1, blocks - 1), (P - 44, blocks // 2)):
        l.scales[line, block] = 255
    for line, block in ((0, 1), (Q - 2, 0), (Q // 2, blocks - 1)):
        r.scales[line, block] = 255
    want = product(l, r)
    assert int(torch.isnan(want).all(dim=1).sum()) == 4 and int(torch.isnan(want).all(dim=0).sum()) == 3
    assert same(b.mx_gemm_by_tile(l, r, tile), want)
    assert same(b.mx_gemm_by_tile(l, r, tile, torch.bfloat16), want)
