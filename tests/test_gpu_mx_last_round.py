"""Products whose last round of 256 x 256 tiles is cut into quarters, in a launch of its own: every output once, quarters behind the edge none."""
import pytest
import torch

from paper_2501_17116_amd import binding as b
from tests.mx_exact import operand, product, same

pytestmark = pytest.mark.gpu

# the last rows and columns of tiles hold at most 128: half of each of their quarters lies behind the edge
CASES = [(5658, 8525, 40, 4, 4), (6219, 7713, 40, 8, 4), (6661, 7250, 40, 4, 8), (4196, 4101, 40, 8, 8), (4196, 4101, 520, 8, 8), (4196, 4100, 1100, 8, 8),
         (5230, 3333, 72, 8, 8)]


@pytest.mark.parametrize("P,Q,Kc,bl,br", CASES)
def test_cut_last_rounds(P, Q, Kc, bl, br):
    n_cu = torch.cuda.get_device_properties(0).multi_processor_count
    tile, rest = b.mx_gemm_tile(P, Q, Kc, bl, br, n_cu)
    if n_cu == 256:
        assert tile == 256 and rest > 0
    l, r = operand(P, Kc, bl, P), operand(Q, Kc, br, Q)
    want = product(l, r)
    assert same(b.mx_gemm(l, r), want)
    assert same(b.mx_gemm(l, r, torch.bfloat16), want)
    ld = (Q + 7) // 8 * 8
    held = torch.full((P, ld + 8), 7.0, device="cuda")
    held[:, :Q] = torch.randint(-64, 64, (P, Q), device="cuda").float()
    total = want + held[:, :Q].double()
    b.mx_gemm(l, r, addend=held[:, :Q], out=held[:, :Q])     # in place: a tile covered twice would add twice
    assert same(held[:, :Q], total)
    assert bool((held[:, Q:] == 7).all())
    low = torch.full((P, ld + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    wide_add = torch.randint(-64, 64, (P, ld + 8), device="cuda").float()[:, :Q]
    b.mx_gemm(l, r, addend=wide_add, out=low[:, :Q])
    assert same(low[:, :Q], want + wide_add.double())
    assert bool((low[:, Q:] == 7).all())
