"""The product's larger tiles where a workgroup goes through several of them: every combination of output, addend, edge and leading dimension
that its stores tell apart.  Codes under scales of 1: sums are multiples of 1/4 below 2^20, exact in fp32, so that fp64 gives the very bits
(rounded once more for bf16)."""
import pytest
import torch

from paper_2501_17116_amd import binding as b

pytestmark = pytest.mark.gpu


def operand(lines, length, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = b.mx_empty(lines, length)
    t.codes.random_(0, 256, generator=g)
    t.codes[:, length // 2:] = 0
    t.scales.fill_(127)
    return t


def product(l, r):
    return b.mx_dequantize(l, torch.float32).double() @ b.mx_dequantize(r, torch.float32).double().t()


def by_tile(l, r, tile, dtype, ld, addend):
    """Into rows that are ld apart, what lies between them kept."""
    P, Q = l.lines, r.lines
    buf = torch.full((P * ld,), 7.0, dtype=dtype, device="cuda")
    b._check(b.lib().mx_gemm_by_tile(l.ref, r.ref, None if addend is None else addend.data_ptr(), buf.data_ptr(), b._dt(buf), ld, tile, b._stream()), "product")
    rows = buf.view(P, ld)
    assert bool((rows[:, Q:] == 7).all())
    return rows[:, :Q]


@pytest.mark.parametrize("tile", [192, 256])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("with_addend", [False, True])
@pytest.mark.parametrize("P,Q,Kc", [(4352, 4352, 40), (4100, 4360, 512), (4200, 4357, 1100), (4353, 4225, 600)])
def test_several_tiles_a_workgroup(P, Q, Kc, with_addend, dtype, tile):
    l, r = operand(P, Kc, P), operand(Q, Kc, Q)
    ld = (Q + 7) // 8 * 8 + 8
    addend = torch.randint(-64, 64, (P, ld), device="cuda").float() if with_addend else None
    want = product(l, r)
    if with_addend:
        want += addend[:, :Q].double()
    got = by_tile(l, r, tile, dtype, ld, addend)
    assert torch.equal(got.double(), want.to(dtype).double())
    again = by_tile(l, r, tile, dtype, ld, addend)
    assert torch.equal(got, again)


@pytest.mark.parametrize("tile", [192, 256])
@pytest.mark.parametrize("dtype,P,Q", [(torch.float32, 8300, 8456), (torch.bfloat16, 8300, 16904), (torch.bfloat16, 8200, 16901)])
def test_outputs_beyond_the_last_level_cache(dtype, P, Q, tile):
    l, r = operand(P, 72, P), operand(Q, 72, Q)
    ld = (Q + 7) // 8 * 8
    assert P * Q * torch.finfo(dtype).bits // 8 > 256 << 20
    got = by_tile(l, r, tile, dtype, ld, None)
    for first in range(0, P, 2048):
        end = min(first + 2048, P)
        part = b.MxTensor(l.codes[first:end].contiguous(), l.scales[first:end].contiguous(), l.length)
        assert torch.equal(got[first:end].double(), product(part, r).to(dtype).double())


@pytest.mark.parametrize("tile", [192, 256])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_very_far_apart(dtype, tile):
    """32 rows so far apart no longer lie within 2^32 bytes of each other."""
    P, Q, ld = 35, 272, (1 << 25) + 8
    l, r = operand(P, 100, 1), operand(Q, 100, 2)
    out = torch.empty((P - 1) * ld + Q, dtype=dtype, device="cuda")
    b._check(b.lib().mx_gemm_by_tile(l.ref, r.ref, None, out.data_ptr(), b._dt(out), ld, tile, b._stream()), "product")
    got = torch.stack([out[i * ld:i * ld + Q] for i in range(P)])
    assert torch.equal(got.double(), product(l, r).to(dtype).double())
