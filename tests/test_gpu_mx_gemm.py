"""The MX product against fp64 on the same codes and scales.

Tolerance of an fp32 result: a matrix instruction adds 64 products to its accumulator; each such step may lose two bits of fp32 against
the largest partial sum there can be, which sum |l||r| bounds (over the planes of 8 bits: less than twice that), and so may each joining
of partial sums (fewer than 16): (4 steps + 16) 2^-21 sum |l||r| with the four passes that two operands of 8 bits take.  A bf16 result is that
rounded once more to eight significant bits: 2^-8 of its value at most."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as mx
from paper_2501_17116_amd import binding as b

pytestmark = pytest.mark.gpu
BITS = [(4, 4), (8, 4), (4, 8), (8, 8)]


def operand(lines, length, bits, seed, spread=2.0):
    """Random codes under random scales, and their values in fp64."""
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(lines, length)) * np.exp(spread * rng.normal(size=(lines, length)))
    c, s = mx.quantize(x, bits)
    return b.MxTensor(torch.from_numpy(mx.pack(c)).cuda(), torch.from_numpy(s).cuda(), length), mx.values(c, s, length)


def bound(vl, vr, length):
    return (4 * np.ceil(length / 64) + 16) * 2.0 ** -21 * (np.abs(vl) @ np.abs(vr).T)


def close(got, ref, tol, bf16=False):
    got = got.float().cpu().numpy().astype(np.float64)
    if bf16:
        tol = 1.01 * tol + 1.01 * 2.0 ** -8 * np.abs(ref)
    worst = np.max(np.abs(got - ref) - tol)
    assert worst <= 0, "off by %g more than allowed at %s" % (worst, np.unravel_index(np.argmax(np.abs(got - ref) - tol), ref.shape))


SHAPES = [(1, 1, 1), (1, 8, 32), (3, 40, 520), (17, 64, 64), (64, 64, 512), (65, 72, 1000), (130, 200, 96), (33, 1000, 2049), (300, 264, 600)]


@pytest.mark.parametrize("bl,br", BITS)
@pytest.mark.parametrize("P,Q,Kc", SHAPES)
def test_products(P, Q, Kc, bl, br):
    l, vl = operand(P, Kc, bl, P + 7 * Q + Kc)
    r, vr = operand(Q, Kc, br, P + 7 * Q + Kc + 1)
    ref, tol = vl @ vr.T, bound(vl, vr, Kc)
    close(b.mx_gemm(l, r), ref, tol)
    close(b.mx_gemm(l, r, torch.bfloat16), ref, tol, bf16=True)


@pytest.mark.parametrize("bl,br", BITS)
@pytest.mark.parametrize("P,Q,Kc", [(2050, 2056, 40), (1800, 3000, 520), (4100, 1032, 1100)])
def test_outputs_of_many_tiles(P, Q, Kc, bl, br):
    """Rows and columns past the last tile's edge, one step of the contraction and several, with an addend and without."""
    l, vl = operand(P, Kc, bl, P + Kc)
    r, vr = operand(Q, Kc, br, Q + Kc)
    ref, tol = vl @ vr.T, bound(vl, vr, Kc)
    close(b.mx_gemm(l, r, torch.bfloat16), ref, tol, bf16=True)
    got = b.mx_gemm(l, r)
    close(got, ref, tol)
    add = torch.randn(P, Q, device="cuda") * float(np.abs(ref).mean())
    host = add.double().cpu().numpy()
    close(b.mx_gemm(l, r, addend=add, out=add), ref + host, tol + 2.0 ** -22 * np.abs(host))
    assert torch.equal(b.mx_gemm(l, r), got)


@pytest.mark.parametrize("tile", [16, 32, 64, 128, 192, 256])
@pytest.mark.parametrize("bl,br", BITS)
@pytest.mark.parametrize("P,Q,Kc", [(1, 8, 8), (70, 40, 2000), (129, 264, 513), (513, 528, 1536)])
def test_every_tile_gives_the_product(P, Q, Kc, bl, br, tile):
    """One row, edges inside every tile, one to eight steps of the contraction, whatever the rule would take."""
    l, vl = operand(P, Kc, bl, P + Kc)
    r, vr = operand(Q, Kc, br, Q + Kc)
    ref, tol = vl @ vr.T, bound(vl, vr, Kc)
    close(b.mx_gemm_by_tile(l, r, tile), ref, tol)
    close(b.mx_gemm_by_tile(l, r, tile, torch.bfloat16), ref, tol, bf16=True)
    add = torch.randn(P, Q, device="cuda") * float(np.abs(ref).mean())
    close(b.mx_gemm_by_tile(l, r, tile, addend=add), ref + add.double().cpu().numpy(), tol + 2.0 ** -22 * np.abs(add.double().cpu().numpy()))


@pytest.mark.parametrize("bl,br", BITS)
@pytest.mark.parametrize("P,Q,Kc", [(5, 24, 100), (200, 136, 700), (600, 520, 1100)])
def test_addend_and_accumulation_and_rows_apart(P, Q, Kc, bl, br):
    l, vl = operand(P, Kc, bl, 11)
    r, vr = operand(Q, Kc, br, 12)
    tol = bound(vl, vr, Kc)
    add = torch.randn(P, Q, device="cuda") * float(np.abs(vl @ vr.T).mean())
    ref = vl @ vr.T + add.double().cpu().numpy()
    tol = tol + 2.0 ** -22 * np.abs(add.double().cpu().numpy())
    close(b.mx_gemm(l, r, addend=add), ref, tol)
    close(b.mx_gemm(l, r, torch.bfloat16, addend=add), ref, tol, bf16=True)
    acc = add.clone()
    b.mx_gemm(l, r, addend=acc, out=acc)
    close(acc, ref, tol)
    wide = torch.full((P + 1, Q + 24), 7.0, device="cuda")     # a view: nothing beside it changes
    b.mx_gemm(l, r, out=wide[:P, 8:8 + Q])
    close(wide[:P, 8:8 + Q], vl @ vr.T, bound(vl, vr, Kc))
    wide[:P, 8:8 + Q] = 7.0
    assert bool((wide == 7.0).all())


@pytest.mark.parametrize("bl,br", BITS)
def test_small_values_come_out_exactly(bl, br):
    """Scales of 1: every product is a multiple of 2^-8 and every sum below 2^16, exact in fp32 in any order."""
    rng = np.random.default_rng(3)
    P, Q, Kc = 96, 160, 1500

    def make(lines, bits):
        x = rng.integers(-32, 33, size=(lines, Kc)) / (16.0 if bits == 8 else 2.0 * 8)
        x[:, ::32] = 4.0   # the scale comes out as 1
        c, s = mx.quantize(x, bits)
        assert np.all(s[:, : -(-Kc // 32)] == 127)
        return b.MxTensor(torch.from_numpy(mx.pack(c)).cuda(), torch.from_numpy(s).cuda(), Kc), mx.values(c, s, Kc)

    l, vl = make(P, bl)
    r, vr = make(Q, br)
    assert np.array_equal(b.mx_gemm(l, r).cpu().numpy().astype(np.float64), vl @ vr.T)


@pytest.mark.parametrize("P,Q", [(8, 16), (300, 264)])
def test_a_nan_block_reaches_its_row_and_column_alone(P, Q):
    l, vl = operand(P, 200, 4, 21)
    r, vr = operand(Q, 200, 8, 22)
    l.scales[5, 3] = 255
    r.scales[Q - 2, 0] = 255
    got = b.mx_gemm(l, r).cpu().numpy()
    bad = np.zeros((P, Q), bool)
    bad[5], bad[:, Q - 2] = True, True
    assert np.array_equal(np.isnan(got), bad)
    assert np.all(np.abs(got - vl @ vr.T)[~bad] <= bound(vl, vr, 200)[~bad])


def test_scales_at_the_ends_of_their_range():
    c = np.full((1, 32, 512), 2, np.uint8)      # ones
    for el, er in ((-126, 126), (-100, 100), (127, -127 + 1), (-60, -60), (60, 60)):
        sl, sr = np.full((32, 16), el + 127, np.uint8), np.full((32, 16), er + 127, np.uint8)
        l = b.MxTensor(torch.from_numpy(mx.pack(c)).cuda(), torch.from_numpy(sl).cuda(), 512)
        r = b.MxTensor(torch.from_numpy(mx.pack(c)).cuda(), torch.from_numpy(sr).cuda(), 512)
        assert bool((b.mx_gemm(l, r) == 512.0 * 2.0 ** (el + er)).all())


def test_contraction_of_no_length():
    l, r = b.mx_empty(9, 0, 4), b.mx_empty(16, 0, 8)
    assert bool((b.mx_gemm(l, r) == 0).all())
    add = torch.randn(9, 16, device="cuda")
    assert torch.equal(b.mx_gemm(l, r, addend=add), add)


def test_the_same_call_gives_the_same_bits():
    l, _ = operand(200, 3000, 8, 31)
    r, _ = operand(264, 3000, 4, 32)
    first = b.mx_gemm(l, r)
    for _ in range(3):
        assert torch.equal(b.mx_gemm(l, r), first)


def test_refusals():
    l, _ = operand(4, 64, 4, 1)
    r, _ = operand(16, 96, 4, 1)
    with pytest.raises(ValueError):
        b.mx_gemm(l, r)
    r, _ = operand(16, 64, 4, 1)
    with pytest.raises(ValueError):
        b.mx_gemm(l, r, out=torch.empty(4, 8, device="cuda"))
    with pytest.raises(TypeError):
        b.mx_gemm(l, r, torch.float16)
    with pytest.raises(ValueError):
        b.mx_gemm(l, r, addend=torch.zeros(4, 16, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        b.mx_gemm(l, r, addend=torch.zeros(4, 24, device="cuda")[:, :16])       # not out's leading dimension
    with pytest.raises(b.Fp4Error):
        b.mx_gemm(l, r, out=torch.empty(4, 18, device="cuda")[:, :16])
