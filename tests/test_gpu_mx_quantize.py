"""MX quantization and its way back on the GPU: codes and scales bit for bit as the oracle's."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as mx
from paper_2501_17116_amd import binding as b

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(rows, cols, dtype, seed=0, kind="mixed"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g)
    if kind == "mixed":   # blocks of very different size, zeros, midpoints, the largest and the smallest numbers
        x *= torch.exp(4 * torch.randn(rows, 1, generator=g)) * torch.exp(2 * torch.randn(1, cols, generator=g))
        x[torch.rand(rows, cols, generator=g) < 0.1] = 0.0
        grid = torch.tensor([0.25, -0.75, 1.25, 1.75, -2.5, 3.5, 5.0, 6.0, 7.0, -0.0])
        pick = torch.rand(rows, cols, generator=g) < 0.2
        x[pick] = grid[torch.randint(0, grid.numel(), (int(pick.sum()),), generator=g)]
    return x.to(DT[dtype])


def check(t, x, lines_of):
    """t against the oracle's form of x's lines."""
    ref_c, ref_s = mx.quantize(lines_of(x.float().numpy().astype(np.float64)), t.bits)
    s = t.scales.cpu().numpy()
    assert np.array_equal(s, ref_s)
    c = mx.unpack(t.codes.cpu().numpy())
    ok = np.repeat(s != 255, mx.BLOCK, axis=1)
    assert np.array_equal(np.where(ok, c, 0), np.where(ok, ref_c, 0))
    return mx.values(ref_c, ref_s, t.length)


SHAPES = [(1, 1), (1, 32), (33, 8), (5, 31), (31, 513), (128, 128), (130, 264), (257, 1000), (64, 1544), (700, 72)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_both_axes_and_back(rows, cols, dtype):
    x = make(rows, cols, dtype, seed=rows * 1009 + cols)
    ld = -(-cols // 8) * 8 + 8          # rows apart, and something else between them
    held = torch.full((rows, ld), float("nan"), dtype=DT[dtype], device="cuda")
    xd = held[:, :cols]
    xd.copy_(x)
    for fr in (4, 8):
        r1 = b.mx_quantize(xd, b.FP4_AXIS_ROW, fr)
        vr = check(r1, x, lambda a: a)
        c1 = b.mx_quantize(xd, b.FP4_AXIS_COL, fr)
        vc = check(c1, x, lambda a: a.T)
        for fc in (4, 8):
            r2, c2 = b.mx_quantize_both(xd, fr, fc)
            assert torch.equal(r2.codes, r1.codes) and torch.equal(r2.scales, r1.scales)
            if fc == fr:
                assert torch.equal(c2.codes, c1.codes) and torch.equal(c2.scales, c1.scales)
        for out in (torch.float32, torch.bfloat16):
            for t, v in ((r1, vr), (c1, vc.T)):
                back = b.mx_dequantize(t, out)
                assert back.shape == x.shape and np.array_equal(back.float().cpu().numpy().astype(np.float64), v)
    assert torch.isnan(held[:, cols:]).all()


@pytest.mark.parametrize("bits", [4, 8])
def test_every_bf16_number_and_scale_edges(bits):
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = x[torch.isfinite(x.float())]
    x = x[:x.numel() // 32 * 32]
    own_block = x.reshape(-1, 32)                                   # neighbours share a scale
    far = torch.zeros(x.numel() // 8, 32, dtype=torch.bfloat16)     # and alone beside zeros
    far[:, 5] = x[::8]
    for rows in (own_block, far):
        t = b.mx_quantize(rows.contiguous().cuda(), b.FP4_AXIS_ROW, bits)
        v = check(t, rows, lambda a: a)
        with np.errstate(over="ignore"):
            v = v.astype(np.float32).astype(np.float64)   # the largest numbers may round up to 2^128, which fp32 does not hold
        assert np.array_equal(b.mx_dequantize(t, torch.float32).cpu().numpy().astype(np.float64), v)


@pytest.mark.parametrize("bits", [4, 8])
def test_fp32_beside_every_midpoint(bits):
    grid = mx.MAGNITUDES
    mid = ((grid[1:] + grid[:-1]) / 2)
    if bits == 8:    # the second code's midpoints beside every value of the first
        mid = np.concatenate([mid] + [g + s * mid / 8 for g in grid for s in (1, -1)])
    mid = np.concatenate([grid, mid, [6.75, 7.0]]).astype(np.float32)
    pts = np.concatenate([mid, np.nextafter(mid, np.float32(np.inf)), np.nextafter(mid, np.float32(-np.inf))])
    pts = np.clip(np.concatenate([pts, -pts]), -7, 7)
    pts = np.concatenate([pts, np.zeros(-len(pts) % 31, np.float32)]).reshape(-1, 31)
    x = np.concatenate([pts, np.full((pts.shape[0], 1), 7, np.float32)], axis=1).astype(np.float32)   # the scale is 1 throughout
    x = np.concatenate([np.ldexp(x, e) for e in (-123, -20, 0, 3, 100)]).astype(np.float32)
    x = np.concatenate([x, np.zeros((-x.shape[0] % 8, 32), np.float32)])
    for axis, arr in ((b.FP4_AXIS_ROW, x), (b.FP4_AXIS_COL, x.T)):
        t = torch.from_numpy(np.ascontiguousarray(arr))
        check(b.mx_quantize(t.cuda(), axis, bits), t, (lambda a: a) if axis == b.FP4_AXIS_ROW else (lambda a: a.T))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bits", [4, 8])
def test_infinities_and_nan_stay_in_their_blocks(dtype, bits):
    x = make(70, 136, dtype, seed=4)
    x[3, 40], x[40, 3], x[69, 135] = float("nan"), float("inf"), -float("inf")
    r, c = b.mx_quantize_both(x.cuda(), bits, bits)
    for t, lines_of in ((r, lambda a: a), (c, lambda a: a.T)):
        v = check(t, x, lines_of)
        for out in (torch.float32, torch.bfloat16):
            got = b.mx_dequantize(t, out).float().cpu().numpy().astype(np.float64)
            assert np.array_equal(got, v.T if t.transposed else v, equal_nan=True)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("transposed", [False, True])
def test_every_code_under_every_scale_comes_back(bits, transposed):
    least = 0 if bits == 4 else 4
    lines = 256 - least
    codes = np.tile(np.arange(512) % 16, (1, lines, 1)).astype(np.uint8)
    if bits == 8:
        codes = np.concatenate([codes, np.tile(np.arange(512) // 16 % 16, (1, lines, 1)).astype(np.uint8)])
    scales = np.tile(np.arange(least, 256, dtype=np.uint8)[:, None], (1, 16))
    t = b.MxTensor(torch.from_numpy(mx.pack(codes)).cuda(), torch.from_numpy(scales).cuda(), 512, transposed)
    ref = mx.values(codes, scales, 512)
    with np.errstate(over="ignore"):
        ref = ref.astype(np.float32).astype(np.float64)   # the largest codes under 2^127 are infinite in fp32
    for out in (torch.float32, torch.bfloat16):
        got = b.mx_dequantize(t, out).float().cpu().numpy().astype(np.float64)
        assert np.array_equal(got.T if transposed else got, ref, equal_nan=True)


def test_nothing_to_do():
    for shape in ((0, 64), (64, 0)):
        x = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        r, c = b.mx_quantize_both(x)
        assert r.shape == c.shape == shape
        assert b.mx_dequantize(r).shape == b.mx_dequantize(c).shape == shape


def test_refusals():
    x = torch.zeros(16, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(TypeError):
        b.mx_quantize(x.half(), b.FP4_AXIS_ROW)
    with pytest.raises(ValueError):
        b.mx_quantize(x, b.FP4_AXIS_TENSOR)
    with pytest.raises(ValueError):
        b.mx_quantize(x.t(), b.FP4_AXIS_ROW)
    with pytest.raises(ValueError):
        b.mx_quantize(x.cpu(), b.FP4_AXIS_ROW)
    with pytest.raises(b.Fp4Error):
        b.mx_quantize(torch.zeros(4, 33, dtype=torch.bfloat16, device="cuda"), b.FP4_AXIS_ROW)   # rows 66 bytes apart
    with pytest.raises(b.Fp4Error):
        b.mx_quantize(x[:, 4:], b.FP4_AXIS_ROW)                                                    # begins 8 bytes off
    t = b.mx_quantize(x, b.FP4_AXIS_ROW)
    with pytest.raises(ValueError):
        b.mx_quantize(x, b.FP4_AXIS_ROW, 6)
    with pytest.raises(ValueError):
        b.MxTensor(t.codes.unsqueeze(0), t.scales, 64)
    with pytest.raises(ValueError):
        b.MxTensor(t.codes, t.scales, 513)
    with pytest.raises(ValueError):
        b.mx_dequantize(t, out=torch.empty(16, 65, dtype=torch.bfloat16, device="cuda"))
