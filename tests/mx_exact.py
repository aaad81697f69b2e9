"""MX operands whose products are exact in fp32 in any order of their sums, and the products in fp64."""
import torch

from paper_2501_17116_amd import binding as b

MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def operand(lines, length, bits, seed, octaves=1):
    """Random codes, zeros behind `length`, under random scales from 1 to 2^octaves."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = b.mx_empty(lines, length, bits)
    t.codes.random_(0, 256, generator=g)
    t.codes[..., (length + 1) // 2:] = 0
    if length % 2:
        t.codes[..., length // 2] &= 15
    t.scales.random_(127, 128 + octaves, generator=g)
    return t


def values(t):
    """fp64, by a table; byte 255 stands for NaN."""
    table = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), dtype=torch.float64, device="cuda")
    planes = t.codes if t.bits == 8 else t.codes.unsqueeze(0)
    total = torch.zeros(t.lines, planes.shape[2] * 2, dtype=torch.float64, device="cuda")
    for p, part in zip(planes, (1.0, 0.125)):
        total[:, 0::2] += table[(p & 15).long()] * part
        total[:, 1::2] += table[(p >> 4).long()] * part
    scale = torch.exp2(t.scales.double() - 127)
    scale[t.scales == 255] = float("nan")
    return (total * scale.repeat_interleave(32, dim=1))[:, :t.length].contiguous()


def product(l, r):
    """fp64, and checked to be exact in fp32: sums of multiples of the smallest product that stay below 2^24 of it, whatever their order."""
    vl, vr = values(l), values(r)
    unit = (1.0 if l.bits == 4 else 0.125) * (1.0 if r.bits == 4 else 0.125) / 4
    largest = torch.nan_to_num(vl, 0.0).abs() @ torch.nan_to_num(vr, 0.0).abs().t().contiguous()
    assert float(largest.max()) < unit * 2 ** 24
    return vl @ vr.t().contiguous()


def same(got, want):
    """Bit for bit, NaN where NaN is wanted."""
    nan = torch.isnan(want)
    return torch.equal(torch.isnan(got), nan) and torch.equal(torch.where(nan, 0.0, got.double()), torch.where(nan, 0.0, want.to(got.dtype).double()))
