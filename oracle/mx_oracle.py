"""Plain numpy oracle of the microscaled (MX) operators, from their definitions: blocks of 32 along a line, one power-of-two scale
each (a byte, exponent + 127), codes by search among E2M1's magnitudes, values and products in fp64.  Test infrastructure only."""
from __future__ import annotations

import numpy as np

BLOCK, PITCH = 32, 512
MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float64)
LEAST = {4: -126, 8: -123}   # smallest exponent of a scale


def pitch(length: int) -> int:
    return -(-length // PITCH) * PITCH


def scale_bytes(amax: np.ndarray, bits: int) -> np.ndarray:
    """Scale bytes of blocks with these largest magnitudes (fp64; NaN or inf: 255): the smallest power of two s with amax <= 7 s."""
    bad = ~np.isfinite(amax)
    m, e = np.frexp(np.where(bad, 1.0, amax))          # m 2^e, m in [0.5, 1); 7 = 0.875 2^3
    e = np.where(m <= 0.875, e - 3, e - 2)
    e = np.where(m == 0, LEAST[bits], np.clip(e, LEAST[bits], 127))
    return np.where(bad, 255, e + 127).astype(np.uint8)


def round_codes(v: np.ndarray) -> np.ndarray:
    """Nearest codes of scaled values, ties to the even code, saturating, the sign kept on zero."""
    mid = (MAGNITUDES[1:] + MAGNITUDES[:-1]) / 2
    a = np.abs(v)
    down, up = np.searchsorted(mid, a, side="left"), np.searchsorted(mid, a, side="right")
    code = np.where(down % 2 == 0, down, up)
    return (code | (np.signbit(v).astype(np.int64) << 3)).astype(np.uint8)


def code_values(codes: np.ndarray) -> np.ndarray:
    return MAGNITUDES[codes & 7] * np.where(codes & 8, -1.0, 1.0)


def quantize(x: np.ndarray, bits: int):
    """x [lines, length] -> (one code per byte [bits / 4, lines, pitch], scale bytes [lines, pitch / 32])."""
    lines, length = x.shape
    p = pitch(length)
    full = np.zeros((lines, p), np.float64)
    full[:, :length] = x
    blocks = full.reshape(lines, p // BLOCK, BLOCK)
    with np.errstate(invalid="ignore"):
        amax = np.abs(blocks).max(axis=2)     # NaN wins
    s = scale_bytes(amax, bits)
    e = np.where(s == 255, 0, s.astype(np.int64) - 127)[:, :, None]
    v = np.ldexp(np.where((s == 255)[:, :, None], 0.0, blocks), -e)
    planes = [round_codes(v)]
    if bits == 8:
        planes.append(round_codes(8 * (v - code_values(planes[0]))))
    return np.stack(planes).reshape(bits // 4, lines, p), s


def values(codes: np.ndarray, scales: np.ndarray, length: int) -> np.ndarray:
    """What one-per-byte codes and their scales stand for, fp64 [lines, length]."""
    v = code_values(codes[0])
    if codes.shape[0] == 2:
        v = v + code_values(codes[1]) / 8
    lines, p = v.shape
    s = scales.astype(np.int64)[:, :, None]
    v = np.where(s == 255, np.nan, np.ldexp(v.reshape(lines, p // BLOCK, BLOCK), s - 127))
    return v.reshape(lines, p)[:, :length]


def pack(codes: np.ndarray) -> np.ndarray:
    """As an MX tensor holds them: two to a byte, the earlier in the low half; one plane without its axis."""
    p = (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)
    return p[0] if p.shape[0] == 1 else p


def unpack(packed: np.ndarray) -> np.ndarray:
    if packed.ndim == 2:
        packed = packed[None]
    return np.stack([packed & 15, packed >> 4], axis=-1).reshape(packed.shape[0], packed.shape[1], -1)


def through(x: np.ndarray, bits: int) -> np.ndarray:
    """x as its MX form along its lines holds it."""
    c, s = quantize(x, bits)
    return values(c, s, x.shape[1])
