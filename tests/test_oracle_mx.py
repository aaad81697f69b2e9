"""The MX oracle against its definitions, element by element."""
import itertools
import math

import numpy as np
import pytest

from oracle import mx_oracle as mx


def _nearest_even(v):
    """By the definition: the magnitude with the least distance, of two the one with the even code."""
    d = np.abs(mx.MAGNITUDES - abs(v))
    best = [c for c in range(8) if d[c] == d.min()]
    return best[0] if len(best) == 1 else next(c for c in best if c % 2 == 0)


def test_codes_are_the_nearest_ones_and_ties_go_to_the_even_code():
    grid = mx.MAGNITUDES
    mid = (grid[1:] + grid[:-1]) / 2
    pts = np.concatenate([grid, mid, np.nextafter(mid, np.inf), np.nextafter(mid, -np.inf), [6.5, 7.0, 100.0]])
    pts = np.concatenate([pts, -pts, np.random.default_rng(0).uniform(-7, 7, 500)])
    for v, c in zip(pts, mx.round_codes(pts)):
        assert (c & 7) == _nearest_even(v), v
        assert bool(c & 8) == bool(np.signbit(v)), v
        assert mx.code_values(np.array([c]))[0] == math.copysign(grid[c & 7], v)


@pytest.mark.parametrize("bits", [4, 8])
def test_scale_of_a_block(bits):
    for e in (-130, -126, -121, -3, 0, 1, 60, 127):
        for m in (1.0, 1.25, 1.5, 1.75, 1.7500002, 1.9999999):
            a = math.ldexp(m, e)
            if a > 3.4028234e38:
                continue
            want = next(k for k in range(e - 6, e + 2) if a <= 7.0 * math.ldexp(1.0, k))
            assert mx.scale_bytes(np.array([a]), bits)[0] == min(max(want, mx.LEAST[bits]), 127) + 127
    assert mx.scale_bytes(np.array([0.0]), bits)[0] == (1 if bits == 4 else 4)
    assert list(mx.scale_bytes(np.array([np.inf, np.nan]), bits)) == [255, 255]


@pytest.mark.parametrize("bits", [4, 8])
def test_values_stay_within_the_grids_error(bits):
    rng = np.random.default_rng(1)
    x = rng.normal(size=(7, 100)) * np.exp(rng.normal(size=(7, 100)) * 3)
    v = mx.through(x, bits)
    for r, b in itertools.product(range(7), range(4)):
        part = slice(b * 32, min(100, b * 32 + 32))
        s = 2.0 ** (int(mx.scale_bytes(np.array([np.abs(x[r, part]).max()]), bits)[0]) - 127)
        a = np.abs(x[r, part]) / s
        half = np.where(a <= 2, 0.25, np.where(a <= 4, 0.5, 1.0))       # of the grid's spacing where the value lies
        if bits == 8:   # what is left lies within +-8 half / 8: its own grid has spacing 1/2, 1 or 2 there, over 6 it saturates
            half = np.where(half == 0.25, 0.25 / 8, np.where(half == 0.5, 0.5 / 8, 2.0 / 8))
        assert np.all(np.abs(v[r, part] - x[r, part]) <= half * s)


def test_eight_bits_have_seven_significant_ones():
    h, l = np.meshgrid(np.arange(16), np.arange(16))
    v = mx.code_values(h) + mx.code_values(l) / 8
    m, _ = np.frexp(v)
    assert np.array_equal(m * 128, np.round(m * 128))


@pytest.mark.parametrize("bits", [4, 8])
def test_a_bad_element_makes_its_block_nan_and_no_other(bits):
    x = np.ones((2, 70))
    x[0, 33], x[1, 69] = np.nan, -np.inf
    v = mx.through(x, bits)
    assert np.isnan(v[0, 32:64]).all() and np.isnan(v[1, 64:]).all()
    assert np.isfinite(np.delete(v[0], range(32, 64))).all() and np.isfinite(v[1, :64]).all()


def test_pack_and_unpack():
    for planes in (1, 2):
        c = np.random.default_rng(2).integers(0, 16, (planes, 3, 512)).astype(np.uint8)
        p = mx.pack(c)
        assert p.shape == ((3, 256) if planes == 1 else (2, 3, 256))
        assert np.array_equal(mx.unpack(p), c)
    assert p[1, 2, 5] == c[1, 2, 10] | (c[1, 2, 11] << 4)
    assert mx.pitch(1) == 512 and mx.pitch(512) == 512 and mx.pitch(513) == 1024 and mx.pitch(0) == 0
