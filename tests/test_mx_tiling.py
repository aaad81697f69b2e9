"""Which kernel takes an MX product: host arithmetic, no GPU."""
import random

import pytest

from paper_2501_17116_amd import binding as b


@pytest.mark.parametrize("shape,tile", [
    ((1, 4096, 4096), 16), ((32, 5120, 13824), 16), ((33, 4768, 696), 16), ((64, 2048, 2048), 16),
    ((62, 2488, 10296), 32), ((256, 4096, 4096), 32), ((512, 512, 512), 32),
    ((1332, 680, 432), 64), ((2114, 432, 736), 64),
    ((2048, 2048, 2048), 128), ((1376, 2080, 1055), 128), ((687, 7680, 576), 128),
    ((8192, 2048, 5504), 256), ((16384, 12288, 4096), 256), ((4096, 4096, 8192), 256),
])
def test_tiles_of_known_shapes(shape, tile):
    assert b.mx_gemm_tile(*shape)[0] == tile


def test_the_passes_of_eight_bits_count():
    assert b.mx_gemm_tile(64, 2048, 2048, 4, 4)[0] == 16 and b.mx_gemm_tile(64, 2048, 2048, 8, 4)[0] == 32
    assert b.mx_gemm_tile(1332, 680, 432, 4, 4)[0] == 64 and b.mx_gemm_tile(1332, 680, 432, 8, 8)[0] == 32
    assert b.mx_gemm_tile(2048, 5504, 8192, 8, 4)[0] == 192


def test_an_empty_contraction_goes_where_nothing_is_requested_ahead():
    for P, Q in ((1, 1), (64, 64), (5000, 5000)):
        assert b.mx_gemm_tile(P, Q, 0) == (64, 0)


def test_last_rounds():
    """At most a quarter of the CUs' worth of tiles, and only behind full rounds."""
    seen = 0
    rng = random.Random(1)
    for _ in range(4000):
        P, Q, K = rng.randint(65, 20000), 8 * rng.randint(1, 2000), rng.randint(1, 16000)
        tile, rest = b.mx_gemm_tile(P, Q, K, rng.choice([4, 8]), rng.choice([4, 8]))
        assert tile in (16, 32, 64, 128, 192, 256)
        t256 = -(-P // 256) * -(-Q // 256)
        if rest:
            seen += 1
            assert tile == 256 and t256 > 256 and rest == t256 % 256 and rest <= 64
    assert seen > 20


def test_refusals():
    for bad in ((0, 8, 8), (8, 0, 8), (8, 8, -1)):
        with pytest.raises(b.Fp4Error):
            b.mx_gemm_tile(*bad)
    with pytest.raises(b.Fp4Error):
        b.mx_gemm_tile(8, 8, 8, compute_units=4)
