"""MX layer calls that have nothing to do launch nothing: a launch on a machine without a GPU would come back as FP4_ERR_HIP, and with
buffers that are not there it would write through them on one that has a GPU."""
import ctypes as C

import pytest

from paper_2501_17116_amd import binding as b

one = C.c_void_p(16)   # non-null, aligned, never dereferenced: no call below reaches a GPU
BIG = 1 << 40


def mx(lines, length, bits=4):
    there = 16 if lines and length else None
    return C.byref(b.fp4_mx(there, there, lines, length, bits))


def fwd(M, K, N, bits=4, dt=1, saved=None, ws=one, nb=BIG):
    ptr = lambda rows, cols: one if rows and cols else None
    return b.lib().mx_linear_fwd(ptr(M, K), dt, M, K, N, (K + 7) // 8 * 8, bits, mx(N, K), ptr(M, N), (N + 7) // 8 * 8, saved, ws, nb, None)


@pytest.mark.parametrize("dt", [b.FP4_F32, b.FP4_BF16])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("M,K", [(1, 8), (8, 64), (33, 4096), (5000, 1000), (8, 0)])
def test_forward_pass_of_no_outputs(M, K, bits, dt):
    assert fwd(M, K, 0, bits, dt) == 0
    assert fwd(M, K, 0, bits, dt, ws=None, nb=0) == 0     # and wants no room for it


@pytest.mark.parametrize("K,N", [(64, 16), (0, 16), (64, 0), (0, 0)])
def test_forward_pass_of_no_tokens(K, N):
    assert fwd(0, K, N) == 0 and fwd(0, K, N, saved=mx(K, 0, 8)) == 0


def test_arguments_are_looked_at_first():
    assert fwd(8, 64, 0, bits=6) == -3
    assert fwd(8, 64, 0, saved=mx(8, 64, 8)) == -2
    assert fwd(8, 64, 0, saved=mx(64, 8, 8), ws=None) == -5   # a checkpoint is work
