"""What the MX entry points refuse, and the room they ask for: host arithmetic, nothing reaches a GPU."""
import ctypes as C
import itertools

import pytest

from paper_2501_17116_amd import binding as b

BIG = 1 << 40
OK, NULL, SHAPE, DTYPE, ARG, WORKSPACE, LIMIT = 0, -1, -2, -3, -4, -5, -8
one = C.c_void_p(16)   # non-null, aligned, never dereferenced: every call below fails first, or has nothing to do


@pytest.fixture(scope="module")
def L():
    return b.lib()


def mx(lines, length, bits=4, codes=16, scales=16):
    return C.byref(b.fp4_mx(codes, scales, lines, length, bits))


def test_pitch(L):
    for n in (0, 1, 511, 512, 513, 4096, 5504, 1 << 40):
        assert L.mx_pitch(n) == b.mx_pitch(n) == (n + 511) // 512 * 512
    assert L.mx_pitch(-1) == -1


def test_quantize_refusals(L):
    q = lambda x=one, dt=0, rows=4, cols=16, ld=16, r=None, c=None: L.mx_quantize(x, dt, rows, cols, ld, r, c, None)
    good = mx(4, 16)
    assert q() == NULL                                             # neither axis
    assert q(x=None, r=good) == NULL
    assert q(dt=2, r=good) == DTYPE
    assert q(ld=8, r=good) == SHAPE                                # ld < cols
    assert q(ld=20, r=good) == ARG                                 # ld % 8
    assert q(x=C.c_void_p(24), r=good) == ARG
    assert q(rows=-1, r=mx(-1, 16)) == SHAPE
    assert q(r=mx(5, 16)) == SHAPE and q(r=mx(4, 17)) == SHAPE
    assert q(c=mx(4, 16)) == SHAPE                                 # along the columns lines are columns
    assert q(r=mx(4, 16, bits=2)) == DTYPE and q(r=good, c=mx(16, 4, bits=16)) == DTYPE
    assert q(r=mx(4, 16, codes=None)) == NULL and q(r=mx(4, 16, scales=None)) == NULL
    assert q(r=mx(4, 16, codes=24)) == ARG and q(r=mx(4, 16, scales=17)) == ARG
    assert q(r=good, c=mx(16, 4, codes=8)) == ARG
    assert q(rows=(1 << 21) + 1, r=mx((1 << 21) + 1, 16)) == LIMIT
    assert q(rows=0, r=mx(0, 16, codes=None, scales=None)) == OK   # nothing to do
    assert q(x=None, cols=0, ld=0, c=mx(0, 4)) == OK


def test_dequantize_refusals(L):
    d = lambda t, tr=0, x=one, dt=0, ld=16: L.mx_dequantize(t, tr, x, dt, ld, None)
    assert d(None) == NULL
    assert d(mx(4, 16), x=None) == NULL
    assert d(mx(4, 16), dt=7) == DTYPE
    assert d(mx(4, 16, bits=9)) == DTYPE
    assert d(mx(4, 16), ld=8) == SHAPE and d(mx(16, 4), tr=1, ld=8) == SHAPE
    assert d(mx(4, 16), ld=17) == ARG
    assert d(mx(4, 16, codes=None)) == NULL and d(mx(4, 16, scales=20)) == ARG
    assert d(mx(-4, 16)) == SHAPE
    assert d(mx(0, 16, codes=None, scales=None), x=None) == OK


def test_gemm_refusals(L):
    g = lambda l, r, add=None, out=one, dt=0, ldo=16: L.mx_gemm(l, r, add, out, dt, ldo, None)
    assert g(None, mx(16, 64)) == NULL and g(mx(4, 64), None) == NULL
    assert g(mx(4, 64), mx(16, 96)) == SHAPE
    assert g(mx(4, 64), mx(17, 64)) == SHAPE                       # ldo < Q
    assert g(mx(4, -1), mx(16, -1)) == SHAPE
    assert g(mx(4, 64), mx(16, 64), ldo=20) == ARG
    assert g(mx(4, 64), mx(16, 64), dt=3) == DTYPE
    assert g(mx(4, 64, bits=5), mx(16, 64)) == DTYPE
    assert g(mx(4, 64), mx(16, 64), out=None) == NULL
    assert g(mx(4, 64), mx(16, 64), add=C.c_void_p(20)) == ARG
    assert g(mx(4, 64, codes=None), mx(16, 64)) == NULL
    assert g(mx(4, 1 << 22), mx(16, 1 << 22)) == LIMIT
    assert g(mx(0, 64), mx(16, 64)) == OK and g(mx(4, 64), mx(0, 64), ldo=0) == OK


def test_layer_refusals(L):
    def fwd(M=8, K=64, N=16, dt=1, lda=64, bits=4, W=None, ldy=16, saved=None, ws=one, nb=BIG, A=one, Y=one):
        return L.mx_linear_fwd(A, dt, M, K, N, lda, bits, mx(N, K) if W is None else W, Y, ldy, saved, ws, nb, None)
    assert fwd(A=None) == NULL and fwd(Y=None) == NULL and fwd(ws=None) == WORKSPACE and fwd(nb=16) == WORKSPACE
    assert fwd(dt=5) == DTYPE and fwd(bits=6) == DTYPE and fwd(lda=56) == SHAPE and fwd(ldy=12) == SHAPE and fwd(ldy=20) == ARG
    assert fwd(W=mx(64, 16)) == SHAPE and fwd(W=mx(16, 64, codes=None)) == NULL
    assert fwd(saved=mx(8, 64, bits=8)) == SHAPE and fwd(saved=mx(64, 8, bits=0)) == DTYPE
    assert fwd(M=0, A=None, Y=None) == OK
    dgrad = lambda M=8, K=64, N=16, W=None, ldy=16, lda=64, ws=one, nb=BIG: L.mx_linear_bwd_dgrad(
        one, 1, M, K, N, ldy, mx(K, N) if W is None else W, one, lda, ws, nb, None)
    assert dgrad(W=mx(16, 64)) == SHAPE and dgrad(ldy=8) == SHAPE and dgrad(lda=32) == SHAPE and dgrad(nb=8) == WORKSPACE
    wgrad = lambda M=8, K=64, N=16, saved=None, bits=4, ldw=16, dW=one, nb=BIG: L.mx_linear_bwd_wgrad(
        one, 1, M, K, N, 16, mx(K, M, bits=8) if saved is None else saved, bits, 0, dW, ldw, one, nb, None)
    assert wgrad(saved=mx(8, 64)) == SHAPE and wgrad(bits=3) == DTYPE and wgrad(ldw=8) == SHAPE and wgrad(dW=None) == NULL and wgrad(nb=8) == WORKSPACE
    both = lambda W=None, saved=None, dA=one, nb=BIG: L.mx_linear_bwd(
        one, 1, 8, 64, 16, 16, mx(64, 16) if W is None else W, mx(64, 8, bits=8) if saved is None else saved, 4, dA, 64, 1, one, 16, one, nb, None)
    assert both(W=mx(16, 64)) == SHAPE and both(saved=mx(64, 9)) == SHAPE and both(dA=None) == NULL and both(nb=8) == WORKSPACE


@pytest.mark.parametrize("op", [b.FP4_OP_MX_FWD, b.FP4_OP_MX_DGRAD, b.FP4_OP_MX_WGRAD, b.FP4_OP_MX_BWD])
def test_workspaces_hold_what_a_pass_quantizes_and_grow_along_every_dimension(L, op):
    sizes = [1, 31, 32, 33, 511, 512, 513, 1000, 4096, 5504, 16384]
    for M, K, N in itertools.product(sizes, repeat=3):
        need = b.workspace_bytes(op, M, K, N, b.FP4_BF16)
        rows, cols = (M, K) if op == b.FP4_OP_MX_FWD else (M, N)
        held = 0
        if op == b.FP4_OP_MX_FWD:
            held = M * (b.mx_pitch(K) + b.mx_pitch(K) // 32)
        if op in (b.FP4_OP_MX_DGRAD, b.FP4_OP_MX_BWD):
            held += M * (b.mx_pitch(N) // 2 + b.mx_pitch(N) // 32)
        if op in (b.FP4_OP_MX_WGRAD, b.FP4_OP_MX_BWD):
            held += N * (b.mx_pitch(M) + b.mx_pitch(M) // 32)
        assert need >= held, (M, K, N)
    for fixed in itertools.product((1, 500, 4096), repeat=2):
        for dim in range(3):
            got = [b.workspace_bytes(op, *fixed[:dim], v, *fixed[dim:], b.FP4_F32) for v in sizes]
            assert got == sorted(got)
    assert b.workspace_bytes(op, -1, 4, 4, b.FP4_F32) == 0
