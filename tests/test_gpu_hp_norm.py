"""The joint of two blocks and its gradients against the formulas in 64 bits and against differences."""
import pytest
import torch

from paper_2501_17116_amd import binding as b
from tests import hp_plain as plain

pytestmark = pytest.mark.gpu

EPS = 1e-5
DTYPES = [torch.bfloat16, torch.float32]
SIZES = [(1, 1), (1, 8), (1, 4096), (3, 7), (5, 513), (17, 1377), (300, 2048), (64, 5120), (2, 16384), (9, 16377), (2100, 72)]


def inputs(M, D, dtype, block=True, after=True, gate="vector", before=True, seed=0, pad=1):
    g = torch.Generator().manual_seed(seed)
    def normal(*s):
        return torch.randn(*s, generator=g)
    x = plain.matrix(normal(M, D) * torch.where(torch.rand(D, generator=g) < 0.01, 30.0, 1.0), dtype, pad)
    blk = plain.matrix(normal(M, D) * 0.5, dtype, 2 * pad) if block else None
    vec = lambda m, s: (m + s * normal(D)).to(dtype).cuda()
    w_after = vec(1.0, 0.1) if block and after else None
    gt = None
    if block and gate == "vector":
        gt = vec(0.5, 0.2)
    if block and gate == "token":
        gt = plain.matrix(torch.sigmoid(normal(M, D)), dtype, 3 * pad)
    return x, blk, vec(1.0, 0.1) if before else None, w_after, gt, normal


def check_forward(norm, x, blk, h, y, saved):
    t = plain.half_step(x.dtype)
    rh, ry, rb, ra, size, size_y = plain.joint(x, blk, norm.w_before, norm.w_after, norm.gate, norm.scale, norm.eps)
    plain.close(h, rh, t * rh.abs() + plain.ROW * size, "h")
    if norm.w_before is not None:
        plain.close(y, ry, t * ry.abs() + plain.ROW * 2 * size_y, "y")
        plain.close(saved.r_before, rb, 2 * plain.ROW * rb, "r_before")
    if norm.w_after is not None:
        plain.close(saved.r_after, ra, plain.ROW * ra, "r_after")


def check_backward(norm, saved, h, dy, dh, blk, got, M):
    t = plain.half_step(h.dtype)
    want = plain.joint_gradients(h, dy, dh, blk, norm.w_before, norm.w_after, norm.gate, norm.scale, saved.r_before, saved.r_after)
    for name, (value, size) in want.items():
        g = getattr(got, name)
        if value.dim() == 2:
            plain.close(g, value, t * value.abs() + 3 * plain.ROW * size, name)
        else:
            plain.close(g, value, (M * plain.U + 3 * plain.ROW) * size, name)
    for name in set(b.HpNormGrads._fields) - set(want):
        assert getattr(got, name) is None, name


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,D", SIZES)
@pytest.mark.parametrize("form", ["plain", "after", "vector", "token", "alone"])
def test_forward_and_backward(M, D, dtype, form):
    x, blk, wb, wa, gate, normal = inputs(M, D, dtype, block=form != "alone", after=form in ("after", "vector", "token"),
                                          gate=form if form in ("vector", "token") else None)
    norm = b.HpNorm(wb, wa, gate, scale=0.7 if form != "plain" else 1.0, eps=EPS)
    saved = b.hp_norm_saved(norm, M)
    h, y = b.hp_norm_fwd(norm, x, blk, saved)
    check_forward(norm, x, blk, h, y, saved)
    dy, dh = plain.matrix(normal(M, D) * 0.1, dtype, 1), plain.matrix(normal(M, D) * 0.1, dtype)
    got = b.hp_norm_bwd(norm, saved, h, dy, dh, blk)
    check_backward(norm, saved, h, dy, dh, blk, got, M)


@pytest.mark.parametrize("dtype", DTYPES)
def test_parts_of_a_joint(dtype):
    M, D = 33, 648
    x, blk, wb, wa, gate, normal = inputs(M, D, dtype)
    dy, dh = plain.matrix(normal(M, D), dtype), plain.matrix(normal(M, D), dtype)
    for before, after, g in [(None, wa, None), (None, None, gate), (wb, None, gate), (None, wa, gate)]:
        norm = b.HpNorm(before, after, g, scale=-1.5)
        saved = b.hp_norm_saved(norm, M)
        h, y = b.hp_norm_fwd(norm, x, blk, saved)
        check_forward(norm, x, blk, h, y, saved)
        assert (y is None) == (before is None)
        for a, c in [(dy, None), (None, dh), (dy, dh)]:
            if a is not None and before is None:
                continue
            check_backward(norm, saved, h, a, c, blk, b.hp_norm_bwd(norm, saved, h, a, c, blk), M)


def test_against_differences():
    """fp32, a step in one direction of all inputs: the gradients' product with it is the change of a weighted sum of the outputs."""
    M, D = 6, 40
    x, blk, wb, wa, gate, normal = inputs(M, D, torch.float32, gate="token", pad=0)
    cy, ch = normal(M, D).cuda(), normal(M, D).cuda()
    leaves = [t.double() for t in (x, blk, wb, wa, gate)]
    steps = [torch.randn(t.shape, generator=torch.Generator().manual_seed(i), dtype=torch.float64).cuda() for i, t in enumerate(leaves)]

    def value(e):
        a = [t + e * s for t, s in zip(leaves, steps)]
        h, y, *_ = plain.joint(a[0], a[1], a[2], a[3], a[4], 0.7, EPS)
        return float((h * ch.double()).sum() + (y * cy.double()).sum())

    norm = b.HpNorm(wb, wa, gate, scale=0.7, eps=EPS)
    saved = b.hp_norm_saved(norm, M)
    h, _ = b.hp_norm_fwd(norm, x, blk, saved)
    d = b.hp_norm_bwd(norm, saved, h, cy, ch, blk)
    got = sum(float((g.double() * s).sum()) for g, s in zip((d.dx, d.dblock, d.dw_before, d.dw_after, d.dgate), steps))
    e = 1e-5
    want = (value(e) - value(-e)) / (2 * e)
    # differences: e^2 times third derivatives of order 10 M D; gradients: fp32
    assert abs(got - want) <= 1e-5 * M * D, (got, want)


def test_rows_of_zeros_and_large_values():
    D = 256
    w = torch.ones(D, device="cuda")
    x = torch.zeros(3, D, device="cuda")
    x[1] = 1e18
    norm = b.HpNorm(w, eps=1e-6)
    saved = b.hp_norm_saved(norm, 3)
    h, y = b.hp_norm_fwd(norm, x, saved=saved)
    assert torch.equal(h, x) and torch.equal(y[0], x[0]) and torch.equal(y[2], x[0])
    assert float((y[1] - 1.0).abs().max()) <= 2 * plain.ROW
    assert float((saved.r_before[0] - 1e3).abs()) <= 1e3 * plain.ROW


def test_padding_is_left_alone_and_in_place():
    M, D = 21, 100
    x, blk, wb, wa, gate, normal = inputs(M, D, torch.bfloat16)
    norm = b.HpNorm(wb, wa, gate)
    ref_h, ref_y = b.hp_norm_fwd(norm, x, blk)
    wide = torch.full((M, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    y_wide = wide.clone()
    h, y = b.hp_norm_fwd(norm, x, blk, h=wide[:, :D], y=y_wide[:, :D])
    assert torch.equal(h, ref_h) and torch.equal(y, ref_y)
    assert bool((wide[:, D:] == 7).all()) and bool((y_wide[:, D:] == 7).all())
    stream = plain.matrix(x)
    h2, y2 = b.hp_norm_fwd(norm, stream, blk, h=stream)
    assert h2.data_ptr() == stream.data_ptr() and torch.equal(stream, ref_h) and torch.equal(y2, ref_y)
    saved = b.hp_norm_saved(norm, M)
    b.hp_norm_fwd(norm, x, blk, saved)
    dy, dh = plain.matrix(normal(M, D)), plain.matrix(normal(M, D))
    ref = b.hp_norm_bwd(norm, saved, ref_h, dy, dh, blk)
    outs = [torch.full((M, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    into = b.HpNormGrads(outs[0][:, :D], outs[1][:, :D], *(torch.zeros(D, device="cuda") for _ in range(3)))
    got = b.hp_norm_bwd(norm, saved, ref_h, dy, dh, blk, into=into)
    assert all(torch.equal(a, c) for a, c in zip(ref, got)) and all(bool((o[:, D:] == 7).all()) for o in outs)
    own = b.HpNormGrads(dh, dy, *(torch.zeros(D, device="cuda") for _ in range(3)))
    got = b.hp_norm_bwd(norm, saved, ref_h, dy, dh, blk, into=own)
    assert all(torch.equal(a, c) for a, c in zip(ref, got))


@pytest.mark.parametrize("D", [648, 5000, 7000, 9001])
def test_gradients_in_place(D):
    """dx and dblock over dh and dy either way round, at the widths whose kernels hold a row, hold it in part, or read it again."""
    M = 40
    x, blk, wb, wa, gate, normal = inputs(M, D, torch.bfloat16)
    norm = b.HpNorm(wb, wa, gate)
    saved = b.hp_norm_saved(norm, M)
    h, _ = b.hp_norm_fwd(norm, x, blk, saved)
    dy, dh = normal(M, D), normal(M, D)
    ref = b.hp_norm_bwd(norm, saved, h, plain.matrix(dy), plain.matrix(dh), blk)
    for turned in (False, True):
        a, c = plain.matrix(dy), plain.matrix(dh)
        into = b.HpNormGrads(*((a, c) if turned else (c, a)), *(torch.empty(D, device="cuda") for _ in range(3)))
        got = b.hp_norm_bwd(norm, saved, h, a, c, blk, into=into)
        assert all(torch.equal(g, r) for g, r in zip(got, ref))


def test_accumulates_and_repeats_its_bits():
    M, D = 1500, 640
    x, blk, wb, wa, gate, normal = inputs(M, D, torch.bfloat16)
    norm = b.HpNorm(wb, wa, gate)
    saved = b.hp_norm_saved(norm, M)
    h, _ = b.hp_norm_fwd(norm, x, blk, saved)
    dy = plain.matrix(normal(M, D))
    one = b.hp_norm_bwd(norm, saved, h, dy, None, blk)
    again = b.hp_norm_bwd(norm, saved, h, dy, None, blk)
    assert all(torch.equal(a, c) for a, c in zip(one, again))
    two = b.hp_norm_bwd(norm, saved, h, dy, None, blk, into=again, accumulate=True)
    for name in ("dgate", "dw_before", "dw_after"):
        assert torch.equal(getattr(two, name), 2 * getattr(one, name)), name


def test_no_tokens():
    D = 64
    w = torch.ones(D, device="cuda")
    x = torch.empty(0, D, device="cuda")
    norm = b.HpNorm(w, w, w)
    saved = b.hp_norm_saved(norm, 0)
    h, y = b.hp_norm_fwd(norm, x, x, saved)
    assert h.shape == y.shape == (0, D)
    d = b.hp_norm_bwd(norm, saved, h, x, x, x)
    for s in (d.dgate, d.dw_before, d.dw_after):
        assert bool((s == 0).all())
        s.fill_(3.0)
    d = b.hp_norm_bwd(norm, saved, h, x, x, x, into=d, accumulate=True)
    assert all(bool((s == 3).all()) for s in (d.dgate, d.dw_before, d.dw_after))


def test_graph_and_streams():
    M, D = 700, 2048
    x, blk, wb, wa, gate, normal = inputs(M, D, torch.bfloat16, pad=0)
    norm = b.HpNorm(wb, wa, gate)
    dy = plain.matrix(normal(M, D))
    saved = b.hp_norm_saved(norm, M)
    ref_h, ref_y = b.hp_norm_fwd(norm, x, blk, saved)
    ref = b.hp_norm_bwd(norm, saved, ref_h, dy, None, blk)
    side, ws = torch.cuda.Stream(), b.Workspace()
    ws.get(b.workspace_bytes(b.FP4_OP_HP_NORM_BWD, M, D, 0, b.FP4_BF16))
    h, y, out = torch.empty_like(x), torch.empty_like(x), b.HpNormGrads(*(torch.empty_like(t) for t in ref))
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            b.hp_norm_fwd(norm, x, blk, saved, h=h, y=y)
            b.hp_norm_bwd(norm, saved, h, dy, None, blk, into=out, ws=ws)
    for _ in range(3):
        for t in (h, y, *out):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(h, ref_h) and torch.equal(y, ref_y) and all(torch.equal(a, c) for a, c in zip(out, ref))
        again = b.hp_norm_bwd(norm, saved, ref_h, dy, None, blk)
        assert all(torch.equal(a, c) for a, c in zip(again, ref))


def test_rows_past_2_to_32_bytes():
    D, M = 16384, 140_000
    x = torch.zeros(M, D, dtype=torch.bfloat16, device="cuda")
    x[-1] = torch.linspace(-2, 2, D, device="cuda").to(torch.bfloat16)
    x[0, 0] = 1.0
    w = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    norm = b.HpNorm(w)
    saved = b.hp_norm_saved(norm, M)
    h, y = b.hp_norm_fwd(norm, x, saved=saved)
    few = torch.stack([x[0], x[-1]])
    fs = b.hp_norm_saved(norm, 2)
    fh, fy = b.hp_norm_fwd(norm, few, saved=fs)
    assert torch.equal(y[0], fy[0]) and torch.equal(y[-1], fy[1]) and torch.equal(h[-1], x[-1])
    d = b.hp_norm_bwd(norm, saved, h, dy=x)
    fd = b.hp_norm_bwd(norm, fs, fh, dy=few)
    assert torch.equal(d.dx[-1], fd.dx[1]) and torch.equal(d.dx[0], fd.dx[0])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,D", [(1500, 1377), (600, 4104), (600, 5120), (600, 6144), (600, 6145), (600, 7001), (600, 8192), (300, 8193), (300, 9001), (520, 16384)])
@pytest.mark.parametrize("form", ["vector", "token"])
def test_more_rows_than_workgroups(M, D, dtype, form):
    """Each width's kernel of the backward pass, its workgroups going from row to row and summing over several."""
    x, blk, wb, wa, gate, normal = inputs(M, D, dtype, gate=form, seed=M + D)
    norm = b.HpNorm(wb, wa, gate, scale=0.7, eps=EPS)
    saved = b.hp_norm_saved(norm, M)
    h, y = b.hp_norm_fwd(norm, x, blk, saved)
    check_forward(norm, x, blk, h, y, saved)
    dy, dh = plain.matrix(normal(M, D) * 0.1, dtype, 1), plain.matrix(normal(M, D) * 0.1, dtype)
    got = b.hp_norm_bwd(norm, saved, h, dy, dh, blk)
    check_backward(norm, saved, h, dy, dh, blk, got, M)
    again = b.hp_norm_bwd(norm, saved, h, dy, dh, blk)
    assert all(torch.equal(a, c) for a, c in zip(got, again))
