"""The head's loss and gradients against the formulas in 64 bits, within the roundings that its form takes, and against differences."""
import pytest
import torch

from paper_2501_17116_amd import binding as b
from tests import hp_plain as plain

pytestmark = pytest.mark.gpu


def inputs(M, D, V, seed=0, ignored=0.1, pad=1, lean=6.0, spread=0.02):
    g = torch.Generator().manual_seed(seed)
    w = torch.randn(V, D, generator=g) * spread
    targets = torch.randint(0, V, (M,), generator=g)
    x = torch.randn(M, D, generator=g) + torch.rand(M, 1, generator=g) * lean * w[targets] / (spread * spread * D)
    out = torch.rand(M, generator=g) < ignored
    targets[out] = torch.where(torch.rand(int(out.sum()), generator=g) < 0.5, -100, V)
    dloss = (torch.rand(M, generator=g) + 0.5) / max(1, M)
    return plain.matrix(x, pad=pad), plain.matrix(w, pad=2 * pad), targets.cuda(), dloss.cuda()


def check(x, w, targets, dloss, dw_dtype=torch.float32):
    want = plain.head(x, w, targets, dloss)
    loss, lse = b.hp_head_fwd(x, w, targets)
    plain.close(lse, *want["lse"], "lse")
    plain.close(loss, *want["loss"], "loss")
    dx, dw = b.hp_head_bwd(x, w, targets, lse, dloss, dw_dtype=dw_dtype)
    for name, got in (("dx", dx), ("dw", dw)):
        value, tol = want[name]
        plain.close(got, value, tol + plain.half_step(got.dtype) * (value.abs() + tol), name)
    return loss, lse, dx, dw


@pytest.mark.parametrize("M,D,V", [(1, 8, 1), (1, 8, 2), (1, 64, 1000), (2, 72, 77), (24, 256, 3001), (32, 200, 129), (33, 512, 640), (64, 136, 1025), (65, 128, 500),
                                   (100, 1376, 999), (129, 64, 128), (300, 192, 1500), (511, 648, 2049), (1055, 328, 4099)])
def test_small(M, D, V):
    check(*inputs(M, D, V))


@pytest.mark.parametrize("M,D,V", [(700, 512, 12000), (1300, 320, 9000)])
def test_large_tiles(M, D, V):
    check(*inputs(M, D, V), dw_dtype=torch.bfloat16)


def test_several_pieces_of_the_vocabulary():
    check(*inputs(140, 16384, 17001, pad=0), dw_dtype=torch.bfloat16)


def test_several_pieces_of_short_rows():
    M, D, V = 260, 16, 900_000
    check(*inputs(M, D, V, pad=0, lean=0.5), dw_dtype=torch.bfloat16)


@pytest.mark.parametrize("M", [32768, 33001])
def test_many_tokens(M):
    """More than the forward pass takes at a time."""
    check(*inputs(M, 32, 300, pad=0), dw_dtype=torch.bfloat16)


@pytest.mark.parametrize("M", [1, 31, 32, 33, 63, 64, 65, 96, 127, 128, 129])
@pytest.mark.parametrize("D,V", [(8, 900), (264, 333), (520, 4100)])
def test_few_tokens(M, D, V):
    """The gradient of x around the sizes where another kernel takes over, widths that end inside its 256 columns."""
    check(*inputs(M, D, V, seed=M))


def test_sharp_and_flat_rows():
    x, w, targets, dloss = inputs(200, 256, 700, spread=0.5, lean=40.0)
    x[:50] *= 4.0
    x[50:60] = 0.0
    loss, lse, dx, dw = check(x, w, targets, dloss)
    assert float((lse[50:60] - torch.log(torch.tensor(700.0))).abs().max()) <= 1e-5


def test_far_logits():
    """Sums of exponentials that only their maximum keeps in range."""
    M, D, V = 64, 64, 300
    x, w, targets, dloss = inputs(M, D, V, spread=1.0, lean=0.0, ignored=0.0)
    x *= 100.0
    loss, lse, _, _ = check(x, w, targets, dloss)
    assert float(lse.max()) > 1000.0 and bool(torch.isfinite(loss).all())
    w *= -1.0
    w -= 100.0
    x.abs_()
    loss, lse, _, _ = check(x, w, targets, dloss)
    assert float(lse.max()) < -1000.0 and bool(torch.isfinite(loss).all())


def test_no_targets_at_all():
    M, D, V = 70, 128, 300
    x, w, targets, dloss = inputs(M, D, V)
    targets.fill_(-1)
    dloss[3] = float("nan")
    loss, lse = b.hp_head_fwd(x, w, targets)
    dx, dw = b.hp_head_bwd(x, w, targets, lse, dloss)
    assert bool((loss == 0).all()) and bool((dx == 0).all()) and bool((dw == 0).all())
    plain.close(lse, *plain.head(x, w, targets)["lse"])


def test_tokens_without_a_target_count_nowhere():
    M, D, V = 90, 128, 300
    x, w, targets, dloss = inputs(M, D, V, ignored=0.0)
    targets[::3] = -100
    dloss[::3] = 1e30
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    keep[::3] = False
    loss, lse, dx, dw = check(x, w, targets, torch.where(keep, dloss, torch.zeros_like(dloss)))
    dx2, dw2 = b.hp_head_bwd(x, w, targets, lse, dloss)
    assert torch.equal(dx2, dx) and torch.equal(dw2, dw) and bool((dx[::3] == 0).all())


def test_gradients_of_every_size():
    """Tiny and huge weights of losses, and of the head's: powers of two change nothing but the exponents."""
    M, D, V = 50, 96, 333
    x, w, targets, dloss = inputs(M, D, V)
    loss, lse = b.hp_head_fwd(x, w, targets)
    dx, dw = b.hp_head_bwd(x, w, targets, lse, dloss)
    for e in (-60, 40):
        f = 2.0 ** e
        dx2, dw2 = b.hp_head_bwd(x, w, targets, lse, dloss * f)
        assert torch.equal(dw2, dw * f) and torch.equal(dx2, (dx.float() * f).bfloat16())


def test_against_differences():
    M, D, V = 5, 24, 37
    x, w, targets, dloss = inputs(M, D, V, ignored=0.0, spread=0.3)
    loss, lse = b.hp_head_fwd(x, w, targets)
    dx, dw = b.hp_head_bwd(x, w, targets, lse, dloss)
    g = torch.Generator().manual_seed(5)
    sx, sw = torch.randn(M, D, generator=g, dtype=torch.float64).cuda(), torch.randn(V, D, generator=g, dtype=torch.float64).cuda()

    def value(e):
        z = (x.double() + e * sx) @ (w.double() + e * sw).t()
        return float((dloss.double() * (torch.logsumexp(z, 1) - z.gather(1, targets[:, None])[:, 0])).sum())

    e = 1e-5
    want = (value(e) - value(-e)) / (2 * e)
    got = float((dx.double() * sx).sum() + (dw.double() * sw).sum())
    # dx is rounded to 2^-8 of itself, operands to 2^-11; the differences' own error is far below
    allowed = float((dx.double() * sx).abs().sum() * 2.0 ** -8 + ((dx.double() * sx).abs().sum() + (dw.double() * sw).abs().sum()) * 2.0 ** -9)
    assert abs(got - want) <= allowed, (got, want, allowed)


def test_accumulates_frozen_sides_padding_and_repeats():
    M, D, V = 150, 264, 700
    x, w, targets, dloss = inputs(M, D, V)
    loss, lse = b.hp_head_fwd(x, w, targets)
    dx, dw = b.hp_head_bwd(x, w, targets, lse, dloss)
    dx2, none = b.hp_head_bwd(x, w, targets, lse, dloss, want_dw=False)
    none2, dw2 = b.hp_head_bwd(x, w, targets, lse, dloss, want_dx=False)
    assert none is None and none2 is None and torch.equal(dx, dx2) and torch.equal(dw, dw2)
    wide = torch.full((V, D + 16), 1.5, device="cuda")
    b.hp_head_bwd(x, w, targets, lse, dloss, dw=wide[:, :D], accumulate=True)
    plain.close(wide[:, :D], dw.double() + 1.5, plain.U * 4 * (dw.double().abs() + 1.5))
    assert bool((wide[:, D:] == 1.5).all())
    narrow = torch.full((M, D + 8), 3.0, dtype=torch.bfloat16, device="cuda")
    b.hp_head_bwd(x, w, targets, lse, dloss, dx=narrow[:, :D], want_dw=False)
    assert torch.equal(narrow[:, :D], dx) and bool((narrow[:, D:] == 3).all())
    assert torch.equal(b.hp_head_bwd(x, w, targets, lse, dloss, dw_dtype=torch.bfloat16)[1], dw.bfloat16())


def test_no_tokens():
    x, w = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(5, 64, dtype=torch.bfloat16, device="cuda")
    t, e = torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda")
    loss, lse = b.hp_head_fwd(x, w, t)
    assert loss.shape == lse.shape == (0,)
    dx, dw = b.hp_head_bwd(x, w, t, lse, e)
    assert dx.shape == (0, 64) and bool((dw == 0).all())
    dw.fill_(2.0)
    b.hp_head_bwd(x, w, t, lse, e, dw=dw, accumulate=True)
    assert bool((dw == 2).all())
    assert b.hp_head_bwd(x, w, t, lse, e, want_dw=False)[0].shape == (0, 64)


def test_no_channels():
    """All logits 0."""
    x, w = torch.empty(5, 0, dtype=torch.bfloat16, device="cuda"), torch.empty(700, 0, dtype=torch.bfloat16, device="cuda")
    t = torch.tensor([0, 699, -1, 700, 3], device="cuda")
    loss, lse = b.hp_head_fwd(x, w, t)
    plain.close(lse, torch.full((5,), 700.0, dtype=torch.float64, device="cuda").log(), torch.full((5,), 260 * plain.U, device="cuda"))
    assert loss[2] == loss[3] == 0 and torch.equal(loss[[0, 1, 4]], lse[[0, 1, 4]])
    dx, dw = b.hp_head_bwd(x, w, t, lse, torch.ones(5, device="cuda"))
    assert dx.shape == (5, 0) and dw.shape == (700, 0)


def test_weights_past_2_to_32_bytes():
    """A vocabulary whose weights, and their gradient, end beyond: tokens that aim at its ends, the rest of it empty."""
    M, D, V = 3, 8192, 270_000
    w = torch.zeros(V, D, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator().manual_seed(3)
    for v in (0, V - 2, V - 1):
        w[v] = (torch.randn(D, generator=g) * 0.05).bfloat16().cuda()
    x = torch.randn(M, D, generator=g).bfloat16().cuda()
    t = torch.tensor([0, V - 1, V - 2], device="cuda")
    dloss = torch.ones(M, device="cuda")
    loss, lse = b.hp_head_fwd(x, w, t)
    dx, dw = b.hp_head_bwd(x, w, t, lse, dloss, dw_dtype=torch.bfloat16)
    # the rows in use, and all the others as one whose logit is 0
    some = torch.cat([w[[0, V - 2, V - 1]].double(), torch.zeros(1, D, dtype=torch.float64, device="cuda")])
    z = x.double() @ some.t().contiguous()
    z[:, 3] = torch.log(torch.tensor(V - 3.0, dtype=torch.float64))
    want = torch.logsumexp(z, 1)
    off = (D + 1) * plain.U * (x.double().abs() @ some.abs().t().contiguous()).amax(1) + 260 * plain.U + (z.abs().amax(1) + want.abs()) * 4 * plain.U
    plain.close(lse, want, off, "lse")
    p = torch.exp(z - want[:, None])
    p[[0, 1, 2], [0, 2, 1]] -= 1.0
    rows = dw[[0, V - 2, V - 1]].double()
    ref = p[:, :3].t().contiguous() @ x.double()
    # dz and x to 11 bits each, the output to 8; the exponentials by the logits' error
    tol = (2.0 ** -8 + 2.0 ** -10) * (p[:, :3].abs().t().contiguous() @ x.double().abs()) + (torch.exp(z - want[:, None])[:, :3] * 3 * off[:, None]).t().contiguous() @ x.double().abs()
    plain.close(rows, ref, tol, "dw")
    few = dw[1000:1003].double()
    same = ((1.0 / torch.exp(want)) @ x.double()).expand(3, D)
    plain.close(few, same, (2.0 ** -8 + 2.0 ** -10 + 4 * float(off.max())) * ((1.0 / torch.exp(want)) @ x.double().abs()).expand(3, D) + 2.0 ** -40 * x.double().abs().sum(0), "empty rows' dw")


def test_graphs_with_workspaces_of_their_own():
    M, D, V = 300, 256, 2000
    x, w, targets, dloss = inputs(M, D, V, pad=0)
    ref_loss, ref_lse = b.hp_head_fwd(x, w, targets)
    ref_dx, ref_dw = b.hp_head_bwd(x, w, targets, ref_lse, dloss)
    runs = []
    for _ in range(2):
        ws = b.Workspace()
        ws.get(max(b.workspace_bytes(op, M, D, V, b.FP4_BF16) for op in (b.FP4_OP_HP_HEAD_FWD, b.FP4_OP_HP_HEAD_BWD)))
        out = [torch.empty_like(t) for t in (ref_loss, ref_lse, ref_dx, ref_dw)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            b.hp_head_fwd(x, w, targets, loss=out[0], lse=out[1], ws=ws)
            b.hp_head_bwd(x, w, targets, out[1], dloss, dx=out[2], dw=out[3], ws=ws)
        runs.append((graph, out, ws))
    streams = [torch.cuda.Stream() for _ in runs]
    for _ in range(3):
        for _, out, _ in runs:
            for t in out:
                t.fill_(float("nan"))
        torch.cuda.synchronize()
        for s, (graph, _, _) in zip(streams, runs):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for _, out, _ in runs:
            assert all(torch.equal(a, c) for a, c in zip(out, (ref_loss, ref_lse, ref_dx, ref_dw)))
        assert torch.equal(b.hp_head_bwd(x, w, targets, ref_lse, dloss)[1], ref_dw)


NOT_FINITE = [(3, 64, 200), (24, 256, 3001), (64, 136, 1025), (300, 192, 1500), (700, 512, 12000)]   # every tile, both joins


@pytest.mark.parametrize("M,D,V", NOT_FINITE)
def test_logits_that_are_not_finite_are_seen(M, D, V):
    """In whichever column: the loss of their tokens is not finite, all others keep their bits."""
    x, w, targets, _ = inputs(M, D, V, ignored=0.0)
    x[:, 0] = 0.0
    targets[:] = targets.clamp(max=V - 2)       # the columns below are never a target's but once
    loss, lse = b.hp_head_fwd(x, w, targets)
    for v in (0, V // 2, V - 1):
        bad = w.clone()
        bad[v, 1] = float("nan")
        l2, e2 = b.hp_head_fwd(x, bad, targets)
        assert bool(torch.isnan(e2).all()) and bool(torch.isnan(l2).all()), ("a row of w", v)
        for t in (0, M - 1):
            others = torch.arange(M, device="cuda") != t
            huge, up = w.clone(), x.clone()
            huge[v, 0], up[t, 0] = 3e38, 3e38    # their product alone leaves fp32
            l2, e2 = b.hp_head_fwd(up, huge, targets)
            assert not bool(torch.isfinite(e2[t])) and not bool(torch.isfinite(l2[t])), ("a logit of inf", v, t)
            assert torch.equal(e2[others], lse[others]) and torch.equal(l2[others], loss[others])
    for t in (0, M // 2, M - 1):
        others = torch.arange(M, device="cuda") != t
        bad = x.clone()
        bad[t] = float("nan")
        l2, e2 = b.hp_head_fwd(bad, w, targets)
        assert bool(torch.isnan(e2[t])) and bool(torch.isnan(l2[t])), ("a row of x", t)
        assert torch.equal(e2[others], lse[others]) and torch.equal(l2[others], loss[others])


@pytest.mark.parametrize("M,D,V", NOT_FINITE)
def test_logits_of_minus_infinity_count_nothing(M, D, V):
    x, w, targets, _ = inputs(M, D, V, ignored=0.0)
    x[:, 0] = 0.0
    targets[:] = targets.clamp(min=V // 3 + 1)
    t = M // 2
    x[t, 0] = 3e38
    few, far = w.clone(), w.clone()
    few[:, 0], far[:, 0] = 0.0, 0.0
    few[:V // 3 + 1, 0], far[:V // 3 + 1, 0] = -3e38, -1e-33     # -inf, and some -3e5, for whole tiles and a part of one
    assert all(torch.equal(a, c) for a, c in zip(b.hp_head_fwd(x, few, targets), b.hp_head_fwd(x, far, targets)))
    few[:, 0] = -3e38
    loss, lse = b.hp_head_fwd(x, few, targets)
    others = torch.arange(M, device="cuda") != t
    assert float(lse[t]) == -float("inf") and bool(torch.isfinite(lse[others]).all()) and bool(torch.isfinite(loss[others]).all())


@pytest.mark.parametrize("M,D,V", [(2, 64, 200), (90, 128, 300), (300, 192, 1500), (700, 512, 12000)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf"), 3e38])
def test_what_tokens_without_a_target_hold_counts_nowhere(M, D, V, value):
    x, w, targets, dloss = inputs(M, D, V, ignored=0.0)
    targets[::3] = -100
    targets[1::9] = V
    out = (targets < 0) | (targets >= V)
    clean, bad, c = x.clone(), x.clone(), dloss.clone()
    clean[out] = 0.0
    bad[out] = value
    c[out] = value
    loss, lse = b.hp_head_fwd(clean, w, targets)
    l2, e2 = b.hp_head_fwd(bad, w, targets)
    assert torch.equal(l2, loss) and torch.equal(e2[~out], lse[~out])
    dx, dw = b.hp_head_bwd(clean, w, targets, lse, dloss)
    dx2, dw2 = b.hp_head_bwd(bad, w, targets, e2, c)
    assert bool(torch.isfinite(dw).all()) and torch.equal(dx2, dx) and torch.equal(dw2, dw)


@pytest.mark.parametrize("M,D,V", [(32, 64, 300), (512, 64, 300), (64, 128, 5000), (700, 512, 12000)])
@pytest.mark.parametrize("shift", [0.0, -90.0, 700.0])
def test_losses_are_not_negative(M, D, V, shift):
    """Near-certain tokens, whose target's logit leads by 15 to 60 and may lie far from 0: the largest logit's own term is exactly 1."""
    g = torch.Generator().manual_seed(M + V)
    w = torch.randn(V, D, generator=g) * 0.05
    w[:, 0] = 1.0
    targets = torch.randint(0, V, (M,), generator=g)
    wt = w[targets].clone()
    wt[:, 0] = 0.0
    x = wt * ((15.0 + 45.0 * torch.rand(M, 1, generator=g)) / wt.square().sum(1, keepdim=True))
    x[:, 0] = shift
    x, w, targets = plain.matrix(x), plain.matrix(w), targets.cuda()
    want = plain.head(x, w, targets)
    loss, lse = b.hp_head_fwd(x, w, targets)
    plain.close(lse, *want["lse"], "lse")
    plain.close(loss, *want["loss"], "loss")
    assert bool((loss >= 0).all()), float(loss.min())


@pytest.mark.parametrize("M,D,V", [(300, 1032, 12100), (1000, 2048, 8200)])
def test_fp32_gradients_of_the_weights_in_large_tiles(M, D, V):
    """More than 188 tiles of 256 x 256: alone, added to what is there, and rounded to bf16."""
    x, w, targets, dloss = inputs(M, D, V)
    loss, lse, dx, dw = check(x, w, targets, dloss)
    wide = torch.full((V, D + 16), 1.5, device="cuda")
    b.hp_head_bwd(x, w, targets, lse, dloss, dw=wide[:, :D], accumulate=True)
    assert torch.equal(wide[:, :D], dw + 1.5) and bool((wide[:, D:] == 1.5).all())
    wide.fill_(-2.0)
    b.hp_head_bwd(x, w, targets, lse, dloss, dw=wide[:, :D])
    assert torch.equal(wide[:, :D], dw) and bool((wide[:, D:] == -2).all())
    assert torch.equal(b.hp_head_bwd(x, w, targets, lse, dloss, dw_dtype=torch.bfloat16)[1], dw.bfloat16())
