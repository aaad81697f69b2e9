"""Embedding lookup and the table's gradient against plain forms: the lookup bit for bit, the sums within their roundings."""
import pytest
import torch

from paper_2501_17116_amd import binding as b
from tests import hp_plain as plain

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


def gradient(dy, ids, V, scale):
    """The sums and their bounds: n terms, the scale and the last rounding."""
    n = torch.zeros(V + 1, dtype=torch.float64, device="cuda")
    to = torch.where((ids >= 0) & (ids < V), ids, torch.full_like(ids, V))
    n.index_add_(0, to, torch.ones_like(to, dtype=torch.float64))
    s = torch.zeros(V + 1, dy.shape[1], dtype=torch.float64, device="cuda").index_add_(0, to, dy.double() * scale)
    a = torch.zeros_like(s).index_add_(0, to, (dy.double() * scale).abs())
    return s[:V], ((n[:, None] + 2) * plain.U * a)[:V]


def some(M, V, kind, seed=0):
    g = torch.Generator().manual_seed(seed)
    if kind == "same":
        ids = torch.full((M,), V // 2)
    elif kind == "even":
        ids = torch.randint(0, V, (M,), generator=g)
    elif kind == "padded":
        ids = torch.randint(-2, V + 2, (M,), generator=g)
        ids[M // 3:M // 2] = -1
        ids[-1:] = 1 << 40
    elif kind == "outside":
        ids = torch.full((M,), -7)
    else:   # a few frequent ones
        ids = (torch.rand(M, generator=g) ** 6 * V).long().clamp(max=V - 1)
    return ids.cuda(), g


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,D,V", [(1, 1, 1), (1, 4096, 32000), (24, 4096, 300), (7, 513, 5), (130, 2055, 1000)])
@pytest.mark.parametrize("kind", ["even", "padded"])
def test_lookup(M, D, V, dtype, kind):
    ids, g = some(M, V, kind)
    table = plain.matrix(torch.randn(V, D, generator=g), dtype, 1)
    wide = torch.full((M, -(-D // 8) * 8 + 16), 7.0, dtype=dtype, device="cuda")
    y = b.hp_embed_fwd(ids, table, scale=1.7, y=wide[:, :D])
    inside = (ids >= 0) & (ids < V)
    want = (table.float()[ids.clamp(0, V - 1)] * 1.7 * inside[:, None]).to(dtype)
    assert torch.equal(y, want) and bool((wide[:, D:] == 7).all())
    assert torch.equal(b.hp_embed_fwd(ids, table)[inside], table[ids[inside]])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,D,V", [(1, 8, 1), (1, 40, 70000), (9, 7, 3), (100, 513, 300), (2500, 264, 50), (5000, 72, 255), (5000, 72, 256), (20000, 40, 66000),
                                   (4099, 2056, 17)])
@pytest.mark.parametrize("kind", ["even", "few", "same", "padded", "outside"])
def test_gradient(M, D, V, dtype, kind):
    ids, g = some(M, V, kind)
    dy = plain.matrix(torch.randn(M, D, generator=g), dtype, 1)
    want, tol = gradient(dy, ids, V, 0.3)
    wide = torch.full((V, -(-D // 8) * 8 + 8), 7.0, device="cuda")
    got = b.hp_embed_bwd(dy, ids, V, scale=0.3, dtable=wide[:, :D])
    plain.close(got, want, tol)
    assert bool((wide[:, D:] == 7).all())
    first = got.clone()
    assert torch.equal(b.hp_embed_bwd(dy, ids, V, scale=0.3), first)
    added = torch.full((V, -(-D // 8) * 8), 2.0, device="cuda")[:, :D]
    got = b.hp_embed_bwd(dy, ids, V, scale=0.3, dtable=added, accumulate=True)
    plain.close(got, want + 2.0, tol + 2 * plain.U * (want.abs() + 2.0))
    absent = torch.ones(V, dtype=torch.bool, device="cuda")
    absent[ids[(ids >= 0) & (ids < V)]] = False
    assert bool((added[absent] == 2.0).all())


def test_every_place_of_a_run():
    """Runs that begin and end at every place around the borders of spans of eight."""
    D, V = 16, 40
    for first in range(0, 18):
        for length in (1, 7, 8, 9, 16, 17, 30):
            ids = torch.cat([torch.zeros(first), torch.full((length,), 5), torch.full((11,), 9)]).long().cuda()
            dy = torch.arange(ids.numel() * D, dtype=torch.float32, device="cuda").reshape(-1, D)
            want = torch.zeros(V, D, device="cuda").index_add_(0, ids, dy)      # whole numbers below 2^24: exact in any order
            assert torch.equal(b.hp_embed_bwd(dy, ids, V), want), (first, length)


def test_no_tokens_and_no_channels():
    ids = torch.empty(0, dtype=torch.int64, device="cuda")
    dt = b.hp_embed_bwd(torch.empty(0, 16, device="cuda"), ids, 5)
    assert bool((dt == 0).all())
    dt.fill_(4.0)
    b.hp_embed_bwd(torch.empty(0, 16, device="cuda"), ids, 5, dtable=dt, accumulate=True)
    assert bool((dt == 4).all())
    assert b.hp_embed_fwd(ids, torch.ones(5, 16, device="cuda")).shape == (0, 16)


def test_graph():
    M, D, V = 3000, 256, 400
    ids, g = some(M, V, "few")
    dy = plain.matrix(torch.randn(M, D, generator=g))
    ref = b.hp_embed_bwd(dy, ids, V)
    out, ws = torch.empty_like(ref), b.Workspace()
    ws.get(b.workspace_bytes(b.FP4_OP_HP_EMBED_BWD, M, D, V, b.FP4_BF16))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.hp_embed_bwd(dy, ids, V, dtable=out, ws=ws)
    for _ in range(3):
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref)
        assert torch.equal(b.hp_embed_bwd(dy, ids, V), ref)


def test_tables_past_2_to_32_bytes():
    D, V = 8192, 270_000
    ids = torch.tensor([V - 1, 0, V - 1, V - 2], device="cuda")
    table = torch.empty(V, D, dtype=torch.bfloat16, device="cuda")
    for i in (0, V - 2, V - 1):
        table[i] = (torch.arange(D, device="cuda") % 251 + i % 7).to(torch.bfloat16)
    assert torch.equal(b.hp_embed_fwd(ids, table), table[ids])
    dy = torch.ones(4, D, dtype=torch.bfloat16, device="cuda")
    dt = b.hp_embed_bwd(dy, ids, V)
    assert [float(dt[i].min()) for i in (0, V - 2, V - 1)] == [1.0, 1.0, 2.0] == [float(dt[i].max()) for i in (0, V - 2, V - 1)]
    assert float(dt[1:V - 2].abs().max()) == 0.0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,D,V", [(8193, 24, 300), (32768, 16, 70000), (32769, 16, 70000), (33001, 23, 300), (70001, 8, 256)])
@pytest.mark.parametrize("kind", ["even", "few", "padded"])
def test_gradient_of_many_tokens(M, D, V, dtype, kind):
    """Passes of small workgroups beside the clearing, and of large ones behind it or without it."""
    ids, g = some(M, V, kind)
    dy = plain.matrix(torch.randn(M, D, generator=g), dtype, 1)
    want, tol = gradient(dy, ids, V, 0.3)
    wide = torch.full((V, -(-D // 8) * 8 + 8), 7.0, device="cuda")
    got = b.hp_embed_bwd(dy, ids, V, scale=0.3, dtable=wide[:, :D])
    plain.close(got, want, tol)
    assert bool((wide[:, D:] == 7).all()) and torch.equal(b.hp_embed_bwd(dy, ids, V, scale=0.3), got)
    wide.fill_(2.0)
    got = b.hp_embed_bwd(dy, ids, V, scale=0.3, dtable=wide[:, :D], accumulate=True)
    plain.close(got, want + 2.0, tol + 2 * plain.U * (want.abs() + 2.0))
    assert bool((wide[:, D:] == 2).all())
