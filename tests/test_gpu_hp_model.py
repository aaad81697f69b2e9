"""The operators together, as a model's training step uses them: lookup, a joint, an MX layer as the block, the joint that closes it, the head with
its loss, and all the way back into one gradient of the table that embedding and head share.  Each step against its plain form on what it was given, and the
captured step against the eager one, bit for bit."""
import threading

import pytest
import torch

from paper_2501_17116_amd import binding as b
from tests import hp_plain as plain
from tests.test_gpu_hp_embed import gradient

pytestmark = pytest.mark.gpu


class Model:
    def __init__(self, M, D, V, seed=0):
        g = torch.Generator().manual_seed(seed)
        normal = lambda *s: torch.randn(*s, generator=g)
        self.M, self.D, self.V = M, D, V
        self.ids = (torch.rand(M, generator=g) ** 4 * V).long().cuda()
        self.targets = torch.randint(0, V, (M,), generator=g).cuda()
        self.targets[::7] = -100
        self.table = (normal(V, D) * 0.05).bfloat16().cuda()
        self.layer = b.mx_prepare_weights((normal(D, D) / D ** 0.5).bfloat16().cuda())
        weights = lambda: (1 + 0.1 * normal(D)).bfloat16().cuda()
        self.first = b.HpNorm(weights())                                               # before the block
        self.last = b.HpNorm(weights(), w_after=weights(), gate=(0.3 * weights()).contiguous(), scale=0.9)   # after it, and before the head
        self.dloss = torch.full((M,), 1.0 / M, device="cuda")

    def step(self, ws=None):
        M, D, V = self.M, self.D, self.V
        o = {}
        o["x"] = b.hp_embed_fwd(self.ids, self.table, scale=D ** 0.5)
        o["s0"], o["s1"] = b.hp_norm_saved(self.first, M), b.hp_norm_saved(self.last, M)
        _, o["a"] = b.hp_norm_fwd(self.first, o["x"], saved=o["s0"])
        o["saved"] = b.mx_checkpoint(M, D)
        o["block"] = b.mx_linear_fwd(o["a"], self.layer.fwd, saved=o["saved"], ws=ws)
        o["h"], o["y"] = b.hp_norm_fwd(self.last, o["x"], o["block"], o["s1"])
        o["loss"], o["lse"] = b.hp_head_fwd(o["y"], self.table, self.targets, ws=ws)
        o["dy"], o["dtable"] = b.hp_head_bwd(o["y"], self.table, self.targets, o["lse"], self.dloss, ws=ws)
        o["of_head"] = o["dtable"].clone()
        o["d1"] = b.hp_norm_bwd(self.last, o["s1"], o["h"], o["dy"], None, o["block"], ws=ws)
        o["da"], o["dW"] = b.mx_linear_bwd(o["d1"].dblock, o["saved"], self.layer.bwd, ws=ws)
        o["d0"] = b.hp_norm_bwd(self.first, o["s0"], o["x"], o["da"], o["d1"].dx, ws=ws)
        b.hp_embed_bwd(o["d0"].dx, self.ids, V, scale=D ** 0.5, dtable=o["dtable"], accumulate=True, ws=ws)
        return o

    def tensors(self, o):
        return [o[k] for k in ("x", "a", "block", "h", "y", "loss", "lse", "dy", "dtable", "da", "dW")] + [t for d in (o["d0"], o["d1"]) for t in d if t is not None]

    def room(self):
        ws = b.Workspace()
        ws.get(max(b.workspace_bytes(op, self.M, self.D, self.V, b.FP4_BF16) for op in range(9, 17)))
        return ws


@pytest.mark.parametrize("M,D,V", [(1, 256, 300), (77, 264, 1000), (600, 512, 3000)])
def test_each_step_of_a_step(M, D, V):
    m = Model(M, D, V)
    o = m.step()
    t = plain.half_step(torch.bfloat16)
    assert torch.equal(o["x"], (m.table[m.ids].float() * D ** 0.5).bfloat16())
    _, ry, *_, size = plain.joint(o["x"], None, m.first.w_before, None, None, 1.0, m.first.eps)
    plain.close(o["a"], ry, t * ry.abs() + 2 * plain.ROW * size, "a")
    rh, ry, _, _, size_h, size = plain.joint(o["x"], o["block"], m.last.w_before, m.last.w_after, m.last.gate, 0.9, m.last.eps)
    plain.close(o["h"], rh, t * rh.abs() + plain.ROW * size_h, "h")
    plain.close(o["y"], ry, t * ry.abs() + 2 * plain.ROW * size, "y")
    want = plain.head(o["y"], m.table, m.targets, m.dloss)
    plain.close(o["loss"], *want["loss"], "loss")
    plain.close(o["dy"], want["dx"][0], want["dx"][1] + t * (want["dx"][0].abs() + want["dx"][1]), "dy")
    plain.close(o["of_head"], *want["dw"], "head's part of the table's gradient")
    for joint, saved, h, dy, dh, block, d in ((m.last, o["s1"], o["h"], o["dy"], None, o["block"], o["d1"]), (m.first, o["s0"], o["x"], o["da"], o["d1"].dx, None, o["d0"])):
        for name, (value, size) in plain.joint_gradients(h, dy, dh, block, joint.w_before, joint.w_after, joint.gate, joint.scale, saved.r_before, saved.r_after).items():
            tol = t * value.abs() + 3 * plain.ROW * size if value.dim() == 2 else (M * plain.U + 3 * plain.ROW) * size
            plain.close(getattr(d, name), value, tol, name)
    sums, tol = gradient(o["d0"].dx, m.ids, V, D ** 0.5)
    total = o["of_head"].double() + sums
    plain.close(o["dtable"], total, tol + 2 * plain.U * (o["of_head"].double().abs() + sums.abs()), "table's gradient")


def test_captured_step():
    m = Model(300, 512, 2000)
    want = [t.clone() for t in m.tensors(m.step())]
    ws, side = m.room(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            o = m.step(ws)
    for _ in range(3):
        for t in m.tensors(o):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(m.tensors(o), want))
        assert all(torch.equal(a, c) for a, c in zip(m.tensors(m.step()), want))


def test_two_streams_and_two_threads_at_once():
    """Each with the workspace that the binding takes for it."""
    models = [Model(300, 512, 2000, seed) for seed in range(2)]
    want = [[t.clone() for t in m.tensors(m.step())] for m in models]
    streams = [torch.cuda.Stream() for _ in models]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for m, s in zip(models, streams):
            with torch.cuda.stream(s):
                got.append(m.tensors(m.step()))
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for g, w in zip(got, want) for a, c in zip(g, w))
    results = [None, None]

    def work(i):      # both on the default stream
        results[i] = [m.tensors(m.step()) for m in [models[i]] * 3][-1]

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for g, w in zip(results, want) for a, c in zip(g, w))
