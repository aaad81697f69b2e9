"""What the high-precision operators around the linear layers are timed on: the joints of a transformer's blocks and its two ends.

A case says by "op" what runs:
  norm        x [M x D] and a block's output -> the next residual stream h = scale x + gate * (block normed, times w_after) and h normed, times w_before
  norm-grad   gradients of both, h, the block's output and the saved inverse norms -> gradients of x, the block, the gate and both weights
  embed       token ids [M] and a table [V x D] -> rows times a scale
  embed-grad  token ids and the rows' gradients -> the table's gradient [V x D] in fp32
  loss        x [M x D], the head's weights [V x D], targets -> softmax cross entropy of each token, and the logarithm of its sum of exponentials
  loss-grad   the same with that logarithm and each loss's gradient at hand -> gradients of x and of the weights
  loss-step   forward and backward pass of the head

Norms are root mean square, 1 / sqrt(mean(x^2) + eps).  A gate is absent, one vector for all tokens, or a row for each.  A target outside
[0, V) has no loss and no gradient; an id outside it gives zeros and no gradient.

Shapes are those of the benchmark's layers (hidden sizes 2048, 4096 and 5120), of the tests, and generic ones.  Activations are N(0, 1) with a
few channels scaled up; table and head N(0, 0.02^2); ids and targets fall off as 1 / rank, as words do; inputs of the head lean towards
their target's weights by different amounts, so that some tokens are near certain and others are not.
"""
import math

import torch

own = False

EPS = 1e-5


def _case(name, op, M, D, V=0, dtype="bf16", block=True, after=False, gate="none", scale=1.0, ids="rank"):
    """block, after, gate, scale: what a norm's joint has; ids: "rank" or "even"."""
    return {"name": name, "op": op, "M": M, "D": D, "V": V, "dtype": dtype, "block": block, "after": after, "gate": gate, "scale": scale, "ids": ids}


def listed():
    return [
        # one decoded token between two blocks of a 7B model: latency
        _case("norm-1x4096", "norm", 1, 4096),
        # a training batch of the 7B model, blocks normed on both sides, gated by a learned vector
        _case("norm-16384x4096-gated", "norm", 16384, 4096, after=True, gate="vector"),
        # the backward pass of the same joint, 13B width, residual stream scaled down
        _case("norm-grad-8192x5120-gated", "norm-grad", 8192, 5120, after=True, gate="vector", scale=0.7),
        # odd everything in fp32, a gate for each token
        _case("norm-grad-1055x1377-f32", "norm-grad", 1055, 1377, dtype="f32", after=True, gate="token"),
        # a batch of decoding sequences looks its tokens up
        _case("embed-24x4096", "embed", 24, 4096, 32000),
        # the table's gradient of a 7B training batch, frequent tokens among them
        _case("embed-grad-16384x4096", "embed-grad", 16384, 4096, 32000, scale=0.5),
        # fp32, a larger table whose rows end inside a piece, tokens spread evenly
        _case("embed-grad-3001x2055-f32", "embed-grad", 3001, 2055, 50003, dtype="f32", ids="even"),
        # scoring the next token of a batch of decoding sequences
        _case("loss-24x4096x32000", "loss", 24, 4096, 32000),
        # evaluation of a 1.3B model over a batch
        _case("loss-8192x2048x32000", "loss", 8192, 2048, 32000),
        # odd everything, the gradients alone
        _case("loss-grad-1055x1376x50003", "loss-grad", 1055, 1376, 50003),
        # the head's part of a training step, 13B width, a micro-batch
        _case("loss-step-2048x5120x32000", "loss-step", 2048, 5120, 32000),
        # the largest: a training batch over a large vocabulary
        _case("loss-step-8192x4096x131072", "loss-step", 8192, 4096, 131072),
    ]


_PRODUCTS = {"loss": 1, "loss-grad": 3, "loss-step": 4}


def _cost(c):
    if c["op"] in _PRODUCTS:
        return 2.0 * c["M"] * c["D"] * c["V"] * _PRODUCTS[c["op"]]
    return 300.0 * c["D"] * (c["M"] * 4 + (c["V"] if c["op"] == "embed-grad" else 0))


def draw(rng):
    """One more case of the same ranges, sizes over their logarithm; the head's widths are multiples of 8."""
    def size(lo, hi, unit=1):
        return max(lo, min(hi, unit * round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / unit)))

    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["norm", "norm-grad", "embed", "embed-grad", "loss", "loss", "loss-grad", "loss-step"])
        head = op in _PRODUCTS
        norm = op.startswith("norm")
        few = rng.random() < 0.3
        block = rng.random() < 0.8
        c = {
            "op": op,
            "M": size(1, 64) if few else size(64, 8192 if head else 16384),
            "D": size(256, 8192, 8 if head or rng.random() < 0.6 else 1),
            "V": 0 if norm else size(1000, 131072),
            "dtype": "f32" if not head and rng.random() < 0.25 else "bf16",
            "block": block or not norm,
            "after": norm and block and rng.random() < 0.5,
            "gate": rng.choice(["none", "vector", "token"]) if norm and block else "none",
            "scale": rng.choice([1.0, 1.0, 0.7]) if not head else 1.0,
            "ids": rng.choice(["rank", "rank", "even"]),
        }
        if _cost(c) <= most:
            return c


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def prepare(case, seed):
    M, D, V, op = case["M"], case["D"], case["V"], case["op"]
    dt = _dtype(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * int(seed) + 31)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)

    def matrix(x):
        """As a program holds it: rows that begin at multiples of 16 bytes."""
        rows, cols = x.shape
        held = torch.zeros(rows, -(-cols // 8) * 8, device="cuda", dtype=dt)[:, :cols]
        return held.copy_(x)

    def activations():
        x = normal(M, D)
        x[:, torch.randperm(D, generator=g, device="cuda")[:max(1, D // 1000)]] *= 20.0
        return x

    def words():
        u = torch.rand(M, generator=g, device="cuda", dtype=torch.float64)
        if case["ids"] == "even":
            return (u * V).long().clamp(max=V - 1)
        rank = torch.exp(u * math.log(V)).long().clamp(1, V) - 1       # density 1 / rank
        return (rank * 7919) % V if V % 7919 else rank                 # frequent ones anywhere in the table

    s = {"case": case}
    if op.startswith("norm"):
        s["block"] = matrix(activations() * 0.5) if case["block"] else None
        s["w_before"] = (1.0 + 0.1 * normal(D)).to(dt)
        s["w_after"] = (1.0 + 0.1 * normal(D)).to(dt) if case["after"] else None
        s["gate"] = (None if case["gate"] == "none" else (0.5 + 0.1 * normal(D)).to(dt) if case["gate"] == "vector"
                     else matrix(torch.sigmoid(normal(M, D))))
        s["x"] = matrix(activations())
        if op == "norm-grad":
            s["h"] = s.pop("x")
            s["dy"], s["dh"] = matrix(normal(M, D) * 0.01), matrix(normal(M, D) * 0.01)
            # what the forward pass left: the inverse norms of each token
            s["r_before"] = torch.rsqrt(s["h"].double().square().mean(1) + EPS).float()
            s["r_after"] = torch.rsqrt(s["block"].double().square().mean(1) + EPS).float() if case["after"] else None
        return s
    s["ids"] = words()
    if op == "embed":
        s["table"] = matrix(normal(V, D) * 0.02)
        return s
    if op == "embed-grad":
        s["dy"] = matrix(normal(M, D) * 0.01)
        return s
    w = normal(V, D) * 0.02
    lean = torch.rand(M, 1, generator=g, device="cuda") * (600.0 / (0.02 * D))    # up to 12 more than the others' logits
    s["x"] = matrix(normal(M, D) + lean * w[s["ids"]])
    s["w"] = matrix(w)
    skip = torch.rand(M, generator=g, device="cuda") < 0.03                       # prompts and padding are not trained on
    skip[0] = False
    s["ids"] = torch.where(skip, torch.full_like(s["ids"], -100), s["ids"])
    s["dloss"] = torch.full((M,), 1.0 / float((~skip).sum()), device="cuda")
    if op == "loss-grad":
        s["lse"] = torch.cat([torch.logsumexp(p.float() @ s["w"].float().t(), 1) for p in s["x"].split(1024)])
    return s


# ---- the plain form ----------------------------------------------------------------------------------------------------------

def _plain_norm(s):
    case, dt = s["case"], _dtype(s["case"])
    h = s["x"].float() * case["scale"]
    if s["block"] is not None:
        u = s["block"].float()
        if s["w_after"] is not None:
            u = u / torch.sqrt((u * u).mean(1, keepdim=True) + EPS) * s["w_after"].float()
        if s["gate"] is not None:
            u = u * s["gate"].float()
        h = h + u
    y = h / torch.sqrt((h * h).mean(1, keepdim=True) + EPS) * s["w_before"].float()
    return {"h": h.to(dt), "y": y.to(dt)}


def _plain_norm_grad(s):
    case, dt = s["case"], _dtype(s["case"])
    h, dy = s["h"].float(), s["dy"].float()
    r = s["r_before"].unsqueeze(1)
    n = h * r
    g = dy * s["w_before"].float()
    t = s["dh"].float() + r * (g - n * (g * n).mean(1, keepdim=True))
    out = {"dx": (t * case["scale"]).to(dt), "dw_before": (dy * n).sum(0)}
    if s["block"] is None:
        return out
    u = v = s["block"].float()
    if s["w_after"] is not None:
        v = u * s["r_after"].unsqueeze(1)
        u = v * s["w_after"].float()
    if s["gate"] is not None:
        out["dgate"] = (t * u).sum(0) if case["gate"] == "vector" else (t * u).to(dt)
        t = t * s["gate"].float()
    if s["w_after"] is not None:
        out["dw_after"] = (t * v).sum(0)
        t = t * s["w_after"].float()
        t = s["r_after"].unsqueeze(1) * (t - v * (t * v).mean(1, keepdim=True))
    out["dblock"] = t.to(dt)
    return out


def _plain_loss(s):
    ids = s["ids"]
    z = s["x"].float() @ s["w"].float().t()
    top = z.amax(1)
    lse = torch.log(torch.exp(z - top.unsqueeze(1)).sum(1)) + top
    has = (ids >= 0) & (ids < s["case"]["V"])
    of = torch.where(has, ids, torch.zeros_like(ids)).unsqueeze(1)
    return torch.where(has, lse - z.gather(1, of).squeeze(1), torch.zeros_like(lse)), lse, z, has, of


def _plain_loss_grad(s, lse, z, has, of):
    z = torch.exp(z - lse.unsqueeze(1))
    z.scatter_add_(1, of, torch.full_like(z[:, :1], -1.0))
    z *= torch.where(has, s["dloss"], torch.zeros_like(lse)).unsqueeze(1)
    return {"dx": (z @ s["w"].float()).to(s["x"].dtype), "dw": (z.t() @ s["x"].float()).to(s["w"].dtype)}


def _run_plain(s):
    case = s["case"]
    op, dt = case["op"], _dtype(case)
    if op == "norm":
        return _plain_norm(s)
    if op == "norm-grad":
        return _plain_norm_grad(s)
    if op == "embed":
        return {"y": (s["table"].index_select(0, s["ids"]).float() * case["scale"]).to(dt)}
    if op == "embed-grad":
        dE = torch.zeros(case["V"], case["D"], device="cuda")
        return {"dE": dE.index_add_(0, s["ids"], s["dy"].float() * case["scale"])}
    loss, lse, z, has, of = _plain_loss(s)
    if op == "loss":
        return {"loss": loss, "lse": lse}
    if op == "loss-grad":
        return _plain_loss_grad(s, s["lse"], z, has, of)
    return {"loss": loss, **_plain_loss_grad(s, lse, z, has, of)}


# ---- the framework's -----------------------------------------------------------------------------------------------------------

def _run_own(s):
    from paper_2501_17116_amd import binding as b

    case = s["case"]
    op = case["op"]
    if op.startswith("norm"):
        norm = b.HpNorm(s["w_before"], w_after=s["w_after"], gate=s["gate"], scale=case["scale"], eps=EPS)
        if op == "norm":
            h, y = b.hp_norm_fwd(norm, s["x"], block=s["block"])
            return {"h": h, "y": y}
        d = b.hp_norm_bwd(norm, b.HpNormSaved(s["r_before"], s["r_after"]), s["h"], dy=s["dy"], dh=s["dh"], block=s["block"])
        return {k: v for k, v in (("dx", d.dx), ("dblock", d.dblock), ("dgate", d.dgate), ("dw_after", d.dw_after), ("dw_before", d.dw_before))
                if v is not None}
    if op == "embed":
        return {"y": b.hp_embed_fwd(s["ids"], s["table"], scale=case["scale"])}
    if op == "embed-grad":
        return {"dE": b.hp_embed_bwd(s["dy"], s["ids"], case["V"], scale=case["scale"])}
    if op == "loss":
        loss, lse = b.hp_head_fwd(s["x"], s["w"], s["ids"])
        return {"loss": loss, "lse": lse}
    if op == "loss-grad":
        dx, dw = b.hp_head_bwd(s["x"], s["w"], s["ids"], s["lse"], s["dloss"], dw_dtype=torch.bfloat16)
        return {"dx": dx, "dw": dw}
    loss, lse = b.hp_head_fwd(s["x"], s["w"], s["ids"])
    dx, dw = b.hp_head_bwd(s["x"], s["w"], s["ids"], lse, s["dloss"], dw_dtype=torch.bfloat16)
    return {"loss": loss, "dx": dx, "dw": dw}


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    """Inputs once, outputs once.  The backward pass of the head forms the logits again, since they are not kept."""
    op, M, D, V = case["op"], float(case["M"]), float(case["D"]), float(case["V"])
    e = 2.0 if case["dtype"] == "bf16" else 4.0
    if op == "norm":
        matrices = 3.0 + case["block"] + (case["gate"] == "token")
        return {"bytes": e * M * D * matrices, "flops": 8.0 * M * D}
    if op == "norm-grad":
        matrices = 4.0 + 2.0 * case["block"] + 2.0 * (case["gate"] == "token")
        return {"bytes": e * M * D * matrices + 8.0 * M, "flops": 20.0 * M * D}
    if op == "embed":
        return {"bytes": 2.0 * e * M * D + 8.0 * M, "flops": M * D}
    if op == "embed-grad":
        return {"bytes": e * M * D + 8.0 * M + 4.0 * V * D, "flops": 2.0 * M * D}
    per_token = 8.0 + 4.0 + 4.0
    if op == "loss":
        return {"bytes": e * (M + V) * D + per_token * M, "flops": 2.0 * M * D * V}
    if op == "loss-grad":
        return {"bytes": 2.0 * e * (M + V) * D + per_token * M, "flops": 6.0 * M * D * V}
    return {"bytes": 2.0 * e * (M + V) * D + per_token * M, "flops": 8.0 * M * D * V}


# ---- once more from the definition, in 64 bits: gradients by automatic differentiation of the forward formulas, the vocabulary in pieces --------

def _joint(x, block, w_before, w_after, gate, scale):
    def unit(a):
        return a * (a.pow(2).sum(1, keepdim=True) / a.shape[1] + EPS).pow(-0.5)

    h = scale * x
    if block is not None:
        u = block if w_after is None else unit(block) * w_after
        h = h + (u if gate is None else gate * u)
    return h, unit(h) * w_before


def _exact_norm(s):
    case = s["case"]

    def wide(name):
        return None if s.get(name) is None else s[name].double()

    if case["op"] == "norm":
        h, y = _joint(wide("x"), wide("block"), wide("w_before"), wide("w_after"), wide("gate"), case["scale"])
        return {"h": h, "y": y}
    # h is at hand as it is: the gradient that reaches it first, then that of what it was made of
    at, w = wide("h").requires_grad_(), wide("w_before").requires_grad_()
    with torch.enable_grad():
        _, y = _joint(at, None, w, None, None, 1.0)
        dh, dw = torch.autograd.grad(y, (at, w), wide("dy"))
    dh = dh + wide("dh")
    out = {"dx": dh * case["scale"], "dw_before": dw}
    if s["block"] is None:
        return out
    names = [n for n in ("block", "gate", "w_after") if s[n] is not None]
    leaves = {n: wide(n).requires_grad_() for n in names}
    with torch.enable_grad():
        h, _ = _joint(torch.zeros_like(dh), leaves["block"], w.detach(), leaves.get("w_after"), leaves.get("gate"), 0.0)
        for n, d in zip(names, torch.autograd.grad(h, [leaves[n] for n in names], dh)):
            out["d" + n] = d
    return out


def _exact_loss(s):
    case, ids, x = s["case"], s["ids"], s["x"].double()
    V, has = case["V"], (s["ids"] >= 0) & (s["ids"] < case["V"])
    piece = 8192
    lse = torch.full((x.shape[0],), -math.inf, dtype=torch.float64, device=x.device)
    for v in range(0, V, piece):
        lse = torch.logaddexp(lse, torch.logsumexp(x @ s["w"][v:v + piece].double().t().contiguous(), 1))
    loss = torch.zeros_like(lse)
    loss[has] = lse[has] - (x[has] * s["w"][ids[has]].double()).sum(1)
    if case["op"] == "loss":
        return {"loss": loss, "lse": lse}
    weight = s["dloss"].double() * has
    rows = torch.arange(x.shape[0], device=x.device)
    dx, dw = torch.zeros_like(x), []
    for v in range(0, V, piece):
        w = s["w"][v:v + piece].double()
        p = torch.softmax(torch.cat([x @ w.t().contiguous(), lse.unsqueeze(1)], 1), 1)[:, :-1]    # e^z / (e^lse + this piece's): undone below
        p = p / (1.0 - p.sum(1, keepdim=True))
        inside = has & (ids >= v) & (ids < v + w.shape[0])
        p[rows[inside], ids[inside] - v] -= 1.0
        p *= weight.unsqueeze(1)
        dx += p @ w
        dw.append(p.t().contiguous() @ x)
    out = {"dx": dx, "dw": torch.cat(dw)}
    return out if case["op"] == "loss-grad" else {"loss": loss, **out}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op.startswith("norm"):
        return _exact_norm(s)
    if op == "embed":
        return {"y": s["table"].double()[s["ids"]] * case["scale"]}
    if op == "embed-grad":
        order = torch.argsort(s["ids"], stable=True)
        rows = torch.cumsum(s["dy"].double()[order] * case["scale"], 0)        # sums of runs of one id, as differences
        ids = s["ids"][order]
        last = torch.cat([ids[1:] != ids[:-1], torch.ones(1, dtype=torch.bool, device=ids.device)]).nonzero().squeeze(1)
        dE = torch.zeros(case["V"], case["D"], dtype=torch.float64, device=ids.device)
        dE[ids[last]] = torch.diff(rows[last], dim=0, prepend=torch.zeros_like(rows[:1]))
        return {"dE": dE}
    return _exact_loss(s)
