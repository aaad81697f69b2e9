"""Plain forms of the high-precision operators in 64 bits, each with how far a result in fp32 arithmetic may lie from it.

Bounds count roundings.  fp32: 2^-24 of the result of each operation, so n of them in a row, or in a sum in whatever order, at most n 2^-24 of the sum
of magnitudes.  An output is rounded once more, by at most finfo(type).eps / 2 of itself.  Magnitudes (`size`) follow the formulas with
absolute values in place of differences."""
import torch

U = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def matrix(x, dtype=torch.bfloat16, pad=0, device="cuda"):
    """x with rows that begin at multiples of 16 bytes, `pad` times 8 elements further apart than they need, which hold NaN."""
    rows, cols = x.shape
    held = torch.full((rows, -(-cols // 8) * 8 + 8 * pad), float("nan"), dtype=dtype, device=device)
    held[:, :cols] = x.to(dtype).to(device)
    return held[:, :cols]


def close(got, want, tol, what=""):
    got = got.double()
    err = (got - want).abs()
    bad = ~(err <= tol)
    assert not bool(bad.any()), "%s: %d of %d off, worst error %g where %g is allowed, at %s" % (
        what, int(bad.sum()), bad.numel(), float(err[bad].max()), float(tol.expand_as(err)[bad][err[bad].argmax()]), bad.nonzero()[0].tolist())


# A row's sum: 16 terms a thread one after another, six exchanges, up to 16 waves: below 40 roundings; with the mean, the root and the quotient
# the inverse norm is off by at most 24 U of itself.
ROW = 48 * U


def joint(x, block, w_before, w_after, gate, scale, eps):
    """h, y, r_before, r_after and the sizes of h and y."""
    x = x.double()
    h, size = scale * x, (scale * x).abs()
    r_after = None
    if block is not None:
        u = block.double()
        if w_after is not None:
            r_after = (u.square().mean(1) + eps).rsqrt()
            u = u * r_after[:, None] * w_after.double()
        if gate is not None:
            u = u * gate.double()
        h, size = h + u, size + u.abs()
    r = (h.square().mean(1) + eps).rsqrt()
    y = size_y = None
    if w_before is not None:
        y, size_y = h * r[:, None] * w_before.double(), size * r[:, None] * w_before.double().abs()
    return h, y, r, r_after, size, size_y


def joint_gradients(h, dy, dh, block, w_before, w_after, gate, scale, r_before, r_after):
    """{name: (gradient, size)} of a joint by its formulas, from the inverse norms that are given."""
    out = {}
    t = size = torch.zeros_like(h, dtype=torch.float64)
    if dh is not None:
        t, size = dh.double(), dh.double().abs()
    if dy is not None:
        n, r, g = h.double() * r_before.double()[:, None], r_before.double()[:, None], dy.double() * w_before.double()
        t = t + r * (g - n * (g * n).mean(1, keepdim=True))
        size = size + r * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True))
        out["dw_before"] = (dy.double() * n).sum(0), (dy.double() * n).abs().sum(0)
    out["dx"] = scale * t, abs(scale) * size
    if block is None:
        return out
    m = block.double()
    if w_after is not None:
        m = m * r_after.double()[:, None]
    w = 1.0 if w_after is None else w_after.double()
    g = 1.0 if gate is None else gate.double()
    u = m * w
    if gate is not None:
        per_token = gate.dim() == 2
        out["dgate"] = (t * u, size * u.abs()) if per_token else ((t * u).sum(0), (size * u.abs()).sum(0))
    q, size_q = t * g * w, size * abs(g) * abs(w)
    if w_after is None:
        out["dblock"] = q, size_q
        return out
    out["dw_after"] = (t * g * m).sum(0), (size * abs(g) * m.abs()).sum(0)
    r = r_after.double()[:, None]
    out["dblock"] = r * (q - m * (q * m).mean(1, keepdim=True)), r * (size_q + m.abs() * (size_q * m.abs()).mean(1, keepdim=True))
    return out


def head(x, w, targets, dloss=None, piece=4096):
    """{name: (value, bound)} of the head; gradients with dloss.

    z: D products summed in fp32, at most D U of the sum of magnitudes.  A sum of exponentials: fewer than 256 roundings a term; an exponential by 2
    to a power: its argument is off by 2 U of the logits, itself by 4 U.  dz is kept in 11 bits (2^-11 of itself, 2^-40 at least), so is dloss x; both
    operands lie under a power of two that leaves at least 2^-39 of their largest; products are summed in fp32."""
    M, D, V = x.shape[0], x.shape[1], w.shape[0]
    xd = x.double()
    has = (targets >= 0) & (targets < V)
    rows = torch.arange(M, device=x.device)
    lse = torch.full((M,), -float("inf"), dtype=torch.float64, device=x.device)
    most, off_z = torch.zeros_like(lse), torch.zeros_like(lse)
    for v in range(0, V, piece):
        wp = w[v:v + piece].double().t().contiguous()
        z = xd @ wp
        lse = torch.logaddexp(lse, torch.logsumexp(z, 1))
        most = torch.maximum(most, z.abs().amax(1))
        off_z = torch.maximum(off_z, (D + 1) * U * (xd.abs() @ wp.abs()).amax(1))
    bound = off_z + 260 * U + (most + lse.abs()) * 4 * U
    zt = torch.zeros_like(lse)
    zt[has] = (xd[has] * w[targets[has]].double()).sum(1)
    loss = torch.where(has, lse - zt, torch.zeros_like(lse))
    out = {"lse": (lse, bound), "loss": (loss, torch.where(has, bound + off_z + 2 * U * (zt.abs() + loss.abs()), torch.zeros_like(bound)))}
    if dloss is None:
        return out
    c = torch.where(has, dloss.double(), torch.zeros_like(lse))
    cx, off_p = c[:, None] * xd, (off_z + bound + (most + lse.abs()) * 4 * U + 8 * U)[:, None]
    largest_x = cx.abs().max() if M else 0.0
    largest_w = float(w.double().abs().max())
    dx, dx_tol, dw, dw_tol = torch.zeros_like(xd), torch.zeros_like(xd), [], []
    for v in range(0, V, piece):
        wp = w[v:v + piece].double()
        p = torch.exp(xd @ wp.t().contiguous() - lse[:, None])
        d = p.clone()
        here = has & (targets >= v) & (targets < v + wp.shape[0])
        d[rows[here], targets[here] - v] -= 1.0
        p, d = p * has[:, None], d * has[:, None]
        off = p * off_p + d.abs() * 2.0 ** -11 + 2.0 ** -40 * has[:, None]
        dx += (d @ wp) * c[:, None]
        dx_tol += c.abs()[:, None] * (off @ wp.abs() + (d.abs() @ torch.ones_like(wp)) * largest_w * 2.0 ** -39 + (V + 80) * U * (d.abs() @ wp.abs()))
        dt = d.t().contiguous()
        dw.append(dt @ cx)
        dw_tol.append(off.t().contiguous() @ cx.abs() + (2.0 ** -11 * 1.001 + (M + 4) * U) * (dt.abs() @ cx.abs())
                      + dt.abs().sum(1, keepdim=True) * largest_x * 2.0 ** -39)
    # what an error of both operands at once adds is below a thousandth of the terms
    out["dx"] = dx, dx_tol * 1.001
    out["dw"] = torch.cat(dw), torch.cat(dw_tol) * 1.001
    return out
