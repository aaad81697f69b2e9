"""Trains a small network of microscaled FP4 layers and serves it token by token.

    python examples/mx_layer.py [--steps 300] [--tokens 1024] [--micro-batches 2]

Two linear layers with a SiLU between them learn a fixed random teacher of the same shape.  Every product of the layers runs on 4-bit operands
with one scale for 32 elements; the activations wait for the weight gradient in 8 bits.  Weights are quantized once a step and serve all its
micro-batches, whose weight gradients add up in place.  Afterwards the trained weights, quantized once, answer single tokens, one launch a layer.
Prints the loss as it falls, what the same training reaches in fp32, and how far single-token answers are from the batched ones.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2501_17116_amd import binding as b  # noqa: E402


class MxLinear(torch.nn.Module):
    """Y = A W with W [K, N] an fp32 master.  Its gradient comes by autograd, or with add_in_place is added to W.grad in the product's own
    launch, which saves a pass over it for every micro-batch; hooks on W and torch.autograd.grad then do not see it."""

    def __init__(self, K: int, N: int, generator: torch.Generator, add_in_place: bool = False):
        super().__init__()
        self.W = torch.nn.Parameter(torch.randn(K, N, generator=generator, device="cuda") / K ** 0.5)
        self.add_in_place = add_in_place
        self.prepare()

    def prepare(self):
        """Quantizes both orientations of the weights: after every optimizer step, before the next forward pass."""
        self.wq = b.mx_prepare_weights(self.W.detach())

    def forward(self, A: torch.Tensor) -> torch.Tensor:
        return _MxLinear.apply(A, self.W, self) if torch.is_grad_enabled() else b.mx_linear_fwd(A, self.wq.fwd)


class _MxLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, A, W, layer):
        ctx.layer, ctx.wq = layer, layer.wq            # the weights of this pass, whatever is prepared before its backward
        ctx.saved = b.mx_checkpoint(*A.shape) if ctx.needs_input_grad[1] else None   # 8 bits an activation instead of the activation
        return b.mx_linear_fwd(A, ctx.wq.fwd, saved=ctx.saved)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dY):
        need_a, need_w, _ = ctx.needs_input_grad
        dY, W = dY.contiguous(), ctx.layer.W
        into = W.grad if need_w and ctx.layer.add_in_place else None
        add = {"grad_bits": 8, "dW": into, "accumulate": into is not None}
        dA = dW = None
        if need_a and need_w:
            dA, dW = b.mx_linear_bwd(dY, ctx.saved, ctx.wq.bwd, **add)
        elif need_w:
            dW = b.mx_linear_bwd_wgrad(dY, ctx.saved, **add)
        elif need_a:
            dA = b.mx_linear_bwd_dgrad(dY, ctx.wq.bwd)
        if need_w and ctx.layer.add_in_place:
            W.grad, dW = dW, None
        return dA, dW, None


def _network(layers, A):
    return layers[1](torch.nn.functional.silu(layers[0](A)))


def train(layers, teacher, steps, tokens, micro_batches, width, seed, report=None):
    """Plain Adam on the layers' masters.  Returns the mean loss of the last tenth of the steps."""
    masters = [l.W for l in layers]
    opt = torch.optim.Adam(masters, lr=2e-3)
    g = torch.Generator(device="cuda").manual_seed(seed)
    last = []
    for step in range(steps):
        total = 0.0
        for _ in range(micro_batches):
            A = torch.randn(tokens // micro_batches, width, generator=g, device="cuda")
            want = torch.nn.functional.silu(A @ teacher[0]) @ teacher[1]
            loss = (_network(layers, A) - want).square().mean() / micro_batches
            loss.backward()
            total += float(loss.detach())
        opt.step()
        opt.zero_grad()
        for l in layers:
            l.prepare()
        if step >= steps - max(1, steps // 10):
            last.append(total)
        if report and (step % max(1, steps // 6) == 0 or step == steps - 1):
            report("step %4d  loss %.4f" % (step, total))
    return sum(last) / len(last)


class _PlainLinear(torch.nn.Module):
    def __init__(self, W):
        super().__init__()
        self.W = torch.nn.Parameter(W.clone())

    def prepare(self):
        pass

    def forward(self, A):
        return A @ self.W


def main(argv=None, report=print):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=300)
    p.add_argument("--tokens", type=int, default=1024)
    p.add_argument("--micro-batches", type=int, default=2)
    p.add_argument("--width", type=int, default=256)
    p.add_argument("--hidden", type=int, default=512)
    a = p.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(1)
    teacher = [torch.randn(a.width, a.hidden, generator=g, device="cuda") / a.width ** 0.5,
               torch.randn(a.hidden, a.width, generator=g, device="cuda") / a.hidden ** 0.5]
    layers = [MxLinear(a.width, a.hidden, g, add_in_place=True), MxLinear(a.hidden, a.width, g, add_in_place=True)]
    plain = [_PlainLinear(l.W.detach()) for l in layers]
    with torch.no_grad():
        A = torch.randn(a.tokens, a.width, generator=g, device="cuda")
        want = torch.nn.functional.silu(A @ teacher[0]) @ teacher[1]
        before = float((_network(layers, A) - want).square().mean())
    mx = train(layers, teacher, a.steps, a.tokens, a.micro_batches, a.width, 2, report)
    fp32 = train(plain, teacher, a.steps, a.tokens, a.micro_batches, a.width, 2)
    report("loss before %.4f, after %d steps %.4f (fp32 layers: %.4f)" % (before, a.steps, mx, fp32))

    with torch.no_grad():
        together = _network(layers, A[:64])
        alone = torch.cat([_network(layers, A[i:i + 1]) for i in range(64)])
        apart = float((alone - together).norm() / together.norm())
    report("64 tokens one by one against all at once: %.2e" % apart)
    return {"before": before, "mx": mx, "fp32": fp32, "apart": apart}


if __name__ == "__main__":
    main()
