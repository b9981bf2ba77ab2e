#!/usr/bin/env python3
"""Trains a small stack of feed-forward sublayers on one GPU, the whole step with this library's calls:

    python examples/train_feed_forward.py [--steps 200] [--tokens 1024] [--width 512] [--hidden 2048] [--layers 2]

A layer is  a = norm(z), u = a W1^T, v = relu(u) W2^T, z' = z + dropout(v)  with W1 and W2 kept in fp32; the norm behind a layer takes
the dropout and the residual with it.  Products run in microscaled 4-bit floating point: activations and weights are rounded to nearest, the
gradients that go backwards stochastically.  The weights' gradients, times the step size, are written by the products straight
into the flat gradient buffer; conef_step compresses them with error feedback, and conef_apply_update takes the compressed step.  The task is to
imitate a random network of the same kind.

torch holds the memory and does what is no operator of the library: the relu, the loss, and plain gradient descent on the norms' gamma and beta.
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

EPS = 1e-5


class Linear:
    """A weight in the flat parameter buffer, as the products take it: quantised by rows for the layer's output, by columns for its
    input's gradient."""

    def __init__(self, B, weight, grad, tokens, device):
        self.B, self.weight, self.grad, self.tokens = B, weight, grad, tokens
        self.outputs, self.inputs = weight.shape
        self.w, self.w_t = B.mx_alloc(self.outputs, self.inputs, device), B.mx_alloc(self.inputs, self.outputs, device)
        self.x, self.x_t = B.mx_alloc(tokens, self.inputs, device), B.mx_alloc(self.inputs, tokens, device)
        self.dy, self.dy_t = B.mx_alloc(tokens, self.outputs, device), B.mx_alloc(self.outputs, tokens, device)

    def room(self):
        t, i, o = self.tokens, self.inputs, self.outputs
        return max(self.B.conef_mx_product_workspace(*s) for s in ((t, o, i), (t, i, o), (o, i, t)))

    def forward(self, x, y, ws, st):
        B = self.B
        B.conef_mx_quantise(self.weight, B.MX_NEAREST, 0, 0, 0, self.w, self.w_t, st)
        B.conef_mx_quantise(x, B.MX_NEAREST, 0, 0, 0, self.x, self.x_t, st)
        B.conef_mx_product(self.x, self.w, self.inputs, 1.0, 0.0, y, ws, st)

    def backward(self, dy, dx, rate, seed, site, step, ws, st):
        """dx, and rate times the weight's gradient into its place of the flat gradient buffer"""
        B = self.B
        B.conef_mx_quantise(dy, B.MX_STOCHASTIC, seed, site, step, self.dy, self.dy_t, st)
        if dx is not None:
            B.conef_mx_product(self.dy, self.w_t, self.outputs, 1.0, 0.0, dx, ws, st)
        B.conef_mx_product(self.dy_t, self.x_t, self.tokens, rate, 0.0, self.grad, ws, st)


def train(steps=200, tokens=1024, width=512, hidden=2048, layers=2, rate=0.5, p=0.1, rank=4, seed=1, device="cuda:0", report=None):
    """Losses of the steps; `report(step, loss)` is called every tenth of them."""
    import torch

    from paper_2312_08538_amd import binding as B

    g = torch.Generator(device=device).manual_seed(seed)
    layout = [(hidden, width), (width, hidden)] * layers
    model = B.Model(layout, rank, 4, 128, B.F32, seed)
    buf = model.alloc(device)
    buf["Q"].normal_(generator=g)
    params = torch.zeros_like(buf["grads"])

    def view(flat, l):
        n, m = layout[l]
        o = model.offsets[l]["grad_off"]
        return flat[o:o + n * m].view(n, m)

    def new(*shape, dtype=torch.bfloat16):
        return torch.zeros(*shape, dtype=dtype, device=device)

    teacher = torch.zeros_like(params)
    for l, (n, m) in enumerate(layout):
        view(params, l).normal_(std=m ** -0.5, generator=g)
        view(teacher, l).normal_(std=m ** -0.5, generator=g)
    linear = [Linear(B, view(params, l), view(buf["grads"], l), tokens, device) for l in range(2 * layers)]
    copied = [Linear(B, view(teacher, l), None, tokens, device) for l in range(2 * layers)]
    gamma, beta = torch.ones(layers + 1, width, device=device), torch.zeros(layers + 1, width, device=device)
    dgamma, dbeta = torch.zeros_like(gamma), torch.zeros_like(beta)
    ws = new(max(max(x.room() for x in linear), B.conef_norm_workspace(tokens, width)), dtype=torch.uint8)
    z, a = [new(tokens, width) for _ in range(layers + 1)], [new(tokens, width) for _ in range(layers + 1)]
    u, f, v = ([new(tokens, n) for _ in range(layers)] for n in (hidden, hidden, width))
    mean, rstd = new(layers + 1, tokens, dtype=torch.float32), new(layers + 1, tokens, dtype=torch.float32)
    dz, dv, da, du = new(tokens, width), new(tokens, width), new(tokens, width), new(tokens, hidden)
    st = B.Model.stream_handle()

    def drop(layer, step):
        return B.conef_drop(p=p, site=layer, seed=seed, step=step)

    def forward(weights, step):
        """the stack's output, a[layers]; the teacher drops nothing (step None) and has its own gamma and beta of 1 and 0"""
        own = step is not None
        one, zero = (gamma, beta) if own else (torch.ones_like(gamma), torch.zeros_like(beta))
        B.conef_norm_forward(None, EPS, z[0], None, one[0], zero[0], None, a[0], mean[0], rstd[0], st)
        for l in range(layers):
            weights[2 * l].forward(a[l], u[l], ws, st)
            f[l].copy_(torch.relu(u[l]))
            weights[2 * l + 1].forward(f[l], v[l], ws, st)
            d = drop(l, step) if own else None
            B.conef_norm_forward(d, EPS, v[l], z[l], one[l + 1], zero[l + 1], z[l + 1], a[l + 1], mean[l + 1], rstd[l + 1], st)
        return a[layers]

    losses = []
    for step in range(steps):
        z[0].normal_(generator=g)
        target = forward(copied, None).float()
        diff = forward(linear, step).float() - target
        losses.append((diff * diff).mean())
        dy, dz_in = (diff * (2.0 / diff.numel())).bfloat16(), None
        for l in range(layers - 1, -1, -1):
            # through the norm behind the layer, its residual and its dropout
            B.conef_norm_backward(drop(l, step), dy, z[l + 1], gamma[l + 1], mean[l + 1], rstd[l + 1], dz_in, dz, dv, dgamma[l + 1],
                                  dbeta[l + 1], ws, st)
            linear[2 * l + 1].backward(dv, du, rate, seed, 2 * l + 1, step, ws, st)
            du.mul_(u[l] > 0)
            linear[2 * l].backward(du, da, rate, seed, 2 * l, step, ws, st)
            dy, dz_in = da, dz
        B.conef_norm_backward(None, da, z[0], gamma[0], mean[0], rstd[0], None, None, None, dgamma[0], dbeta[0], ws, st)
        # the weights' step: compressed with error feedback, and taken
        model.step(buf, step)
        B.conef_apply_update(model.ctx, buf["P"], buf["Q"], params, st)
        gamma.sub_(dgamma, alpha=rate)
        beta.sub_(dbeta, alpha=rate)
        if report and step % max(1, steps // 10) == 0:
            report(step, float(losses[-1]))
    torch.cuda.synchronize()
    model.close()
    return [float(x) for x in losses]


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, default in (("steps", 200), ("tokens", 1024), ("width", 512), ("hidden", 2048), ("layers", 2)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--rate", type=float, default=0.5)
    a = ap.parse_args()
    losses = train(a.steps, a.tokens, a.width, a.hidden, a.layers, a.rate, report=lambda s, x: print(f"step {s:5d}  loss {x:.5f}", flush=True))
    print(f"first {losses[0]:.5f}  last {sum(losses[-10:]) / len(losses[-10:]):.5f} (mean of ten)")


if __name__ == "__main__":
    main()
