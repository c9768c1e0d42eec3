"""Data-parallel training steps in four bits, from the products that make the gradient to the weights.

A two-layer network learns a random teacher on N simulated nodes.  Per step and node the linear layers' three products
run on microscaled 4-bit operands (gradients rounded stochastically); the nodes' gradients are aggregated -- in 4-bit
blocks while samples for the basis are collected, in GradiVeQ's compressed domain afterwards; the aggregate moves the weights
through momentum and orthogonalisation.

    python examples/train_four_bit.py [steps]
"""
import math
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parent.parent))

D_IN, D_HID, D_OUT, BATCH, NODES = 256, 512, 128, 384, 4
COLLECT = 6            # iterations whose aggregates the basis is fitted on


class Linear4:
    """y = x W^T with all three products in 4 bits.  W: a [out, in] view of a flat weight buffer."""

    def __init__(self, ctx, w):
        self.ctx, self.w = ctx, w

    def quantize(self):
        """Once per step: the weights along their rows (forward) and along their columns (for dx)."""
        self.w4, self.w4_t = self.ctx.mx4_quantize_both(self.w)

    def forward(self, x):
        self.x4, self.x4_t = self.ctx.mx4_quantize_both(x)      # along the rows for y, along the columns for dW
        y = torch.empty((x.shape[0], self.w.shape[0]), device="cuda", dtype=torch.bfloat16)
        return self.ctx.mx4_matmul(self.x4, self.w4, y), self.x4_t

    def backward(self, dy, x4_t, dw, seed, node, need_dx=True):
        """dW into `dw` (float32 [out, in]); returns dx."""
        dy4, dy4_t = self.ctx.mx4_quantize_both(dy, stochastic=True, seed=seed, node=node)
        self.ctx.mx4_matmul(dy4_t, x4_t, dw)
        if not need_dx:
            return None
        dx = torch.empty((dy.shape[0], self.w.shape[1]), device="cuda", dtype=torch.bfloat16)
        return self.ctx.mx4_matmul(dy4, self.w4_t, dx)


def train(steps=40, seed=0, lr=0.02, verbose=False):
    from paper_1811_03617_b200 import gvq

    gen = torch.Generator(device="cuda").manual_seed(seed)
    shapes = [(D_HID, D_IN), (D_OUT, D_HID)]
    lens = [m * n for m, n in shapes]
    layout = gvq.HostLayout(256, 32, [0, lens[0]], lens)
    ctx = gvq.Context(layout)
    plan = gvq.OrthoPlan(ctx, [m for m, _ in shapes], [n for _, n in shapes])
    M = ctx.M

    def randn(*s):
        return torch.randn(s, generator=gen, device="cuda")
    teacher = randn(D_OUT, D_IN) / math.sqrt(D_IN)
    weights = torch.cat([randn(m * n) / math.sqrt(n) for m, n in shapes])
    momentum = torch.zeros(M, device="cuda")
    layers = [Linear4(ctx, weights[o:o + m * n].view(m, n)) for o, (m, n) in zip((0, lens[0]), shapes)]
    grads = [torch.zeros(M, device="cuda") for _ in range(NODES)]
    views = [[g[o:o + m * n].view(m, n) for o, (m, n) in zip((0, lens[0]), shapes)] for g in grads]
    history = torch.zeros((COLLECT, M), device="cuda")
    g_hat = torch.zeros(M, device="cuda")
    s_sum = torch.empty((ctx.S, ctx.k), device="cuda")
    Ut = torch.empty((2, 32, 256), device="cuda")
    mu, ev = torch.empty((2, 256), device="cuda"), torch.empty((2, 256), device="cuda")

    losses = []
    for it in range(steps):
        for layer in layers:
            layer.quantize()
        total = torch.zeros((), device="cuda")
        for n in range(NODES):
            x = randn(BATCH, D_IN)
            target = (x @ teacher.T).to(torch.bfloat16)
            a, x_t = layers[0].forward(x)
            h = a.clamp_min(0)
            y, h_t = layers[1].forward(h)
            diff = (y - target).float()
            total += diff.square().mean()
            dy = (diff * (2.0 / (BATCH * NODES))).to(torch.bfloat16)
            dh = layers[1].backward(dy, h_t, views[n][1], seed=it, node=2 * n)
            layers[0].backward(dh * (a > 0), x_t, views[n][0], seed=it, node=2 * n + 1, need_dx=False)
        if it < COLLECT:
            ctx.mx4_quantize_aggregate(grads, g_hat, stochastic=True, seed=1000 + it)
            history[it].copy_(g_hat)
            if it == COLLECT - 1:
                ctx.fit_basis(history, NODES, NODES, Ut, mu, ev)
        else:
            ctx.compress_aggregate(grads, Ut, mu, s_sum)
            ctx.decompress(s_sum, Ut, mu, grads, NODES, g_hat)
        plan.step(g_hat, momentum, weights, lr=lr, beta=0.9)
        losses.append(total / NODES)
    ctx.device_status()
    losses = [float(v) for v in losses]
    if verbose:
        for i in range(0, steps, max(1, steps // 10)):
            print(f"step {i:4d}  loss {losses[i]:.4f}{'  (4-bit exchange)' if i < COLLECT else ''}")
        print(f"step {steps - 1:4d}  loss {losses[-1]:.4f}")
    return losses


if __name__ == "__main__":
    train(int(sys.argv[1]) if len(sys.argv) > 1 else 40, verbose=True)
