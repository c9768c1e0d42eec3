"""A gated feed-forward block in training and answering.

Training: the block's two products and their activation in 16 bits (one kernel; the projections are kept), its last projection and that
one's gradients in 8-bit integers (gradients rounded stochastically), the block's own gradients, written into a flat gradient, and the
orthogonalised update of all three matrices.  Answering: the trained matrices kept in 8 bits, a few tokens at a time.

    python examples/train_gated_block.py [steps]
"""
import math
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parent.parent))

D, F, BATCH = 256, 640, 384
SHAPES = [(F, D), (F, D), (D, F)]              # gate, up, down: [out][in], one after the other in the flat weights


class GatedBlock:
    def __init__(self, seed=0):
        from paper_1811_03617_b200 import gvq
        self.gvq = gvq
        lens = [m * n for m, n in SHAPES]
        offs = [sum(lens[:i]) for i in range(3)]
        self.ctx = gvq.Context(gvq.HostLayout(64, 4, offs, lens))
        self.plan = gvq.OrthoPlan(self.ctx, [m for m, _ in SHAPES], [n for _, n in SHAPES])
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.weights = torch.cat([torch.randn(m * n, generator=gen, device="cuda") / math.sqrt(n) for m, n in SHAPES]).bfloat16()
        self.momentum, self.grad = (torch.zeros(self.ctx.M, device="cuda") for _ in range(2))

        def views(flat):
            return [flat[o:o + m * n].view(m, n) for o, (m, n) in zip(offs, SHAPES)]
        self.w_gate, self.w_up, self.w_down = views(self.weights)
        self.d_gate, self.d_up, self.d_down = views(self.grad)

    def _like(self, x, cols):
        return torch.empty((x.shape[0], cols), device="cuda", dtype=torch.bfloat16)

    def forward(self, x):
        ctx = self.ctx
        self.x, self.g, self.u, self.h = x, self._like(x, F), self._like(x, F), self._like(x, F)
        ctx.gated_forward(x, self.w_gate, self.w_up, self.h, act="silu", gate=self.g, up=self.u)
        h8, self.h8_t = ctx.i8_quantize_both(self.h)
        w8, self.w8_t = ctx.i8_quantize_both(self.w_down)
        return ctx.i8_matmul(h8, w8, self._like(x, D))

    def backward(self, dy, seed):
        """All gradients into the flat gradient; returns dx."""
        ctx = self.ctx
        dy8, dy8_t = ctx.i8_quantize_both(dy, stochastic=True, seed=seed)
        self.dh = ctx.i8_matmul(dy8, self.w8_t, self._like(dy, F))
        ctx.i8_matmul(dy8_t, self.h8_t, self.d_down)
        dx = self._like(dy, D)
        ctx.gated_backward(self.dh, self.g, self.u, self.x, self.w_gate, self.w_up, act="silu", dx=dx, dw_gate=self.d_gate, dw_up=self.d_up)
        return dx

    def step(self, lr):
        self.plan.step(self.grad, self.momentum, self.weights, lr=lr, beta=0.9)

    def kept(self):
        """The matrices as an answering program keeps them."""
        return [self.ctx.i8_quantize(w) for w in (self.w_gate, self.w_up, self.w_down)]

    def answer(self, x, kept):
        ctx = self.ctx
        h = ctx.i8_gated(ctx.i8_quantize(x), kept[0], kept[1], self._like(x, F), act="silu")
        return ctx.i8_matmul(ctx.i8_quantize(h), kept[2], self._like(x, D))


def train(steps=40, seed=0, lr=0.02, verbose=False):
    block, teacher = GatedBlock(seed), GatedBlock(seed + 1)
    gen = torch.Generator(device="cuda").manual_seed(seed + 2)
    losses = []
    for it in range(steps):
        x = torch.randn(BATCH, D, generator=gen, device="cuda").bfloat16()
        diff = (block.forward(x) - teacher.forward(x)).float()
        losses.append(diff.square().mean())
        block.backward((diff * (2.0 / diff.numel())).bfloat16(), seed=it)
        block.step(lr)
    block.ctx.device_status()
    teacher.ctx.device_status()
    losses = [float(v) for v in losses]
    if verbose:
        for i in range(0, steps, max(1, steps // 10)):
            print(f"step {i:4d}  loss {losses[i]:.5f}")
    return losses, block


if __name__ == "__main__":
    train(int(sys.argv[1]) if len(sys.argv) > 1 else 40, verbose=True)
