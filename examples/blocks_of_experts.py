"""A model of blocks on letter windows: embeddings, a residual stream, mixtures of experts, clipped changes.

    python examples/blocks_of_experts.py [--dtype f32|bf16] [--steps 100] [--patterns 512]

A pattern is a window of seven letters.  Each letter's row of a table joins a stream of its own (a row of 64 units); two blocks
follow.  A block norms the stream, sends each row to 2 of 8 experts (two-layer sigmoid nets) by sigmoid scores within its best 2 of
4 groups of experts, and adds their gated outputs, normed, gated and scaled, to the stream.  The seven rows of a window, normed
once more, are the input of one layer with 26 outputs.  After a step each router's bias is moved against the load of its experts,
which is all that it is for, and all changes together are scaled down to a bound before the momentum update.

Every product, norm, choice and gradient runs in the library's kernels; torch holds the buffers, adds two gradients of
one input, and applies the update and the outputs' slope.  G is minus the gradient of half the squared error.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
for path in (HERE, os.path.dirname(HERE)):
    if path not in sys.path:
        sys.path.insert(0, path)

from experts_and_adapters import Momentum  # noqa: E402
from paper_1801_01554_gb300 import bp, synth  # noqa: E402

LETTERS, WINDOW, WIDTH, HIDDEN, OUTPUTS = 29, 7, 64, 32, 32   # (26 outputs, padded to whole 16-byte pieces)
EXPERTS, CHOICES, GROUPS, OPEN, BLOCKS = 8, 2, 4, 2, 2
SCALE, BOUND = 0.5, 1.0


def windows(n, seed):
    """Letters of n windows [n, 7] and three-hot targets."""
    X, T = synth.nettalk_patterns(n, seed)
    ids = torch.tensor(X.reshape(n, WINDOW, LETTERS).argmax(2), dtype=torch.int32, device="cuda")
    return ids.contiguous(), torch.nn.functional.pad(torch.tensor(T), (0, OUTPUTS - T.shape[1])).float().cuda().contiguous()


class Block:
    """One block: norm, router, experts, mix, and its way back into the stream."""

    def __init__(self, rows, dtype, gen):
        t = torch.bfloat16 if dtype == bp.BP_BF16 else torch.float32
        picked = rows * CHOICES
        self.rows, self.picked, self.dtype = rows, picked, dtype
        self.R = Momentum((1, EXPERTS, WIDTH), WIDTH ** -0.5, dtype, gen)
        self.W1 = Momentum((EXPERTS, HIDDEN, WIDTH), WIDTH ** -0.5, dtype, gen)
        self.W2 = Momentum((EXPERTS, WIDTH, HIDDEN), HIDDEN ** -0.5, dtype, gen)
        self.wo, self.gate, self.wi = (Momentum((k, WIDTH) if k else (WIDTH,), 0.0, bp.BP_F32, gen) for k in (0, 1, 0))
        for m in (self.wo, self.gate, self.wi):
            m.w.fill_(1.0)
            m.use.fill_(1.0)
        self.bias = torch.zeros(EXPERTS, device="cuda")
        self.linear = bp.Experts(1, WIDTH, EXPERTS, dtype, max_rows=rows)
        self.router = bp.ScoredRouter(EXPERTS, CHOICES, dtype, rows, bp.BP_SCORES_SIGMOID, GROUPS, OPEN, 2, True, 1.0)
        self.layer1 = bp.Experts(EXPERTS, WIDTH, HIDDEN, dtype, max_rows=picked)
        self.layer2 = bp.Experts(EXPERTS, HIDDEN, WIDTH, dtype, max_rows=picked)
        self.stream = bp.Residual(WIDTH, dtype, rows, bp.BP_NORM_RMS, bp.BP_NORM_RMS, 1e-5)

        def buf(*shape, dtype=t):
            return torch.zeros(shape, dtype=dtype, device="cuda")
        self.all = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
        self.logits, self.dlogits = buf(rows, EXPERTS), buf(rows, EXPERTS)
        self.expert, self.place = buf(rows, CHOICES, dtype=torch.int32), buf(rows, CHOICES, dtype=torch.int32)
        self.g, self.dg = buf(rows, CHOICES, dtype=torch.float32), buf(rows, CHOICES, dtype=torch.float32)
        self.offsets, self.source = buf(EXPERTS + 1, dtype=torch.int32), buf(picked, dtype=torch.int32)
        self.A, self.dA = buf(picked, HIDDEN), buf(picked, HIDDEN)
        self.O, self.dO, self.dP = buf(picked, WIDTH), buf(picked, WIDTH), buf(picked, WIDTH)
        self.F, self.dF, self.Y, self.H = (buf(rows, WIDTH) for _ in range(4))
        self.dX, self.dH, self.dR = (buf(rows, WIDTH) for _ in range(3))
        self.stats = buf(rows, 4, dtype=torch.float32)

    def weights(self):
        return self.R, self.W1, self.W2, self.wo, self.gate, self.wi

    def way(self):
        return dict(wo=self.wo.w, gate=self.gate.w, n_gates=1, scale=SCALE, wi=self.wi.w)

    def forward(self, X, H):
        """The stream behind the block, and its norm: Y, H."""
        n, k = self.rows, self.picked
        self.H_in = H
        self.linear.forward(self.R.use, None, H, n, None, self.all, n, self.logits)
        self.router.forward(self.logits, self.bias, n, self.expert, self.g, self.offsets, self.source, self.place)
        self.layer1.forward(self.W1.use, None, H, n, self.source, self.offsets, k, self.A, squash=True)
        self.layer2.forward(self.W2.use, None, self.A, k, None, self.offsets, k, self.O, squash=True)
        bp.bp_mix(self.O, k, self.place, self.g, n, CHOICES, WIDTH, self.dtype, self.F)
        self.stream.forward(X, self.F, n, self.Y, self.H, self.stats, **self.way())
        return self.Y, self.H

    def backward(self, dY, dH):
        """The gradients of the stream and of its norm before the block, from those behind it (dY None: 0)."""
        n, k = self.rows, self.picked
        self.stream.backward(self.Y, self.F, n, self.stats, dY, dH, self.dX, self.dF, Gwo=self.wo.g, Ggate=self.gate.g,
                             Gwi=self.wi.g, **self.way())
        bp.bp_mix_backward(self.dF, self.O, k, self.place, self.g, n, CHOICES, WIDTH, self.dtype, self.dO, self.dg)
        self.router.backward(self.logits, n, self.expert, self.dg, self.dlogits)
        self.linear.backward(self.R.use, self.H_in, n, None, self.all, n, self.dlogits, dX=self.dR, GW=self.R.g)
        D2 = self.dO * self.O * (1 - self.O)
        self.layer2.backward(self.W2.use, self.A, k, None, self.offsets, k, D2, dX=self.dA, GW=self.W2.g, squash=True)
        self.layer1.backward(self.W1.use, self.H_in, n, self.source, self.offsets, k, self.dA, dX=self.dP, GW=self.W1.g)
        bp.bp_mix(self.dP, k, self.place, None, n, CHOICES, WIDTH, self.dtype, self.dH)   # the rows of a pattern
        return self.dX, self.dH.add_(self.dR)

    def balance(self, rate=0.01):
        """The bias of experts with more rows than the mean goes down, that of the others up."""
        load = (self.offsets[1:] - self.offsets[:-1]).float()
        self.bias.sub_(rate * torch.sign(load - load.mean()))

    def check(self):
        for layer in (self.linear, self.layer1, self.layer2, self.stream):
            layer.check()


class Model:
    def __init__(self, n, dtype, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        t = torch.bfloat16 if dtype == bp.BP_BF16 else torch.float32
        rows = n * WINDOW
        self.n, self.rows, self.dtype, self.t = n, rows, dtype, t
        self.table = Momentum((LETTERS, WIDTH), 1.0, dtype, gen)
        self.wi = Momentum((WIDTH,), 0.0, bp.BP_F32, gen)
        self.wi.w.fill_(1.0)
        self.W = Momentum((1, OUTPUTS, WINDOW * WIDTH), (WINDOW * WIDTH) ** -0.5, dtype, gen)
        self.b = Momentum((1, OUTPUTS), 0.0, bp.BP_F32, gen)
        self.b.w.fill_(-2.0)   # few of a pattern's targets are ones
        self.blocks = [Block(rows, dtype, gen) for _ in range(BLOCKS)]
        self.embed = bp.Embedding(LETTERS, WIDTH, dtype, max_ids=rows)
        self.first = bp.Residual(WIDTH, dtype, rows, bp.BP_NORM_NONE, bp.BP_NORM_RMS, 1e-5)
        self.head = bp.Experts(1, WINDOW * WIDTH, OUTPUTS, dtype, max_rows=n)
        self.all = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        self.X, self.H, self.dX, self.dHead = (torch.zeros(rows, WIDTH, dtype=t, device="cuda") for _ in range(4))
        self.stats, self.Y = torch.zeros(rows, 4, device="cuda"), torch.zeros(n, OUTPUTS, dtype=t, device="cuda")
        self.clip = bp.Clip([m.g for m in self.weights()])
        self.norm = torch.zeros(1, device="cuda")

    def weights(self):
        return [self.table, self.wi, self.W, self.b] + [m for block in self.blocks for m in block.weights()]

    def forward(self, ids):
        self.embed.forward(self.table.use, ids, self.rows, self.X)
        self.first.forward(self.X, None, self.rows, None, self.H, self.stats, wi=self.wi.w)
        x, h = self.X, self.H
        for block in self.blocks:
            x, h = block.forward(x, h)
        self.head.forward(self.W.use, self.b.w, h, self.n, None, self.all, self.n, self.Y, squash=True)
        return self.Y

    def gradients(self, ids, T):
        """Every weight's change from the patterns' mean, unclipped, in m.g; returns the errors [n, outputs]."""
        y = self.forward(ids).float()
        err = T - y
        D = (err * y * (1 - y) / self.n).to(self.t)
        h = self.blocks[-1].H
        self.head.backward(self.W.use, h, self.n, None, self.all, self.n, D, dX=self.dHead, GW=self.W.g, Gb=self.b.g)
        dx, dh = None, self.dHead
        for block in reversed(self.blocks):
            dx, dh = block.backward(dx, dh)
        self.first.backward(self.X, None, self.rows, self.stats, dx, dh, self.dX, wi=self.wi.w, Gwi=self.wi.g)
        self.embed.backward(ids, self.rows, self.dX, self.table.g)
        return err

    def step(self, ids, T, lr):
        """One update; returns the squared error a pattern (a tensor)."""
        err = self.gradients(ids, T)
        self.clip.run(BOUND, self.norm)
        for m in self.weights():
            m.update(lr)
        for block in self.blocks:
            block.balance()
        return err.square().sum() / self.n

    def check(self):
        for layer in [self.embed, self.first, self.head, self.clip] + self.blocks:
            layer.check()


def train(dtype, steps, patterns, lr=0.3):
    """Squared errors a pattern, step by step."""
    ids, T = windows(patterns, seed=1)
    model = Model(patterns, dtype)
    errors = [model.step(ids, T, lr) for _ in range(steps)]
    model.check()
    return torch.stack(errors).cpu(), model


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--dtype", choices=["f32", "bf16"], default="f32")
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--patterns", type=int, default=512)
    a = ap.parse_args()
    e, model = train(bp.BP_BF16 if a.dtype == "bf16" else bp.BP_F32, a.steps, a.patterns)
    rows = [(b.offsets[1:] - b.offsets[:-1]).tolist() for b in model.blocks]
    print(f"squared error a pattern {e[0]:.3f} -> {e[-1]:.3f}; norm of the last changes {float(model.norm):.3f}; rows of the experts {rows}")


if __name__ == "__main__":
    main()
