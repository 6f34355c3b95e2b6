"""A mixture of experts on letter windows, and adapters for readers who want other answers.

    python examples/experts_and_adapters.py [--dtype f32|bf16] [--steps 200] [--patterns 1024]

1. Mixture.  A router (one linear layer) sends each pattern to 2 of 8 experts, two-layer sigmoid nets
   of the letter-to-phoneme shape; the pattern's answer is the gated sum of their outputs.  A step is:
   router forward, both layers' products grouped by expert, the mix, then the gradients back through all
   of them and the momentum update of every weight.
2. Adapters.  The mean expert's first layer stays as it is for everyone; each of three readers has a
   low-rank adapter beside it, trained on that reader's own targets, all in one pass over rows of very
   different numbers.

Every product and gradient runs in the library's kernels; torch holds the buffers, applies the update and
the outputs' slope.  G is minus the gradient of half the squared error, as everywhere in the library.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_1801_01554_gb300 import bp, synth  # noqa: E402

EXPERTS, CHOICES, HIDDEN = 8, 2, 64


def letters(n, dtype, seed):
    """Letter windows and three-hot targets; bfloat16 rows are padded to whole 16-byte pieces."""
    X, T = synth.nettalk_patterns(n, seed)
    X, T = torch.tensor(X), torch.tensor(T)
    if dtype == bp.BP_BF16:
        X = torch.nn.functional.pad(X, (0, 208 - 203))
        T = torch.nn.functional.pad(T, (0, 32 - 26))
    t = torch.bfloat16 if dtype == bp.BP_BF16 else torch.float32
    return X.to(t).cuda().contiguous(), T.float().cuda().contiguous()


class Momentum:
    """float32 master weights, their velocity, and the copy in the kernels' type."""

    def __init__(self, shape, scale, dtype, gen):
        self.w = torch.randn(shape, generator=gen, device="cuda") * scale
        self.v = torch.zeros_like(self.w)
        self.g = torch.zeros_like(self.w)
        self.t = torch.bfloat16 if dtype == bp.BP_BF16 else torch.float32
        self.use = self.w.to(self.t)

    def update(self, lr, momentum=0.9):
        self.v.mul_(momentum).add_(self.g, alpha=lr)
        self.w.add_(self.v)
        self.use.copy_(self.w)


class Mixture:
    """A router over experts of two layers, for a fixed number of patterns a step."""

    def __init__(self, n, n_in, n_out, dtype, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        t = torch.bfloat16 if dtype == bp.BP_BF16 else torch.float32
        rows = n * CHOICES
        self.n, self.rows, self.n_out, self.dtype = n, rows, n_out, dtype
        self.R = Momentum((1, EXPERTS, n_in), n_in ** -0.5, dtype, gen)
        self.W1 = Momentum((EXPERTS, HIDDEN, n_in), n_in ** -0.5, dtype, gen)
        self.W2 = Momentum((EXPERTS, n_out, HIDDEN), HIDDEN ** -0.5, dtype, gen)
        self.b1 = Momentum((EXPERTS, HIDDEN), 0.0, bp.BP_F32, gen)
        self.b2 = Momentum((EXPERTS, n_out), 0.0, bp.BP_F32, gen)
        self.b2.w.fill_(-2.0)   # few of a pattern's targets are ones
        self.b2.update(0.0)
        self.linear = bp.Experts(1, n_in, EXPERTS, dtype, max_rows=n)   # the router's layer: one group
        self.router = bp.Router(EXPERTS, CHOICES, dtype, max_patterns=n)
        self.layer1 = bp.Experts(EXPERTS, n_in, HIDDEN, dtype, max_rows=rows)
        self.layer2 = bp.Experts(EXPERTS, HIDDEN, n_out, dtype, max_rows=rows)

        def buf(*shape, dtype=t):
            return torch.zeros(shape, dtype=dtype, device="cuda")
        self.all = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        self.logits, self.dlogits = buf(n, EXPERTS), buf(n, EXPERTS)
        self.expert, self.place = buf(n, CHOICES, dtype=torch.int32), buf(n, CHOICES, dtype=torch.int32)
        self.gate, self.dgate = buf(n, CHOICES, dtype=torch.float32), buf(n, CHOICES, dtype=torch.float32)
        self.offsets, self.source = buf(EXPERTS + 1, dtype=torch.int32), buf(rows, dtype=torch.int32)
        self.A, self.dA = buf(rows, HIDDEN), buf(rows, HIDDEN)
        self.H, self.dH = buf(rows, n_out), buf(rows, n_out)
        self.Y = buf(n, n_out)

    def forward(self, X):
        self.linear.forward(self.R.use, None, X, self.n, None, self.all, self.n, self.logits)
        self.router.forward(self.logits, self.n, self.expert, self.gate, self.offsets, self.source, self.place)
        self.layer1.forward(self.W1.use, self.b1.w, X, self.n, self.source, self.offsets, self.rows, self.A,
                            squash=True)
        self.layer2.forward(self.W2.use, self.b2.w, self.A, self.rows, None, self.offsets, self.rows, self.H,
                            squash=True)
        bp.bp_mix(self.H, self.rows, self.place, self.gate, self.n, CHOICES, self.n_out, self.dtype, self.Y)
        return self.Y

    def step(self, X, T, lr):
        """One update from the patterns' mean change; returns the squared error a pattern (a tensor)."""
        err = T - self.forward(X).float()
        D = (err / self.n).to(self.Y.dtype)
        bp.bp_mix_backward(D, self.H, self.rows, self.place, self.gate, self.n, CHOICES, self.n_out, self.dtype,
                           self.dH, self.dgate)
        self.router.backward(self.logits, self.n, self.expert, self.gate, self.dgate, self.dlogits)
        self.linear.backward(None, X, self.n, None, self.all, self.n, self.dlogits, GW=self.R.g)
        D2 = self.dH * self.H * (1 - self.H)
        self.layer2.backward(self.W2.use, self.A, self.rows, None, self.offsets, self.rows, D2, dX=self.dA,
                             GW=self.W2.g, Gb=self.b2.g, squash=True)
        self.layer1.backward(None, X, self.n, self.source, self.offsets, self.rows, self.dA, GW=self.W1.g,
                             Gb=self.b1.g)
        for m in (self.R, self.W1, self.W2, self.b1, self.b2):
            m.update(lr)
        return err.square().sum() / self.n

    def check(self):
        for layer in (self.linear, self.layer1, self.layer2):
            layer.check()


def train_mixture(dtype, steps, patterns, lr=2.0):
    """Squared errors a pattern, step by step."""
    X, T = letters(patterns, dtype, seed=1)
    net = Mixture(patterns, X.shape[1], T.shape[1], dtype)
    errors = [net.step(X, T, lr) for _ in range(steps)]
    net.check()
    return torch.stack(errors).cpu(), net


def train_adapters(net, dtype, steps, patterns, rank=8, lr=20.0):
    """Squared errors a pattern of three readers' rows, step by step, with the shared layer as it is."""
    X, T = letters(patterns, dtype, seed=2)
    n, n_in, n_out = patterns, X.shape[1], T.shape[1]
    t = X.dtype
    gen = torch.Generator(device="cuda").manual_seed(3)
    W = torch.randn(n_out, n_in, generator=gen, device="cuda").mul_(n_in ** -0.5).to(t)
    b = torch.full((n_out,), -2.0, device="cuda")
    readers = 3
    ends = torch.tensor([0, n // 2, n // 2 + n // 3, n], dtype=torch.int32, device="cuda")
    reader = torch.arange(readers, dtype=torch.int32, device="cuda")
    for i in range(readers):   # each reader has the targets in another order
        lo, hi = int(ends[i]), int(ends[i + 1])
        T[lo:hi] = T[lo:hi].roll(i, dims=1)
    A = Momentum((readers, rank, n_in), n_in ** -0.5, dtype, gen)
    B = Momentum((readers, rank, n_out), 0.0, dtype, gen)
    U = torch.zeros(n, rank, device="cuda")
    Y = torch.zeros(n, n_out, dtype=t, device="cuda")
    errors = []
    with bp.Adapters(readers, rank, n_in, n_out, dtype, max_rows=n, max_requests=readers) as layer:
        for _ in range(steps):
            where = (ends, reader, readers, n)
            layer.forward(W, b, A.use, B.use, None, X, *where, U, Y, squash=True)
            y = Y.float()
            err = T - y
            D = (err * y * (1 - y) / n).to(t)
            layer.backward(W, A.use, B.use, None, X, U, *where, D, GA=A.g, GB=B.g)
            A.update(lr)
            B.update(lr)
            errors.append(err.square().sum() / n)
        layer.check()
    return torch.stack(errors).cpu()


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--dtype", choices=["f32", "bf16"], default="f32")
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--patterns", type=int, default=1024)
    a = ap.parse_args()
    dtype = bp.BP_BF16 if a.dtype == "bf16" else bp.BP_F32
    e, net = train_mixture(dtype, a.steps, a.patterns)
    rows = (net.offsets[1:] - net.offsets[:-1]).tolist()
    print(f"mixture: squared error a pattern {e[0]:.3f} -> {e[-1]:.3f}; rows of the experts {rows}")
    e = train_adapters(net, dtype, a.steps, a.patterns)
    print(f"adapters: squared error a pattern {e[0]:.3f} -> {e[-1]:.3f}")


if __name__ == "__main__":
    main()
