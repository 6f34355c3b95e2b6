"""What the tests of the router, expert and adapter layers share: inputs, device buffers and the
bound on a rounded sum (test infrastructure).

The bound.  A product sum is taken in float32 (by the tensor cores at the least as 16 products a
step, truncated to 24 bits; a sum in one accumulator has at most 128 such steps, or is added up
from such parts; the FMA kernels round to nearest), so that its error is at most 128 * 2^-23 =
2^-16 of the sum of the products' magnitudes.  A value stored as bfloat16 is rounded once more,
by half a unit of its eighth significant bit, 2^-8 of itself at most.  The logistic has a slope of at most 1/4 and is evaluated with a few
float32 roundings, 2^-20.
"""
import numpy as np

from paper_1801_01554_gb300 import bp, synth

try:
    import torch
except ImportError:   # pragma: no cover
    torch = None

SUM = 2.0 ** -16
BF16 = 2.0 ** -8
FUNC = 2.0 ** -20


def rounded(x, dtype):
    """float64 values that the dtype holds exactly."""
    return synth.round_to(np.asarray(x, dtype=np.float64), "bf16" if dtype == bp.BP_BF16 else "f32")


def dev(x, dtype=None):
    """A CUDA tensor: float32 or bfloat16 values, or int32 for whole numbers."""
    if x is None:
        return None
    x = np.asarray(x)
    if x.dtype.kind in "iu":
        return torch.tensor(x, dtype=torch.int32, device="cuda")
    t = torch.tensor(x, dtype=torch.float32, device="cuda")
    return t.to(torch.bfloat16) if dtype == bp.BP_BF16 else t


def empty(shape, dtype, fill=float("nan")):
    t = torch.bfloat16 if dtype == bp.BP_BF16 else torch.float32
    return torch.full(shape, fill, dtype=t, device="cuda")


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def assert_sum(got, want, mag, dtype, squash=False, what=""):
    """got within the bound of the oracle's sum `want` (its logistic with squash)."""
    err_sum = SUM * mag
    if squash:
        want = 1.0 / (1.0 + np.exp(-want))
        err_sum = err_sum / 4 + FUNC * want
    bound = err_sum + (BF16 if dtype == bp.BP_BF16 else 2.0 ** -23) * (np.abs(want) + err_sum) + 1e-30
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:4].tolist(),
                           float(np.max(np.abs(got - want) / bound)))


def ragged(rng, n, parts, empties=True):
    """Ascending offsets [parts + 1] of n rows; with empties some parts get none."""
    w = rng.random(parts) ** 3
    if empties and parts > 2:
        w[rng.integers(0, parts, size=max(1, parts // 4))] = 0.0
    if w.sum() == 0:
        w[0] = 1.0
    cut = np.round(np.cumsum(w) / w.sum() * n).astype(np.int32)
    cut[-1] = n
    return np.concatenate([[0], cut]).astype(np.int32)
