"""Clipping of values whose norm, or whose factor, float32 does not hold.

Bounds: those of test_gpu_clip, 20 * 2^-24 of a value and half a unit of bfloat16; where the result is below float32's (bfloat16's)
normal numbers half a unit there, 2^-150 (2^-134), and one more unit of float32 ahead of a second rounding.
"""
import numpy as np
import pytest

from expert_cases import BF16, dev, empty, host, rounded
from oracle import blocks_oracle as O
from paper_1801_01554_gb300 import bp

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

NORM, VALUE = 18 * 2.0 ** -24, 20 * 2.0 ** -24
MOST = float(np.finfo(np.float32).max)
SMALLEST = 2.0 ** -149


def check(values, dtypes, max_norm, in_place):
    ins = [dev(v, t) for v, t in zip(values, dtypes)]
    outs = None if in_place else [empty(v.shape, t) for v, t in zip(values, dtypes)]
    norm = torch.full((1,), -1.0, device="cuda")
    with bp.Clip(ins, outs) as clip:
        clip.run(max_norm, norm)
        clip.check()   # nothing is latched
    want, clipped = O.clip(values, max_norm)
    assert want > max_norm
    if want > MOST * (1 + 2.0 ** -25):
        assert float(norm) == np.inf
    else:
        assert abs(float(norm) - want) <= NORM * want
    for x, w, t in zip(ins if in_place else outs, clipped, dtypes):
        half, least = (BF16, 2.0 ** -134) if t == bp.BP_BF16 else (0.0, 2.0 ** -150)
        err, bound = np.abs(host(x) - w), (VALUE + half) * np.abs(w) + least + SMALLEST
        assert (err <= bound).all(), float(np.max(err / bound))


# a few values go to one launch, more of them to two
@pytest.mark.parametrize("sizes", [[5, 3], [20000, 7], [200000, 31, 9000]], ids=sum)
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("scale,max_norm", [
    (3e38, 1.0), (3e38, 1e30), (3e38, 3e38), (1e38, 1e-9), (3e38, 1e-20), (1e30, 1e-8), (1e37, 1e-3), (1e25, 1e-25), (1e38, 1e-38),
    (1e-36, 1e-41), (1e38, SMALLEST)])
def test_factors_below_float32(scale, max_norm, in_place, sizes):
    rng = np.random.default_rng([sum(sizes), 5])
    dtypes = [bp.BP_BF16 if i == 1 else bp.BP_F32 for i in range(len(sizes))]
    values = [rounded(rng.choice([-1.0, 1.0], size=s) * rng.uniform(0.5, 1.0, size=s) * scale, t) for s, t in zip(sizes, dtypes)]
    values[0][:2] = rounded(scale, bp.BP_F32), -rounded(scale, bp.BP_F32)
    check(values, dtypes, float(np.float32(max_norm)), in_place)


def test_two_values_beyond_float32_together():
    """Both values are finite; their norm is not, as float32 has it."""
    check([np.full(2, float(np.float32(3e38)))], [bp.BP_F32], 1.0, False)
    check([np.full(2, MOST)], [bp.BP_F32], MOST, True)
