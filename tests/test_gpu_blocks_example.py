"""Embeddings, residual stream, router by scores, experts, mix and clipping together: the example runs in both dtypes, and every
change of a float32 step is the oracle's."""
import os
import sys

import numpy as np
import pytest

from expert_cases import host
from oracle import blocks_oracle as B
from oracle import experts_oracle as O
from paper_1801_01554_gb300 import bp

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

EPS = float(np.float32(1e-5))


@pytest.mark.parametrize("dtype", [bp.BP_F32, bp.BP_BF16])
def test_the_example_runs(dtype):
    import blocks_of_experts as ex
    e, model = ex.train(dtype, 3, 100)
    assert np.isfinite(e.numpy()).all() and np.isfinite(float(model.norm))
    for m in model.weights():
        assert torch.isfinite(m.w).all()
    for block in model.blocks:
        load = (block.offsets[1:] - block.offsets[:-1]).cpu().numpy()
        assert load.sum() == block.rows * ex.CHOICES and (block.bias != 0).any()


def test_a_step_is_the_oracles():
    """Every change of one float32 step before it is clipped, the norm, and the clipped changes, from the oracle's operators chained
    in float64.  Normwise 1e-4: sums of up to 1,500 terms through some twenty operators, each within 2e-6 of its own."""
    import blocks_of_experts as ex
    n = 60
    ids, T = ex.windows(n, seed=5)
    model = ex.Model(n, bp.BP_F32, seed=6)
    gen = torch.Generator(device="cuda").manual_seed(7)
    for block in model.blocks:   # weights and biases of no special value
        block.bias.normal_(0, 0.05, generator=gen)
        for m in (block.wo, block.gate, block.wi):
            m.w.normal_(1, 0.2, generator=gen)
    model.wi.w.normal_(1, 0.2, generator=gen)
    model.gradients(ids, T)
    model.check()
    got = [host(m.g) for m in model.weights()]
    table, wi, W, b = (host(m.w) for m in (model.table, model.wi, model.W, model.b))
    flat = ids.cpu().numpy().ravel()
    x = B.embed(table, flat, 1.0)
    x0, h = x, B.norm_in(x, wi, None, B.RMS, EPS)[0]
    kept = []
    for block in model.blocks:
        w = {k: host(getattr(block, k).w) for k in ("R", "W1", "W2", "wo", "gate", "wi")}
        z = h @ w["R"][0].T
        expert, gate, offsets, source, place = O.route_scored(z, host(block.bias), ex.CHOICES, "sigmoid", ex.GROUPS, ex.OPEN, 2, True)
        np.testing.assert_array_equal(block.expert.cpu().numpy(), expert)
        a = O.logistic(O.experts_forward(w["W1"], None, h, source, offsets, len(source))[0])
        o = O.logistic(O.experts_forward(w["W2"], None, a, None, offsets, len(source))[0])
        f = O.mix(o, place, gate)
        y = B.residual(x, f, w["wo"], None, w["gate"], None, ex.SCALE, B.RMS, EPS)[0]
        kept.append((w, h, z, expert, gate, offsets, source, place, a, o, f, y))
        x, h = y, B.norm_in(y, w["wi"], None, B.RMS, EPS)[0]
    hw = h.reshape(n, -1)
    out = O.logistic(hw @ W[0].T + b[0])
    d = (host(T) - out) * out * (1 - out) / n
    want = {"W": (d.T @ hw)[None], "b": d.sum(0)[None]}
    dy, dh = None, (d @ W[0]).reshape(h.shape)
    of_blocks = []
    for w, hin, z, expert, gate, offsets, source, place, a, o, f, y in reversed(kept):
        g = B.residual_backward(y, f, w["wo"], None, w["gate"], None, ex.SCALE, w["wi"], dy, dh, B.RMS, B.RMS, EPS)
        do = np.zeros_like(o)
        dgate = O.mix_backward(g["dF"][0], o, place, gate, do)
        dz = O.route_scored_backward(z, expert, dgate, "sigmoid", True)[0]
        (da, _), (g2, _), _ = O.experts_backward(w["W2"], a, None, offsets, do * o * (1 - o), True)
        (dp, _), (g1, _), _ = O.experts_backward(w["W1"], hin, source, offsets, da, False)
        of_blocks.append([(dz.T @ hin)[None], g1, g2] + [g[k][0] for k in ("Gwo", "Ggate", "Gwi")])
        dy, dh = g["dX"][0], O.mix(dp, place, np.ones(place.shape)) + dz @ w["R"][0]
    g = B.residual_backward(x0, None, None, None, None, None, 1.0, wi, dy, dh, B.NONE, B.RMS, EPS)
    want = [B.embed_backward(flat, g["dX"][0], 1.0, len(table))[0], g["Gwi"][0], want["W"], want["b"]]
    want += [x for block in reversed(of_blocks) for x in block]
    for i, (a, b) in enumerate(zip(got, want)):
        assert a.shape == b.shape and np.abs(a - b).max() <= 1e-4 * np.abs(b).max(), i
    bound = 0.25 * float(np.sqrt(sum((a * a).sum() for a in got)))
    model.clip.run(bound, model.norm)
    model.clip.check()
    norm, clipped = B.clip(got, float(np.float32(bound)))
    assert abs(float(model.norm) - norm) <= 2e-6 * norm
    for m, c in zip(model.weights(), clipped):
        assert np.abs(host(m.g) - c).max() <= 2e-6 * np.abs(c).max()
