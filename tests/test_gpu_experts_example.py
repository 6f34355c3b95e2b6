"""The example that runs the router, expert, mix and adapter layers together learns: the error falls,
in both dtypes to about the same value, and a mixture's step is the oracle's."""
import os
import sys

import numpy as np
import pytest

from expert_cases import host
from oracle import experts_oracle as O
from paper_1801_01554_gb300 import bp

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("dtype", [bp.BP_F32, bp.BP_BF16])
def test_the_example_learns(dtype):
    import experts_and_adapters as ex
    e, net = ex.train_mixture(dtype, 150, 500)
    e = e.numpy()
    # 500 patterns of 3-hot targets: the best constant answer, 3/26 everywhere, errs by 3 - 9/26
    assert np.isfinite(e).all() and e[-1] < 0.9 * (3 - 9 / 26) < e[0]
    a = ex.train_adapters(net, dtype, 150, 500).numpy()
    assert np.isfinite(a).all() and a[-1] < 0.9 * a[0]


def test_a_mixture_step_is_the_oracles():
    """Every change of one float32 step, from the oracle's operators chained in float64.  Normwise
    1e-4: sums of up to 1,000 products through five operators, each within 1e-6 of its own."""
    import experts_and_adapters as ex
    n = 200
    X, T = ex.letters(n, bp.BP_F32, seed=5)
    net = ex.Mixture(n, X.shape[1], T.shape[1], bp.BP_F32, seed=6)
    w = {k: host(getattr(net, k).w) for k in ("R", "W1", "W2", "b1", "b2")}
    x, t = host(X), host(T)
    net.step(X, T, lr=0.0)
    net.check()
    z = x @ w["R"][0].T
    expert, gate, offsets, source, place = O.route(z, ex.CHOICES, "chosen")
    a = O.logistic(O.experts_forward(w["W1"], w["b1"], x, source, offsets, len(source))[0])
    h = O.logistic(O.experts_forward(w["W2"], w["b2"], a, None, offsets, len(source))[0])
    d = (t - O.mix(h, place, gate)) / n
    dh = np.zeros_like(h)
    dgate = O.mix_backward(d, h, place, gate, dh)
    dz = O.route_backward(z, expert, gate, dgate, "chosen")
    (da, _), (g2, _), (gb2, _) = O.experts_backward(w["W2"], a, None, offsets, dh * h * (1 - h), True)
    _, (g1, _), (gb1, _) = O.experts_backward(w["W1"], x, source, offsets, da, False)
    np.testing.assert_array_equal(net.expert.cpu().numpy(), expert)
    for name, got, want in (("W1", net.W1.g, g1), ("W2", net.W2.g, g2), ("b1", net.b1.g, gb1), ("b2", net.b2.g, gb2),
                            ("R", net.R.g[0], dz.T @ x)):
        assert np.abs(host(got) - want).max() <= 1e-4 * np.abs(want).max(), name
