"""The oracle of the router by scores against differences and a choice one by one, and what the library
refuses before it touches the GPU (no GPU)."""
import ctypes
import itertools
import os

import numpy as np
import pytest

from oracle import experts_oracle as O
from paper_1801_01554_gb300 import bp, build

P = 0x10000   # an address that is never read


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(bp.lib_path()):
        build.build()
    return bp.load()


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
def test_gradient_is_the_difference(kind, renormalise):
    rng = np.random.default_rng(3)
    z, bias, dgate = rng.standard_normal((7, 12)), rng.standard_normal(12) * 0.1, rng.standard_normal((7, 3))
    z[2, 4:] = -np.inf
    z[3] = -np.inf
    way = dict(kind=kind, renormalise=renormalise, scale=1.5)
    groups = dict(n_groups=4, open_groups=2, group_top=2)
    expert = O.route_scored(z, bias, 3, **way, **groups)[0]
    assert (expert[3] == -1).all() and (expert[2] < 4).all()

    def loss():
        again, gate = O.route_scored(z, bias, 3, **way, **groups)[:2]
        assert (again == expert).all()
        return (gate * dgate).sum()
    got, mag = O.route_scored_backward(z, expert, dgate, **way)
    for i in np.ndindex(*z.shape):
        was = z[i]
        if was == -np.inf:
            assert got[i] == 0
            continue
        z[i] = was + 1e-6
        up = loss()
        z[i] = was - 1e-6
        assert abs((up - loss()) / 2e-6 - got[i]) < 1e-8 and mag[i] >= abs(got[i]) - 1e-15
        z[i] = was


def test_choice_is_the_best_one():
    """Against every set of open groups, for every pattern, one expert at a time."""
    rng = np.random.default_rng(4)
    E, G, k = 12, 4, 4
    z, bias = np.round(rng.standard_normal((40, E)), 1), np.round(rng.standard_normal(E) * 0.2, 1)
    z[rng.random(z.shape) < 0.3] = -np.inf
    for top, open_ in itertools.product((1, 2), (2, 3)):
        expert = O.route_scored(z, bias, k, "sigmoid", G, open_, top)[0]
        for t in range(len(z)):
            c = [1 / (1 + np.exp(-x)) + b if x > -np.inf else -np.inf for x, b in zip(z[t], bias)]
            worth = [sum(sorted((x for x in c[g * 3:g * 3 + 3] if x > -np.inf), reverse=True)[:top]) if max(c[g * 3:g * 3 + 3]) > -np.inf
                     else -np.inf for g in range(G)]
            groups = sorted(range(G), key=lambda g: (-worth[g], g))[:open_]
            best = sorted((e for e in range(E) if e // 3 in groups and c[e] > -np.inf), key=lambda e: (-c[e], e))[:k]
            assert expert[t].tolist() == best + [-1] * (k - len(best))


GOOD = (8, 2, 0, 4, 0, 2, 1, 1, 0, 1.0)


@pytest.mark.parametrize("at,value", [(0, 0), (0, 513), (0, 7), (1, 0), (1, 5), (2, 5), (3, 0), (3, 2 ** 31 - 1), (4, 2), (4, -1), (5, 0),
                                      (5, 3), (5, 33), (6, 0), (6, 3), (7, 0), (7, 3), (9, float("nan")), (9, float("inf"))])
def test_create_refuses(lib, at, value):
    out = ctypes.c_void_p()
    args = GOOD[:at] + (value,) + GOOD[at + 1:]
    assert lib.bp_scored_router_create(*args, ctypes.byref(out)) == bp.BP_EINVAL
    assert out.value is None and lib.bp_last_error()
    assert lib.bp_scored_router_create(*GOOD, None) == bp.BP_EINVAL


def test_null_routers_are_refused(lib):
    assert lib.bp_route_scored(None, P, P, 1, P, P, P, P, P, None) == bp.BP_EINVAL
    assert lib.bp_route_scored_backward(None, P, 1, P, P, P, None) == bp.BP_EINVAL
    lib.bp_scored_router_destroy(None)   # NULL-safe
