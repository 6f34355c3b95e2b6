"""The oracle's gradients against differences of its forward passes, and the refusals of the
router, mix, expert and adapter calls (CPU: no device work is reached)."""
import ctypes
import os

import numpy as np
import pytest

from oracle import experts_oracle as O
from paper_1801_01554_gb300 import bp

H = 1e-6   # central differences of float64: error H^2 and 1e-16 / H


def difference(f, x):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        old = x[i]
        x[i] = old + H
        up = f()
        x[i] = old - H
        down = f()
        x[i] = old
        g[i] = (up - down) / (2 * H)
    return g


@pytest.mark.parametrize("gates", ["chosen", "all"])
def test_route_gradient_is_the_difference(gates):
    rng = np.random.default_rng(1)
    z = rng.standard_normal((5, 7))
    z[1, 3] = z[2, 0] = -np.inf
    z[3, :] = -np.inf
    z[4, 1:] = -np.inf
    dg = rng.standard_normal((5, 3))
    expert, gate, *_ = O.route(z, 3, gates)
    got = O.route_backward(z, expert, gate, np.where(expert >= 0, dg, 7.0), gates)
    finite = np.isfinite(z)
    x = np.where(finite, z, 0.0)

    def loss():
        _, g, *_ = O.route(np.where(finite, x, -np.inf), 3, gates)
        return float((g * dg).sum())
    want = np.where(finite, difference(loss, x), 0.0)
    np.testing.assert_allclose(got, want, atol=1e-8)


def test_mix_gradient_is_the_difference():
    rng = np.random.default_rng(2)
    Hm, D = rng.standard_normal((6, 4)), rng.standard_normal((3, 4))
    place = np.array([[0, 4], [5, -1], [2, 3]])
    gate = rng.random((3, 2))
    dH = np.zeros_like(Hm)
    dgate = O.mix_backward(D, Hm, place, gate, dH)
    np.testing.assert_allclose(dH, difference(lambda: float((O.mix(Hm, place, gate) * D).sum()), Hm), atol=1e-8)
    np.testing.assert_allclose(dgate, difference(lambda: float((O.mix(Hm, place, gate) * D).sum()), gate), atol=1e-8)


def test_experts_gradient_is_the_difference():
    rng = np.random.default_rng(3)
    W, b = rng.standard_normal((3, 2, 4)), rng.standard_normal((3, 2))
    X = rng.standard_normal((5, 4))
    source = np.array([0, 2, 2, 4, 1, 0])
    offsets = np.array([0, 2, 2, 6])
    D = rng.standard_normal((6, 2))
    (dX, _), (GW, _), (Gb, _) = O.experts_backward(W, X, source, offsets, D, False)

    def loss():
        return float((O.experts_forward(W, b, X, source, offsets, 6)[0] * D).sum())
    np.testing.assert_allclose(GW, difference(loss, W), atol=1e-7)
    np.testing.assert_allclose(Gb, difference(loss, b), atol=1e-7)
    per_pattern = np.zeros_like(X)
    np.add.at(per_pattern, source, dX)
    np.testing.assert_allclose(per_pattern, difference(loss, X), atol=1e-7)


def test_adapters_gradient_is_the_difference():
    rng = np.random.default_rng(4)
    W, A, B = rng.standard_normal((3, 4)), rng.standard_normal((2, 2, 4)), rng.standard_normal((2, 2, 3))
    scale, net = np.array([0.5, 2.0]), rng.standard_normal((6, 4))
    offsets, adapter = np.array([0, 1, 3, 3, 5, 6]), np.array([1, 0, 0, -1, 1])
    D = rng.standard_normal((6, 3))

    def loss():
        X = O.logistic(net)
        return float((O.adapters_forward(W, None, A, B, scale, X, offsets, adapter)[0][0] * D).sum())
    X = O.logistic(net)
    U = O.adapters_forward(W, None, A, B, scale, X, offsets, adapter)[1][0]
    (dX, _), (GA, _), (GB, _) = O.adapters_backward(W, A, B, scale, X, U, offsets, adapter, D, True)
    np.testing.assert_allclose(dX, difference(loss, net), atol=1e-7)   # through the logistic
    np.testing.assert_allclose(GA, difference(loss, A), atol=1e-7)
    np.testing.assert_allclose(GB, difference(loss, B), atol=1e-7)


# ------------------------------------------------------------------ refusals
@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(bp.lib_path()):
        from paper_1801_01554_gb300 import build
        build.build()
    return bp.load()


@pytest.mark.parametrize("args,status", [
    ((0, 1, 0, 8, 0), bp.BP_EINVAL), ((513, 1, 0, 8, 0), bp.BP_EINVAL), ((8, 0, 0, 8, 0), bp.BP_EINVAL),
    ((4, 5, 0, 8, 0), bp.BP_EINVAL), ((64, 17, 0, 8, 0), bp.BP_EINVAL), ((8, 2, 3, 8, 0), bp.BP_EINVAL),
    ((8, 2, 0, 0, 0), bp.BP_EINVAL), ((8, 2, 0, 2 ** 30, 0), bp.BP_EINVAL), ((8, 2, 0, 8, 2), bp.BP_EINVAL)])
def test_router_create_refuses(lib, args, status):
    out = ctypes.c_void_p()
    assert lib.bp_router_create(*args, ctypes.byref(out)) == status
    assert out.value is None and lib.bp_last_error()


@pytest.mark.parametrize("args,status", [
    ((0, 8, 8, 0, 1), bp.BP_EINVAL), ((513, 8, 8, 0, 1), bp.BP_EINVAL), ((2, 0, 8, 0, 1), bp.BP_EINVAL),
    ((2, 8, 0, 0, 1), bp.BP_EINVAL), ((2, 8, 8, 2, 1), bp.BP_EINVAL), ((2, 8, 8, 0, 0), bp.BP_EINVAL),
    ((2, 12, 8, 1, 1), bp.BP_ESHAPE), ((2, 8, 12, 1, 1), bp.BP_ESHAPE), ((2, 2 ** 21, 8, 0, 1), bp.BP_EINVAL)])
def test_experts_create_refuses(lib, args, status):
    out = ctypes.c_void_p()
    assert lib.bp_experts_create(*args, ctypes.byref(out)) == status
    assert out.value is None and lib.bp_last_error()


@pytest.mark.parametrize("args,status", [
    ((0, 4, 8, 8, 0, 1, 1), bp.BP_EINVAL), ((65536, 4, 8, 8, 0, 1, 1), bp.BP_EINVAL),
    ((2, 0, 8, 8, 0, 1, 1), bp.BP_EINVAL), ((2, 129, 8, 8, 0, 1, 1), bp.BP_EINVAL),
    ((2, 4, 8, 8, 5, 1, 1), bp.BP_EINVAL), ((2, 4, 8, 8, 0, 0, 1), bp.BP_EINVAL),
    ((2, 4, 8, 8, 0, 1, 0), bp.BP_EINVAL), ((2, 4, 9, 8, 1, 1, 1), bp.BP_ESHAPE)])
def test_adapters_create_refuses(lib, args, status):
    out = ctypes.c_void_p()
    assert lib.bp_adapters_create(*args, ctypes.byref(out)) == status
    assert out.value is None and lib.bp_last_error()


def test_null_handles_are_refused(lib):
    assert lib.bp_route(None, *[None] * 1, 0, *[None] * 6) == bp.BP_EINVAL
    assert lib.bp_route_backward(None, None, 0, *[None] * 5) == bp.BP_EINVAL
    assert lib.bp_experts_forward(None, None, None, None, 0, None, None, 0, 0, None, None) == bp.BP_EINVAL
    assert lib.bp_experts_backward(None, None, None, 0, None, None, 0, None, 0, None, None, None, 0,
                                   None) == bp.BP_EINVAL
    assert lib.bp_experts_check(None, None) == bp.BP_EINVAL
    assert lib.bp_adapters_forward(None, *[None] * 8, 0, 0, 0, None, None, None) == bp.BP_EINVAL
    assert lib.bp_adapters_backward(None, *[None] * 8, 0, 0, None, 0, None, None, None, 0, None) == bp.BP_EINVAL
    assert lib.bp_adapters_check(None, None) == bp.BP_EINVAL
    for free in (lib.bp_router_destroy, lib.bp_experts_destroy, lib.bp_adapters_destroy):
        free(None)
    for create, args in ((lib.bp_router_create, 5), (lib.bp_experts_create, 5), (lib.bp_adapters_create, 7)):
        assert create(*[1] * args, None) == bp.BP_EINVAL


P = 0x10000   # an address that is never read


@pytest.mark.parametrize("args,status,word", [
    ((P, 4, P, P, 4, 2, 12, 1, P, None), bp.BP_ESHAPE, "multiples of 8"),
    ((P, 4, P, P, 4, 0, 8, 1, P, None), bp.BP_EINVAL, "k"),
    ((P, 4, P, P, 4, 17, 8, 1, P, None), bp.BP_EINVAL, "k"),
    ((P, 4, P, P, -1, 2, 8, 1, P, None), bp.BP_EINVAL, "n"),
    ((P, -1, P, P, 4, 2, 8, 1, P, None), bp.BP_EINVAL, "n_rows"),
    ((P, 4, P, P, 4, 2, 0, 0, P, None), bp.BP_EINVAL, "n_out"),
    ((P, 4, P, P, 4, 2, 8, 2, P, None), bp.BP_EINVAL, "dtype"),
    ((P + 8, 4, P, P, 4, 2, 8, 1, P, None), bp.BP_EINVAL, "d_H must be 16-byte"),
    ((P, 4, P + 2, P, 4, 2, 8, 1, P, None), bp.BP_EINVAL, "d_place must be 4-byte"),
    ((P, 4, P, P + 1, 4, 2, 8, 1, P, None), bp.BP_EINVAL, "d_gate"),
    ((P, 4, P, P, 4, 2, 8, 1, P + 4, None), bp.BP_EINVAL, "d_Y must be 16-byte"),
    ((None, 4, P, P, 4, 2, 8, 1, P, None), bp.BP_EINVAL, "d_H is NULL"),
    ((P, 4, None, P, 4, 2, 8, 1, P, None), bp.BP_EINVAL, "d_place is NULL"),
    ((P, 4, P, P, 4, 2, 8, 1, None, None), bp.BP_EINVAL, "d_Y is NULL"),
    ((None, 0, None, None, 0, 2, 8, 1, None, None), bp.BP_OK, "")])   # no patterns: nothing to do
def test_mix_refuses(lib, args, status, word):
    assert lib.bp_mix(*args) == status
    assert word in lib.bp_last_error().decode()


@pytest.mark.parametrize("args,word", [
    ((P, None, 4, P, P, 4, 2, 8, 1, P, P, None), "d_H is NULL"),
    ((P, P, 4, P, P, 4, 2, 8, 1, None, P, None), "d_dH is NULL"),
    ((P, P, 4, P, P, 4, 2, 8, 1, P + 8, P, None), "d_dH must be 16-byte"),
    ((P, P, 4, P, P, 4, 2, 8, 1, P, P + 2, None), "d_dgate"),
    ((None, P, 4, P, P, 4, 2, 8, 1, P, P, None), "d_D is NULL")])
def test_mix_backward_refuses(lib, args, word):
    assert lib.bp_mix_backward(*args) == bp.BP_EINVAL
    assert word in lib.bp_last_error().decode()


def test_binding_refuses_wrong_types():
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError, match="int32"):
        bp._ints(torch.zeros(4, dtype=torch.int64), "offsets")
    with pytest.raises(ValueError, match="bfloat16"):
        bp._values(torch.zeros(4), bp.BP_BF16, "X")
    with pytest.raises(ValueError, match="float32"):
        bp._floats(torch.zeros(4, dtype=torch.float64), "gate")
    with pytest.raises(ValueError, match="CUDA"):
        bp._floats(torch.zeros(4), "gate")
