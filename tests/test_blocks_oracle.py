"""The blocks' oracle against differences, and what the library refuses before it touches the GPU (no GPU)."""
import ctypes
import os

import numpy as np
import pytest

from oracle import blocks_oracle as O
from paper_1801_01554_gb300 import bp, build

P = 0x10000   # an address that is never read


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(bp.lib_path()):
        build.build()
    return bp.load()


def difference(f, x, step=1e-6):
    """The gradient of f() by x, a value at a time."""
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        was = x[i]
        x[i] = was + step
        up = f()
        x[i] = was - step
        g[i] = (up - f()) / (2 * step)
        x[i] = was
    return g


# ------------------------------------------------------------------ embedding
def test_embedding_gradient_is_the_difference():
    rng = np.random.default_rng(0)
    table, D = rng.standard_normal((5, 3)), rng.standard_normal((9, 3))
    ids = np.array([0, 4, 4, -1, 2, 0, 4, 7, -3])
    G, mag = O.embed_backward(ids, D, 1.5, 5)
    np.testing.assert_allclose(G, difference(lambda: (O.embed(table, ids, 1.5) * D).sum(), table), atol=1e-8)
    assert (G[[1, 3]] == 0).all() and (mag >= np.abs(G)).all()


@pytest.mark.parametrize("args,status", [((0, 8, 0, 1), bp.BP_EINVAL), (((1 << 24) + 1, 8, 0, 1), bp.BP_EINVAL),
                                         ((4, 0, 0, 1), bp.BP_EINVAL), ((4, (1 << 20) + 1, 0, 1), bp.BP_EINVAL),
                                         ((4, 8, 2, 1), bp.BP_EINVAL), ((4, 8, 0, 0), bp.BP_EINVAL),
                                         ((4, 8, 0, (1 << 26) + 1), bp.BP_EINVAL), ((4, 12, 1, 1), bp.BP_ESHAPE)])
def test_embedding_create_refuses(lib, args, status):
    out = ctypes.c_void_p()
    assert lib.bp_embedding_create(*args, ctypes.byref(out)) == status
    assert out.value is None and lib.bp_last_error()
    assert lib.bp_embedding_create(4, 8, 0, 1, None) == bp.BP_EINVAL


def test_null_embeddings_are_refused(lib):
    assert lib.bp_embed(None, P, P, 1, 1.0, P, None) == bp.BP_EINVAL
    assert lib.bp_embed_backward(None, P, 1, P, 1.0, P, 0, None) == bp.BP_EINVAL
    assert lib.bp_embedding_check(None, None) == bp.BP_EINVAL
    lib.bp_embedding_destroy(None)   # NULL-safe


# ------------------------------------------------------------------ residual stream
@pytest.mark.parametrize("out", [0, 1, 2])
@pytest.mark.parametrize("into", [0, 1, 2])
def test_residual_gradient_is_the_difference(out, into):
    rng = np.random.default_rng(out * 3 + into)
    n, w, eps, scale = 6, 5, 1e-3, 0.7
    v = dict(X=rng.standard_normal((n, w)), F=rng.standard_normal((n, w)) + 1, gate=rng.standard_normal((3, w)))
    if out:
        v["wo"] = rng.standard_normal(w)
    if out == 2:
        v["bo"] = rng.standard_normal(w)
    if into:
        v["wi"] = rng.standard_normal(w)
    if into == 2:
        v["bi"] = rng.standard_normal(w)
    off = np.array([0, 2, 2, 5])   # an empty range, and a row of none
    dY, dH = rng.standard_normal((n, w)), rng.standard_normal((n, w)) if into else None

    def forward():
        y = O.residual(v["X"], v["F"], v.get("wo"), v.get("bo"), v["gate"], off, scale, out, eps)[0]
        return y, O.norm_in(y, v.get("wi"), v.get("bi"), into, eps)[0] if into else 0.0

    def loss():
        y, h = forward()
        return (y * dY).sum() + ((h * dH).sum() if into else 0.0)
    got = O.residual_backward(forward()[0], v["F"], v.get("wo"), v.get("bo"), v["gate"], off, scale, v.get("wi"), dY, dH, out, into, eps)
    for name, x in v.items():
        g, mag = got["d" + name if name in "XF" else "G" + name]
        np.testing.assert_allclose(g, difference(loss, x), atol=2e-8, err_msg=name)
        assert (mag >= np.abs(g) - 1e-12).all()


@pytest.mark.parametrize("args,status", [((0, 0, 4, 1, 1, 1, 1e-5), bp.BP_EINVAL), ((8193, 0, 4, 1, 1, 1, 1e-5), bp.BP_EINVAL),
                                         ((12, 1, 4, 1, 1, 1, 1e-5), bp.BP_ESHAPE), ((8, 3, 4, 1, 1, 1, 1e-5), bp.BP_EINVAL),
                                         ((8, 0, 0, 1, 1, 1, 1e-5), bp.BP_EINVAL), ((8, 0, 2 ** 31 - 1, 1, 1, 1, 1e-5), bp.BP_EINVAL),
                                         ((8, 0, 4, -1, 1, 1, 1e-5), bp.BP_EINVAL), ((8, 0, 4, 1, 3, 1, 1e-5), bp.BP_EINVAL),
                                         ((8, 0, 4, 1, 1, -1, 1e-5), bp.BP_EINVAL), ((8, 0, 4, 1, 1, 1, 0.0), bp.BP_EINVAL),
                                         ((8, 0, 4, 1, 1, 1, float("nan")), bp.BP_EINVAL),
                                         ((8, 0, 4, 1, 1, 1, float("inf")), bp.BP_EINVAL)])
def test_residual_create_refuses(lib, args, status):
    out = ctypes.c_void_p()
    assert lib.bp_residual_create(*args, ctypes.byref(out)) == status
    assert out.value is None and lib.bp_last_error()
    assert lib.bp_residual_create(8, 0, 4, 1, 1, 1, 1e-5, None) == bp.BP_EINVAL


def test_null_streams_are_refused(lib):
    assert lib.bp_residual_forward(None, P, P, 1, P, P, P, P, 1, 1.0, P, P, P, P, P, None) == bp.BP_EINVAL
    assert lib.bp_residual_backward(None, P, P, 1, P, P, P, P, 1, 1.0, P, P, P, P, P, P, P, P, P, P, P, 0, None) == bp.BP_EINVAL
    assert lib.bp_residual_check(None, None) == bp.BP_EINVAL
    lib.bp_residual_destroy(None)   # NULL-safe


# ------------------------------------------------------------------ clipping
def test_clip_oracle():
    norm, out = O.clip([np.array([3.0, 0.0]), np.zeros(0), np.array([[-4.0]])], 2.5)
    assert norm == 5.0 and [x.tolist() for x in out] == [[1.5, 0.0], [], [[-2.0]]]
    norm, out = O.clip([np.array([3.0, 4.0]) * 2.0 ** 120], np.inf)
    assert norm == 5 * 2.0 ** 120 and out[0].tolist() == [3 * 2.0 ** 120, 2.0 ** 122]


def clip_create(lib, ins, outs, sizes, dtypes, n=None):
    out = ctypes.c_void_p()
    k = len(ins)
    st = lib.bp_clip_create((ctypes.c_void_p * k)(*ins), None if outs is None else (ctypes.c_void_p * k)(*outs),
                            (ctypes.c_int64 * k)(*sizes), (ctypes.c_int * k)(*dtypes), k if n is None else n, ctypes.byref(out))
    assert out.value is None
    return st, lib.bp_last_error().decode()


@pytest.mark.parametrize("ins,outs,sizes,dtypes,word", [
    ([P], None, [4], [2], "dtype"), ([P], None, [-1], [0], "size"), ([P], None, [2 ** 41], [0], "size"),
    ([P, P << 20], None, [2 ** 40, 1], [1, 1], "sum"), ([None], None, [1], [0], "NULL"), ([P + 2], None, [1], [0], "aligned"),
    ([P + 1], None, [1], [1], "aligned"), ([P], [P + 0x1002], [1], [0], "aligned"), ([P], [None], [1], [0], "NULL"),
    ([P, P + 12], None, [4, 4], [0, 0], "overlap"), ([P, P + 4096], [P + 8192, P + 8200], [4, 4], [0, 0], "overlap"),
    ([P], [P + 4], [4], [0], "overlaps"), ([P + 4], [P], [4], [0], "overlaps"),
    ([P, P + 4096], [P + 4096, P + 8192], [4, 4], [0, 0], "overlaps"), ([P, P + 16], [P, P + 8], [4, 4], [0, 1], "overlap"),
    ([P, P, P + 4096], [P, P + 8192, P + 4096], [4, 4, 1], [0, 0, 0], "overlaps")])
def test_clip_create_refuses(lib, ins, outs, sizes, dtypes, word):
    st, message = clip_create(lib, ins, outs, sizes, dtypes)
    assert st == bp.BP_EINVAL and word in message, message


def test_clip_numbers_of_tensors(lib):
    for n in (0, -1, 65536):
        assert clip_create(lib, [P], None, [1], [0], n)[0] == bp.BP_EINVAL
    out = ctypes.c_void_p()
    assert lib.bp_clip_create(None, None, None, None, 1, ctypes.byref(out)) == bp.BP_EINVAL
    assert lib.bp_clip_run(None, 1.0, P, None) == bp.BP_EINVAL
    assert lib.bp_clip_check(None, None) == bp.BP_EINVAL
    lib.bp_clip_destroy(None)   # NULL-safe
