"""Routers, embeddings and clipping at sizes where another way is taken: ids that the sort does not hold in registers, chunks of
more values than a block takes at a time, patterns on either side of the order's launches and of a warp's share.

Bounds: those of test_gpu_clip and test_gpu_scored_router; a token's changes as test_gpu_embedding_long has them, 160 * 2^-24.
"""
import numpy as np
import pytest

import test_gpu_router as R
import test_gpu_scored_router as S
from expert_cases import BF16, dev, empty, host, rounded
from paper_1801_01554_gb300 import bp

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32 = 2.0 ** -24


# ------------------------------------------------------------ ids
def ids_of(rng, kind, n, V):
    ids = np.full(n, V - 1) if kind == "one" else rng.integers(0, V, size=n)
    if kind == "skewed":
        ids[rng.random(n) < 0.3] = V // 2
    if kind != "one":
        ids[rng.random(n) < 0.1] = -1
    return ids.astype(np.int32)


def change(ids, D, V, scale):
    """The change in 64 bits, and its magnitude."""
    live = ids >= 0
    G, mag = ([np.bincount(ids[live], weights=f(D[live, c]), minlength=V) for c in range(D.shape[1])] for f in (lambda x: x, np.abs))
    return scale * np.stack(G, 1), abs(scale) * np.stack(mag, 1)


@pytest.mark.parametrize("dtype,width", [(bp.BP_F32, 1), (bp.BP_BF16, 8)])
@pytest.mark.parametrize("V", [6, 1000, 300_000])   # one, two and three passes
@pytest.mark.parametrize("kind", ["any", "skewed", "one"])
@pytest.mark.parametrize("n", [131_072, 131_073, 300_001])
def test_more_ids_than_the_sort_holds(n, kind, V, dtype, width):
    rng = np.random.default_rng([n, V])
    ids, D = ids_of(rng, kind, n, V), rounded(rng.standard_normal((n, width)), dtype)
    G, again, idd, dd = empty((V, width), bp.BP_F32), empty((V, width), bp.BP_F32), dev(ids), dev(D, dtype)
    want, mag = change(ids, D, V, -0.5)
    with bp.Embedding(V, width, dtype, max_ids=n) as layer:
        layer.backward(idd, n, dd, G, scale=-0.5)
        layer.backward(idd, n, dd, again, scale=-0.5)
        layer.check()
        assert torch.equal(G, again)
        assert (np.abs(host(G) - want) <= 160 * F32 * mag).all()
        G.fill_(2.0)
        layer.backward(idd, n, dd, G, scale=-0.5, accumulate=True)
        layer.check()
        assert (np.abs(host(G) - want - 2.0) <= 160 * F32 * (mag + 2.0)).all()
        idd[n // 2] = V   # names no token
        layer.backward(idd, n, dd, G)
        with pytest.raises(bp.BPError) as e:
            layer.check()
        assert e.value.status == bp.BP_ESTATE


@pytest.mark.parametrize("n", [9000, 140_000])
def test_lists_one_after_another(n):
    """Calls behind one another on a stream, with other ids each, and nothing between them that waits."""
    V, width, rng = 20_000, 8, np.random.default_rng(n)
    lists = [ids_of(rng, kind, n, V) for kind in ("any", "skewed", "one", "any")]
    D = rounded(rng.standard_normal((n, width)), bp.BP_BF16)
    idd, dd, out = [dev(x) for x in lists], dev(D, bp.BP_BF16), [empty((V, width), bp.BP_F32) for _ in range(12)]
    with bp.Embedding(V, width, bp.BP_BF16, max_ids=n) as layer:
        for i, G in enumerate(out):
            layer.backward(idd[i % 4], n, dd, G)
        layer.check()
    for i, G in enumerate(out):
        want, mag = change(lists[i % 4], D, V, 1.0)
        assert (np.abs(host(G) - want) <= 160 * F32 * mag).all()


# ------------------------------------------------------------ clipping
@pytest.mark.parametrize("in_place", [True, False])
def test_chunks_of_several_tiles(in_place):
    """2^29 values and some: chunks are longer than a tile from there on.  Tensors off 16 bytes, and two types."""
    g = torch.Generator(device="cuda").manual_seed(4)
    large = torch.empty(2 ** 29 + 8, dtype=torch.bfloat16, device="cuda")
    for part in large.split(2 ** 27):
        part.copy_(torch.randn(part.numel(), generator=g, device="cuda"))
    x = [large[3:], torch.randn(2 ** 20 + 5, generator=g, device="cuda")[1:]]
    before = [t.clone() for t in x]
    outs = None if in_place else [torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")[1:] for t in x]
    want = sum(float(p.double().square().sum()) for t in x for p in t.split(2 ** 26)) ** 0.5
    norm = torch.zeros(1, device="cuda")
    with bp.Clip(x, outs) as clip:
        clip.run(float("inf"), norm)
        clip.check()
        assert abs(float(norm) - want) <= 18 * F32 * want
        clip.run(want / 8, norm)   # (want / 8 as float32 has it: within 2^-24 of itself)
        clip.check()
    assert abs(float(norm) - want) <= 18 * F32 * want
    for t, b in zip(x if in_place else outs, before):
        half = BF16 if t.dtype == torch.bfloat16 else 0.0
        for p, q in zip(t.split(2 ** 26), b.split(2 ** 26)):
            w = q.double() / 8
            assert bool(((p.double() - w).abs() <= (21 * F32 + half) * w.abs() + 1e-38).all())
    if not in_place:
        assert all(torch.equal(t, b) for t, b in zip(x, before))


# ------------------------------------------------------------ routers
@pytest.mark.parametrize("n", [64, 65, 2047, 2048, 2049])
@pytest.mark.parametrize("dtype", [bp.BP_F32, bp.BP_BF16])
def test_patterns_either_side_of_the_orders_launches(n, dtype):
    E, k, rng = 70, 5, np.random.default_rng(n)
    z = rounded(rng.standard_normal((n, E)) + rng.standard_normal(E), dtype)
    z[rng.random(z.shape) < 0.1] = -np.inf
    dgate = rounded(rng.standard_normal((n, k)), bp.BP_F32)
    R.check(z, k, "chosen", dtype, dgate)
    bias = rounded(rng.standard_normal(E) * 0.1, bp.BP_F32)
    S.check(z, bias, k, dtype, "sigmoid", dgate, 7, 3, 2, True)
    S.check(z, bias, k, dtype, "softmax", dgate, 7, 3, 1, False)


@pytest.mark.parametrize("dtype", [bp.BP_F32, bp.BP_BF16])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("n,E,k,G,open_,top", [
    (6007, 256, 8, 8, 4, 2), (5001, 512, 16, 1, 1, 1), (5001, 493, 3, 17, 4, 2), (5003, 31, 2, 1, 1, 1), (5003, 128, 4, 1, 1, 1),
    (5002, 64, 6, 8, 3, 2)])
def test_more_patterns_than_warps_for_them(n, E, k, G, open_, top, kind, dtype):
    rng = np.random.default_rng([n, E, k])
    z = rounded(rng.standard_normal((n, E)) * 1.5 + rng.standard_normal(E), dtype)
    z[rng.random(z.shape) < 0.05] = -np.inf
    if dtype == bp.BP_F32:   # some that float32 scores cannot tell apart
        z[::7] = rounded(0.75 + rng.integers(0, 40, size=z[::7].shape) * 2.0 ** -24, bp.BP_F32)
    z[11], z[n - 1] = -np.inf, 0.0
    bias, dgate = rounded(rng.standard_normal(E) * 0.1, bp.BP_F32), rounded(rng.standard_normal((n, k)), bp.BP_F32)
    S.check(z, bias, k, dtype, kind, dgate, G, open_, top, True, 2.5)
    S.check(z, None, k, dtype, kind, dgate, G, open_, top, False)
