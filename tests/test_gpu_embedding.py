"""Embeddings against the float64 oracle.

A row of the lookup is rounded to float32 and, for bfloat16, once more: 2^-24 and 2^-8 of itself.  A change of a
token with m ids is a chain of at most 32 additions to a piece, of m / 32 + 2 pieces, with the scale and what
was there before behind it: 2^-24 of the magnitudes for each, (40 + m / 32) * 2^-24 in all.
"""
import numpy as np
import pytest

from expert_cases import BF16, dev, empty, host, rounded
from oracle import blocks_oracle as O
from paper_1801_01554_gb300 import bp

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32 = 2.0 ** -24


def check(ids, V, width, dtype, scale, got_y, got_g, table, D, before=None):
    half = F32 + (BF16 if dtype == bp.BP_BF16 else 0.0)
    want = O.embed(table, ids, scale)
    assert (np.abs(host(got_y) - want) <= half * np.abs(want) + 1e-37).all()
    want, mag = O.embed_backward(ids, D, scale, V)
    if before is not None:
        want, mag = want + before, mag + np.abs(before)
    m = np.bincount(ids[(ids >= 0) & (ids < V)], minlength=V)[:, None]
    assert (np.abs(host(got_g) - want) <= (40 + m / 32) * F32 * mag + 1e-37).all()


def make(rng, kind, n, V):
    if kind == "one":
        return np.full(n, V // 2, dtype=np.int32)
    if kind == "runs":   # lengths around the tiles' 32, in shuffled order
        ids = np.repeat(np.arange(V), rng.choice([0, 1, 2, 15, 31, 32, 33, 34, 63, 64, 65, 100], size=V))[:n]
        ids = np.concatenate([ids, np.full(n - len(ids), V - 1)])
        return rng.permutation(ids).astype(np.int32)
    ids = rng.integers(0, V, size=n)
    if kind == "holes":
        ids[rng.random(n) < 0.3] = -1
    return ids.astype(np.int32)


@pytest.mark.parametrize("dtype,width", [(bp.BP_F32, 1), (bp.BP_F32, 15), (bp.BP_F32, 64), (bp.BP_F32, 133), (bp.BP_F32, 516),
                                         (bp.BP_BF16, 8), (bp.BP_BF16, 264), (bp.BP_BF16, 2056)])
@pytest.mark.parametrize("kind,n,V", [("any", 0, 5), ("any", 1, 1), ("any", 1, 300), ("any", 31, 7), ("one", 32, 3), ("one", 33, 3),
                                      ("one", 65, 1), ("holes", 96, 40), ("holes", 1000, 511), ("runs", 1500, 60),
                                      ("runs", 4096, 200)])
def test_embedding_matches_oracle(kind, n, V, width, dtype):
    rng = np.random.default_rng([n, V, width])
    ids = make(rng, kind, n, V)
    table, D = rounded(rng.standard_normal((V, width)), dtype), rounded(rng.standard_normal((n, width)), dtype)
    Y, G = empty((n, width), dtype), empty((V, width), bp.BP_F32)
    td, dd, idd = dev(table, dtype), dev(D, dtype), dev(ids)
    with bp.Embedding(V, width, dtype, max_ids=n + 5) as layer:
        layer.forward(td, idd, n, Y, scale=1.75)
        layer.backward(idd, n, dd, G, scale=1.75)
        layer.check()
        check(ids, V, width, dtype, 1.75, Y, G, table, D)


@pytest.mark.parametrize("dtype,width", [(bp.BP_F32, 9), (bp.BP_F32, 128), (bp.BP_BF16, 256), (bp.BP_BF16, 264)])
@pytest.mark.parametrize("kind,n,V", [("any", 4096, 1088), ("holes", 4096, 1089), ("runs", 4095, 544), ("any", 1000, 314),
                                      ("any", 1000, 315), ("any", 9, 66), ("one", 9, 67)])
def test_either_side_of_a_block_a_token(kind, n, V, width, dtype):
    """Calls with as many tokens as a block a token is taken for, and one more; once over what was there."""
    rng = np.random.default_rng([n, V, width, 5])
    ids = make(rng, kind, n, V)
    table, D = rounded(rng.standard_normal((V, width)), dtype), rounded(rng.standard_normal((n, width)), dtype)
    Y, G, twice = empty((n, width), dtype), empty((V, width), bp.BP_F32), empty((V, width), bp.BP_F32)
    td, dd, idd = dev(table, dtype), dev(D, dtype), dev(ids)
    with bp.Embedding(V, width, dtype, max_ids=n) as layer:
        layer.forward(td, idd, n, Y, scale=1.75)
        layer.backward(idd, n, dd, G, scale=1.75)
        layer.backward(idd, n, dd, twice, scale=1.75)
        layer.backward(idd, n, dd, twice, scale=1.75, accumulate=True)
        layer.check()
        check(ids, V, width, dtype, 1.75, Y, G, table, D)
    assert torch.equal(twice, G * 2)


@pytest.mark.parametrize("dtype,width", [(bp.BP_F32, 9), (bp.BP_BF16, 16)])
@pytest.mark.parametrize("kind,n,V", [("any", 70001, 1 << 18), ("one", 40000, 1 << 24), ("runs", 9000, 400), ("holes", 5000, 1000)])
def test_long_lists_and_wide_tokens(kind, n, V, width, dtype):
    """More ids than one block sorts, tokens of three passes, one run over every tile; the changes that were there are kept."""
    if V == 1 << 24:
        width = 1 if dtype == bp.BP_F32 else 8
    rng = np.random.default_rng([n, 1])
    ids = make(rng, kind, n, V)
    D = rounded(rng.standard_normal((n, width)), dtype)
    dd, idd = dev(D, dtype), dev(ids)
    used, where = np.unique(ids[ids >= 0], return_inverse=True)
    with bp.Embedding(V, width, dtype, max_ids=n) as layer:
        G = empty((V, width), bp.BP_F32)
        layer.backward(idd, n, dd, G, scale=0.5)
        again = empty((V, width), bp.BP_F32)
        layer.backward(idd, n, dd, again, scale=0.5)
        assert torch.equal(G, again)
        del again
        want, mag = O.embed_backward(where, D[ids >= 0], 0.5, len(used))
        m = np.bincount(where, minlength=len(used))[:, None]
        ud = torch.tensor(used, device="cuda")
        assert (np.abs(host(G[ud]) - want) <= (40 + m / 32) * F32 * mag + 1e-37).all()
        rest = torch.ones(V, dtype=torch.bool, device="cuda")
        rest[ud] = False
        assert (G[rest] == 0).all()
        G.fill_(3.0)
        layer.backward(idd, n, dd, G, scale=0.5, accumulate=True)
        layer.check()
        assert (np.abs(host(G[ud]) - want - 3.0) <= (40 + m / 32) * F32 * (mag + 3.0)).all()
        assert (G[rest] == 3.0).all()


def test_ids_outside_the_table_are_zeros_and_reported():
    V, width, n = 10, 24, 70
    rng = np.random.default_rng(2)
    ids = rng.integers(0, V, size=n).astype(np.int32)
    table, D = rounded(rng.standard_normal((V, width)), bp.BP_BF16), rounded(rng.standard_normal((n, width)), bp.BP_BF16)
    with bp.Embedding(V, width, bp.BP_BF16, max_ids=n) as layer:
        for bad in (V, -2, 2 ** 31 - 1, -2 ** 31):
            ids[17] = bad
            Y, G = empty((n, width), bp.BP_BF16), empty((V, width), bp.BP_F32)
            layer.forward(dev(table, bp.BP_BF16), dev(ids), n, Y)
            with pytest.raises(bp.BPError) as e:
                layer.check()
            assert e.value.status == bp.BP_ESTATE and "id" in str(e.value)
            layer.check()
            layer.backward(dev(ids), n, dev(D, bp.BP_BF16), G)
            with pytest.raises(bp.BPError):
                layer.check()
            check(ids, V, width, bp.BP_BF16, 1.0, Y, G, table, D)
        ids[17] = -1   # an empty place
        layer.forward(dev(table, bp.BP_BF16), dev(ids), n, Y)
        layer.check()
        assert (Y[17] == 0).all()


def test_float_rows_off_16_bytes():
    V, width, n = 7, 64, 50
    rng = np.random.default_rng(4)
    ids = rng.integers(0, V, size=n).astype(np.int32)
    table, D = rounded(rng.standard_normal((V, width)), bp.BP_F32), rounded(rng.standard_normal((n, width)), bp.BP_F32)

    def off(x=None, shape=None):
        b = torch.full((int(np.prod(shape or x.shape)) + 1,), float("nan"), device="cuda")
        if x is not None:
            b[1:] = dev(x).view(-1)
        return b[1:]
    t, d, Y, G = off(table), off(D), off(shape=(n, width)), off(shape=(V, width))
    with bp.Embedding(V, width, bp.BP_F32, max_ids=n) as layer:
        layer.forward(t, dev(ids), n, Y)
        layer.backward(dev(ids), n, d, G)
        check(ids, V, width, bp.BP_F32, 1.0, Y.view(n, width), G.view(V, width), table, D)


def test_replayed_with_other_ids():
    """One graph of both directions on a side stream, replayed for other ids and rows, then a direct call."""
    V, width, n, dtype = 321, 72, 900, bp.BP_BF16
    rng = np.random.default_rng(8)
    table = rounded(rng.standard_normal((V, width)), dtype)
    td, idd, dd = dev(table, dtype), dev(np.zeros(n, dtype=np.int32)), empty((n, width), dtype, 0.0)
    Y, G = empty((n, width), dtype), empty((V, width), bp.BP_F32)
    with bp.Embedding(V, width, dtype, max_ids=n) as layer:
        s = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            layer.forward(td, idd, n, Y, scale=2.0, stream=s)
            layer.backward(idd, n, dd, G, scale=2.0, stream=s)
        for i in range(4):
            ids = make(rng, ("any", "one", "runs", "holes")[i], n, V)
            D = rounded(rng.standard_normal((n, width)), dtype)
            idd.copy_(dev(ids))
            dd.copy_(dev(D, dtype))
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                graph.replay()
            s.synchronize()
            check(ids, V, width, dtype, 2.0, Y, G, table, D)
            first = G.clone()
            torch.cuda.synchronize()
            layer.backward(idd, n, dd, G, scale=2.0, stream=s)
            layer.check(s)
            assert torch.equal(first, G)
        del graph


def test_embedding_refuses():
    with bp.Embedding(10, 16, bp.BP_BF16, max_ids=4) as layer:
        t, y, i = torch.zeros(10, 16, device="cuda").bfloat16(), torch.zeros(5, 16, device="cuda").bfloat16(), dev(np.zeros(5, int))
        g = torch.zeros(10, 16, device="cuda")
        for call in (lambda: layer.forward(t, i, 5, y), lambda: layer.forward(t, i, -1, y), lambda: layer.backward(i, 5, y, g)):
            with pytest.raises(bp.BPError) as e:
                call()
            assert e.value.status == bp.BP_EINVAL and "n must be" in str(e.value)
        for x in (float("nan"), float("inf")):
            with pytest.raises(bp.BPError) as e:
                layer.forward(t, i, 4, y, scale=x)
            assert e.value.status == bp.BP_EINVAL and "scale" in str(e.value)
        with pytest.raises(bp.BPError) as e:
            layer.forward(t.view(-1)[1:].data_ptr(), i, 4, y)
        assert e.value.status == bp.BP_EINVAL and "d_table" in str(e.value)
        with pytest.raises(bp.BPError) as e:
            layer.backward(i, 4, y, None)
        assert e.value.status == bp.BP_EINVAL and "d_G" in str(e.value)
        for call in (lambda: layer.forward(t[:9], i, 4, y), lambda: layer.forward(t, i.long(), 4, y),
                     lambda: layer.forward(t.float(), i, 4, y), lambda: layer.backward(i, 4, y, g[:9]),
                     lambda: layer.backward(i, 4, y[:3], g), lambda: layer.backward(i[:3], 4, y, g)):
            with pytest.raises(ValueError):
                call()
        layer.check()
