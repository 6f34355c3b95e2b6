"""Embeddings, residual stream and clipping at their edges: nothing to do, more ranges than rows, each path of the changes of a
table for the same ids, and long lists replayed.  Bounds: those of test_gpu_embedding, test_gpu_residual and test_gpu_clip."""
import numpy as np
import pytest

from expert_cases import dev, empty, host, rounded
from oracle import blocks_oracle as O
from paper_1801_01554_gb300 import bp

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32 = 2.0 ** -24


def close(got, ids, D, scale, V):
    want, mag = O.embed_backward(ids, D, scale, V)
    m = np.bincount(ids[(ids >= 0) & (ids < V)], minlength=V)[:, None]
    assert (np.abs(host(got) - want) <= (40 + m / 32) * F32 * mag + 1e-37).all()


@pytest.mark.parametrize("n", [10, 1000, 6000])
@pytest.mark.parametrize("V", [20, 3000])
def test_only_empty_places(n, V):
    ids = dev(np.full(n, -1, dtype=np.int32))
    D, G, Y, table = (torch.ones(s, 16, device="cuda") for s in (n, V, n, V))
    with bp.Embedding(V, 16, bp.BP_F32, max_ids=n) as layer:
        layer.backward(ids, n, D, G, accumulate=True)
        layer.forward(table, ids, n, Y)
        layer.check()
        assert (G == 1).all() and (Y == 0).all()
        layer.backward(ids, n, D, G)
        layer.check()
        assert (G == 0).all()


@pytest.mark.parametrize("dtype,width", [(bp.BP_F32, 33), (bp.BP_F32, 256), (bp.BP_BF16, 520)])
@pytest.mark.parametrize("n", [4095, 4096, 4097, 9000])
@pytest.mark.parametrize("V", [3, 60, 255, 257, 5000])
def test_every_path_of_the_changes(n, V, width, dtype):
    """Either side of the sizes where another kernel takes over; a token with a third of the ids, tokens with none."""
    rng = np.random.default_rng([n, V])
    ids = rng.integers(0, V, size=n).astype(np.int32)
    ids[rng.random(n) < 0.33] = V // 2
    ids[rng.random(n) < 0.05] = -1
    D = rounded(rng.standard_normal((n, width)), dtype)
    G, again = empty((V, width), bp.BP_F32), empty((V, width), bp.BP_F32)
    idd, dd = dev(ids), dev(D, dtype)
    with bp.Embedding(V, width, dtype, max_ids=n) as layer:
        layer.backward(idd, n, dd, G, scale=0.5)
        layer.backward(idd, n, dd, again, scale=0.5)
        layer.check()
        assert torch.equal(G, again)
        close(G, ids, D, 0.5, V)
        layer.backward(idd, n, dd, again, scale=0.5, accumulate=True)
        torch.cuda.synchronize()
        assert (np.abs(host(again) - 2 * host(G)) <= 2 * F32 * np.abs(host(G)) * 2 + 1e-37).all()


def test_a_long_list_replayed():
    n, V, width, rng = 9000, 700, 40, np.random.default_rng(3)
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    idd, dd, G = dev(np.zeros(n, dtype=np.int32)), empty((n, width), bp.BP_BF16, 0.0), empty((V, width), bp.BP_F32)
    with bp.Embedding(V, width, bp.BP_BF16, max_ids=n) as layer:
        with torch.cuda.graph(graph, stream=s):
            layer.backward(idd, n, dd, G, stream=s)
        for _ in range(3):
            ids, D = rng.integers(-1, V, size=n).astype(np.int32), rounded(rng.standard_normal((n, width)), bp.BP_BF16)
            idd.copy_(dev(ids))
            dd.copy_(dev(D, bp.BP_BF16))
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                graph.replay()
            s.synchronize()
            close(G, ids, D, 1.0, V)
        layer.check(s)
        del graph


def test_more_ranges_of_gates_than_rows():
    n, width, gates, rng = 5, 48, 300, np.random.default_rng(4)
    offsets = np.sort(np.concatenate([[0, n], rng.integers(0, n + 1, size=gates - 1)])).astype(np.int32)
    X, F, dY = (rounded(rng.standard_normal((n, width)), bp.BP_F32) for _ in range(3))
    gate = rounded(rng.standard_normal((gates, width)), bp.BP_F32)
    Y, st, G = empty((n, width), bp.BP_F32), empty((n, 4), bp.BP_F32), empty((gates, width), bp.BP_F32)
    k = dict(gate=dev(gate), offsets=dev(offsets), n_gates=gates, scale=1.0)
    with bp.Residual(width, bp.BP_F32, n, O.RMS, O.NONE, 1e-5, max_gates=gates) as layer:
        layer.forward(dev(X), dev(F), n, Y, None, st, **k)
        layer.backward(None, dev(F), n, st, dev(dY), None, Ggate=G, **k)
        layer.check()
    want, mag = O.residual(X, F, None, None, gate, offsets, 1.0, O.RMS, 1e-5)
    assert (np.abs(host(Y) - want) <= 2.0 ** -18 * (mag + np.abs(X))).all()
    want, mag = O.residual_backward(Y.cpu().double().numpy(), F, None, None, gate, offsets, 1.0, None, dY, None, O.RMS, O.NONE, 1e-5)["Ggate"]
    assert (np.abs(host(G) - want) <= 2.0 ** -16 * mag + 1e-37).all()


def test_clipping_nothing():
    norm, none = torch.ones(1, device="cuda"), torch.zeros(0, device="cuda")
    with bp.Clip([none, none]) as clip:
        clip.run(0.0, norm)
        clip.check()
        assert float(norm) == 0.0


def test_many_small_changes():
    """Many chunks of a few values each, in place, with a bound just below and just above the norm."""
    x = torch.randn(3000, generator=torch.Generator().manual_seed(1)).cuda()
    pieces = [x[i:i + 3] for i in range(0, 3000, 3)]
    want = x.double().norm().item()
    before = x.clone()
    with bp.Clip(pieces) as clip:
        clip.run(want * 1.001)
        clip.check()
        assert torch.equal(x, before)
        clip.run(want * 0.5)
        clip.check()
    assert (x - before * 0.5).abs().max().item() <= 40 * F32 * before.abs().max().item()
