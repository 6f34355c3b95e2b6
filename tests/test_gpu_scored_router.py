"""The router by scores against the float64 oracle.

Choices, offsets, sources and places are whole numbers and must be equal.  A gate: expf (two units), its argument, a difference d
(half a unit of it, above and below the line), a sum of at most 32 + 5 additions, a quotient or two: 2^-18 + |d| 2^-23 of itself, d at
most 104 (beyond that it vanishes).  A gradient is at most two of these and as many products: twice that of its terms' magnitudes.
"""
import numpy as np
import pytest

from expert_cases import BF16, dev, empty, host, rounded
from oracle import experts_oracle as O
from paper_1801_01554_gb300 import bp

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

KINDS = {"softmax": bp.BP_SCORES_SOFTMAX, "sigmoid": bp.BP_SCORES_SIGMOID}
NAMES = ("expert", "gate", "offsets", "source", "place")


def outputs(n, E, k):
    return [torch.full(shape, 99, dtype=t, device="cuda") for shape, t in
            (((n, k), torch.int32), ((n, k), torch.float32), ((E + 1,), torch.int32), ((n * k,), torch.int32), ((n, k), torch.int32))]


def check(z, bias, k, dtype, kind, dgate=None, n_groups=1, open_groups=1, group_top=1, renormalise=False, scale=1.0):
    n, E = z.shape
    out, zd, dz = outputs(n, E, k), dev(z, dtype), empty((n, E), dtype)
    with bp.ScoredRouter(E, k, dtype, max(n, 1), KINDS[kind], n_groups, open_groups, group_top, renormalise, scale) as r:
        r.forward(zd, dev(bias), n, *out)
        if dgate is not None:
            r.backward(zd, n, out[0], dev(dgate), dz)
        torch.cuda.synchronize()
    want = O.route_scored(z, bias, k, kind, n_groups, open_groups, group_top, renormalise, scale)
    for i in (0, 2, 3, 4):
        np.testing.assert_array_equal(out[i].cpu().numpy(), want[i], err_msg=NAMES[i])
    open_ = np.where(z > -np.inf, z, np.nan)
    with np.errstate(all="ignore"):
        import warnings
        with warnings.catch_warnings():
            warnings.simplefilter("ignore")
            d = np.nan_to_num(np.nanmax(open_, 1) - np.nanmin(open_, 1), posinf=104.0, nan=0.0).clip(0, 104)[:, None]
    tol = 2.0 ** -18 + d * 2.0 ** -23
    got = host(out[1])
    assert (np.isnan(got) == np.isnan(want[1])).all()
    assert (np.abs(got - want[1]) <= tol * np.abs(want[1]) + 1e-37)[~np.isnan(got)].all()
    if dgate is not None:
        want, mag = O.route_scored_backward(z, want[0], dgate, kind, renormalise, scale)
        half = BF16 if dtype == bp.BP_BF16 else 0.0
        assert (np.abs(host(dz) - want) <= half * np.abs(want) + 2 * tol * mag + 1e-37).all()
    return out


@pytest.mark.parametrize("dtype", [bp.BP_F32, bp.BP_BF16])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
@pytest.mark.parametrize("n,E,k,G,open_,top", [
    (1, 1, 1, 1, 1, 1), (1, 64, 6, 8, 3, 2), (5, 3, 3, 3, 3, 2), (33, 8, 4, 4, 2, 1), (256, 60, 4, 12, 5, 1), (257, 60, 8, 12, 5, 2),
    (300, 512, 16, 1, 1, 1), (300, 512, 16, 32, 2, 2), (129, 493, 3, 17, 4, 2), (700, 256, 8, 8, 4, 2), (90, 510, 5, 5, 2, 1),
    (4100, 40, 4, 1, 1, 1), (64, 32, 2, 32, 2, 2), (1000, 100, 7, 10, 1, 1)])
def test_choices_match_oracle(n, E, k, G, open_, top, kind, renormalise, dtype):
    rng = np.random.default_rng([n, E, k, G])
    z = rounded(rng.standard_normal((n, E)) * 1.5 + rng.standard_normal(E), dtype)
    z[rng.random(z.shape) < 0.05] = -np.inf
    bias = rounded(rng.standard_normal(E) * 0.1, bp.BP_F32)
    dgate = rounded(rng.standard_normal((n, k)), bp.BP_F32)
    check(z, bias, k, dtype, kind, dgate, G, open_, top, renormalise, 2.5)
    if E <= 100:
        check(z, None, k, dtype, kind, dgate, G, open_, top, renormalise)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("G,open_,top", [(1, 1, 1), (4, 2, 1), (4, 2, 2)])
def test_scores_that_float32_cannot_tell_apart(kind, G, open_, top):
    """Logits a unit of float32 apart, biases that shift by as little, ties, and biases that nearly cancel the
    scores: the choice is float64's."""
    rng = np.random.default_rng(11)
    n, E, k = 400, 48, 6
    z = (np.float32(0.75) + rng.integers(0, 40, size=(n, E)).astype(np.float32) * np.float32(2.0 ** -24)).astype(np.float64)
    z[::3] = 0.75 + rng.integers(0, 3, size=z[::3].shape) * 2.0 ** -23
    for bias in (None, np.zeros(E), rounded(rng.integers(0, 3, size=E) * 2.0 ** -27, bp.BP_F32), rounded(-1 / (1 + np.exp(-z[0])), bp.BP_F32),
                 np.full(E, -2.0 ** 30), rounded(rng.integers(0, 2, size=E) * 1e30, bp.BP_F32)):
        check(z, bias, k, bp.BP_F32, kind, None, G, open_, top, True)


@pytest.mark.parametrize("dtype", [bp.BP_F32, bp.BP_BF16])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
@pytest.mark.parametrize("G,open_,top", [(1, 1, 1), (6, 2, 2)])
def test_closed_experts_and_extreme_logits(kind, renormalise, G, open_, top, dtype):
    low = -3.3895313892515355e38 if dtype == bp.BP_BF16 else -float(np.finfo(np.float32).max)
    rng = np.random.default_rng(5)
    n, E, k = 300, 24, 4
    z = rounded(rng.integers(-2, 3, size=(n, E)).astype(float), dtype)   # many ties
    z[rng.random(z.shape) < 0.5] = -np.inf
    z[3], z[150], z[9], z[12], z[20], z[21] = -np.inf, -np.inf, low, low, -low, -100.0
    z[7], z[7, 5] = 0.0, -0.0
    z[11], z[11, 13] = -np.inf, low
    z[12, 20] = -low
    z[22, 3:9] = np.inf
    z[23], z[23, 7] = 40.0, 41.0
    z[24] = -60.0 - np.arange(E)
    bias = rounded(rng.standard_normal(E), bp.BP_F32)
    bias[4] = -np.inf
    bias[5] = np.nan
    dgate = rounded(rng.standard_normal((n, k)), bp.BP_F32)
    check(z, None, k, dtype, kind, dgate, G, open_, top, renormalise, -0.5)
    check(z, bias, k, dtype, kind, dgate, G, open_, top, renormalise)
    bias[9] = np.inf
    check(z, bias, k, dtype, kind, dgate, G, open_, top, renormalise)


def test_nan_logits_are_seen():
    z = np.zeros((300, 8))
    z[:, 2] = 1.0
    z[4, 2] = np.nan
    z[6] = np.nan
    z[280, 7] = np.nan
    for kind in KINDS:
        for G in (1, 2):
            for n in (200, 300):
                check(z[:n], np.zeros(8), 2, bp.BP_F32, kind, None, G, 1, 2, True)


def test_no_patterns():
    out = check(np.zeros((0, 8)), None, 2, bp.BP_F32, "softmax", np.zeros((0, 2)))
    assert out[2].cpu().tolist() == [0] * 9


def test_refuses():
    with bp.ScoredRouter(8, 2, bp.BP_F32, max_patterns=4, n_groups=2) as r:
        z, b = torch.zeros(5, 8, device="cuda"), torch.zeros(8, device="cuda")
        i, f = torch.zeros(16, dtype=torch.int32, device="cuda"), torch.zeros(16, device="cuda")
        for call in (lambda: r.forward(z, b, 5, i, f, i, i, i), lambda: r.backward(z, -1, i, f, z)):
            with pytest.raises(bp.BPError) as e:
                call()
            assert e.value.status == bp.BP_EINVAL and "n must be" in str(e.value)
        with pytest.raises(bp.BPError) as e:
            r.forward(z, b, 4, i, f, None, i, i)
        assert e.value.status == bp.BP_EINVAL and "d_offsets" in str(e.value)
        for call in (lambda: r.forward(z, b[:7], 4, i, f, i, i, i), lambda: r.forward(z.bfloat16(), b, 4, i, f, i, i, i),
                     lambda: r.forward(z, b.bfloat16(), 4, i, f, i, i, i), lambda: r.backward(z, 4, i, f[:3], z)):
            with pytest.raises(ValueError):
                call()


@pytest.mark.parametrize("n", [90, 9001])
def test_replayed_for_other_logits(n):
    """A graph of both directions on a side stream, replayed: what direct calls write, bit for bit."""
    E, k, rng = 60, 4, np.random.default_rng(9)
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    bias, dgate = rounded(rng.standard_normal(E) * 0.1, bp.BP_F32), dev(rounded(rng.standard_normal((n, k)), bp.BP_F32))
    zd, bd, out, dz = empty((n, E), bp.BP_BF16, 0.0), dev(bias), outputs(n, E, k), empty((n, E), bp.BP_BF16)
    with bp.ScoredRouter(E, k, bp.BP_BF16, n + 7, bp.BP_SCORES_SIGMOID, 12, 5, 2, True) as r:
        with torch.cuda.graph(graph, stream=s):
            r.forward(zd, bd, n, *out, stream=s)
            r.backward(zd, n, out[0], dgate, dz, stream=s)
        for _ in range(2):
            z = rounded(rng.standard_normal((n, E)) * 2, bp.BP_BF16)
            zd.copy_(dev(z, bp.BP_BF16))
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                graph.replay()
            s.synchronize()
            want = O.route_scored(z, bias, k, "sigmoid", 12, 5, 2, True)
            for i in (0, 2, 3, 4):
                np.testing.assert_array_equal(out[i].cpu().numpy(), want[i], err_msg=NAMES[i])
            kept = [x.clone() for x in out + [dz]]
            torch.cuda.synchronize()
            r.forward(zd, bd, n, *out, stream=s)
            r.backward(zd, n, out[0], dgate, dz, stream=s)
            s.synchronize()
            for a, b in zip(kept, out + [dz]):
                assert torch.equal(a, b)
        del graph
