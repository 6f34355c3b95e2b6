"""Router and mix against the float64 oracle.

Choices, offsets, sources and places are whole numbers and must be equal.  Gates: exp and a
quotient in float32 of differences that are exact or rounded once, and a sum of at most 512
terms: 2^-19 of themselves.  Gradients by the bound of expert_cases.
"""
import numpy as np
import pytest

from expert_cases import BF16, SUM, dev, empty, host, rounded
from oracle import experts_oracle as O
from paper_1801_01554_gb300 import bp

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

GATE = 2.0 ** -19
NAMES = {"chosen": bp.BP_GATES_CHOSEN, "all": bp.BP_GATES_ALL}


def run(z, k, gates, dtype, dgate=None):
    n, E = z.shape
    out = dict(expert=torch.full((n, k), 99, dtype=torch.int32, device="cuda"),
               gate=torch.full((n, k), 99.0, device="cuda"),
               offsets=torch.full((E + 1,), 99, dtype=torch.int32, device="cuda"),
               source=torch.full((n * k,), 99, dtype=torch.int32, device="cuda"),
               place=torch.full((n, k), 99, dtype=torch.int32, device="cuda"))
    zd = dev(z, dtype)
    with bp.Router(E, k, dtype, max_patterns=max(n, 1), gates=NAMES[gates]) as r:
        r.forward(zd, n, **out)
        if dgate is not None:
            out["dz"] = empty((n, E), dtype)
            r.backward(zd, n, out["expert"], out["gate"], dev(dgate), out["dz"])
        torch.cuda.synchronize()
    return out


def check(z, k, gates, dtype, dgate):
    got = run(z, k, gates, dtype, dgate)
    expert, gate, offsets, source, place = O.route(z, k, gates)
    for name, want in (("expert", expert), ("offsets", offsets), ("source", source), ("place", place)):
        np.testing.assert_array_equal(got[name].cpu().numpy(), want, err_msg=name)
    np.testing.assert_allclose(host(got["gate"]), gate, rtol=GATE, atol=1e-37)
    want = O.route_backward(z, expert, gate, dgate, gates)
    mag = np.abs(dgate).max(initial=0.0) * z.shape[1]   # magnitudes of what a gradient adds up, at most
    tol = SUM * min(mag, 4 * np.abs(dgate).max(initial=0.0)) + (BF16 if dtype == bp.BP_BF16 else 0) * np.abs(want)
    assert (np.abs(host(got["dz"]) - want) <= tol + 1e-37).all()


@pytest.mark.parametrize("dtype", [bp.BP_F32, bp.BP_BF16])
@pytest.mark.parametrize("gates", ["chosen", "all"])
@pytest.mark.parametrize("n,E,k", [(1, 16, 2), (1, 1, 1), (5, 3, 3), (128, 8, 2), (129, 33, 4), (300, 64, 6), (777, 100, 1),
                                   (260, 512, 16), (4100, 40, 4), (40, 129, 16)])
def test_route_matches_oracle(n, E, k, gates, dtype):
    rng = np.random.default_rng([n, E, k])
    z = rounded(rng.standard_normal((n, E)) * 2 + rng.standard_normal(E), dtype)
    check(z, k, gates, dtype, rounded(rng.standard_normal((n, k)), bp.BP_F32))


@pytest.mark.parametrize("gates", ["chosen", "all"])
def test_closed_experts_ties_and_extreme_logits(gates):
    """Closed experts (-infinity), patterns with none open, ties, both zeros, the types' lowest
    values, and differences of logits that overflow."""
    for dtype in (bp.BP_F32, bp.BP_BF16):
        low = -3.3895313892515355e38 if dtype == bp.BP_BF16 else -float(np.finfo(np.float32).max)
        rng = np.random.default_rng(5)
        z = rounded(rng.integers(-2, 3, size=(200, 24)).astype(float), dtype)   # many ties
        z[rng.random(z.shape) < 0.5] = -np.inf
        z[3] = -np.inf
        z[150] = -np.inf
        z[7] = 0.0
        z[7, 5] = -0.0
        z[9] = low
        z[11] = -np.inf
        z[11, 13] = low
        z[12] = low
        z[12, 20] = -low
        check(z, 4, gates, dtype, rounded(rng.standard_normal((200, 4)), bp.BP_F32))


def test_nan_logits_are_seen():
    z = np.zeros((130, 8))
    z[:, 2] = 1.0
    z[4, 2] = np.nan
    z[6] = np.nan
    for gates in ("chosen", "all"):
        got = run(z, 2, gates, bp.BP_F32)
        expert, gate = got["expert"].cpu().numpy(), host(got["gate"])
        assert expert[4].tolist() == [0, 1] and np.isnan(gate[4]).all()
        assert expert[6].tolist() == [-1, -1] and (gate[6] == 0).all()
        assert np.isfinite(np.delete(gate, [4, 6], 0)).all()


def test_no_patterns():
    got = run(np.zeros((0, 8)), 2, "chosen", bp.BP_F32, np.zeros((0, 2)))
    assert got["offsets"].cpu().tolist() == [0] * 9


def test_route_refuses():
    with bp.Router(8, 2, bp.BP_F32, max_patterns=4) as r:
        z = torch.zeros(5, 8, device="cuda")
        i, f = torch.zeros(16, dtype=torch.int32, device="cuda"), torch.zeros(16, device="cuda")
        with pytest.raises(bp.BPError) as e:
            r.forward(z, 5, i, f, i, i, i)
        assert e.value.status == bp.BP_EINVAL and "n must be" in str(e.value)
        with pytest.raises(ValueError):
            r.forward(z, 4, i, f, i, i, i[:3])
        with pytest.raises(ValueError):
            r.forward(z.bfloat16(), 4, i, f, i, i, i)


def test_many_blocks_twice_on_a_side_stream():
    """More blocks than one scan step of 32, repeated: the same bits."""
    rng = np.random.default_rng(9)
    z = rounded(rng.standard_normal((9001, 20)), bp.BP_F32)
    want = O.route(z, 3, "all")
    s = torch.cuda.Stream()
    with bp.Router(20, 3, bp.BP_F32, max_patterns=10000, gates=bp.BP_GATES_ALL) as r:
        zd = dev(z)
        n = len(z)
        outs = []
        s.wait_stream(torch.cuda.current_stream())
        for _ in range(2):
            out = [torch.empty(n, 3, dtype=torch.int32, device="cuda"), torch.empty(n, 3, device="cuda"),
                   torch.empty(21, dtype=torch.int32, device="cuda"), torch.empty(n * 3, dtype=torch.int32, device="cuda"),
                   torch.empty(n, 3, dtype=torch.int32, device="cuda")]
            torch.cuda.synchronize()
            r.forward(zd, n, *out, stream=s)
            outs.append(out)
        s.synchronize()
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    for got, name, w in zip(outs[0], ("expert", "gate", "offsets", "source", "place"), want):
        if name != "gate":
            np.testing.assert_array_equal(got.cpu().numpy(), w, err_msg=name)


# ------------------------------------------------------------------ mix
@pytest.mark.parametrize("dtype,n_out", [(bp.BP_F32, 1), (bp.BP_F32, 26), (bp.BP_F32, 37), (bp.BP_F32, 1024), (bp.BP_BF16, 8),
                                         (bp.BP_BF16, 264), (bp.BP_BF16, 2048), (bp.BP_BF16, 4096)])
@pytest.mark.parametrize("n,k", [(1, 1), (7, 2), (130, 4), (33, 16), (2500, 2)])
def test_mix_matches_oracle(n, k, n_out, dtype):
    if n * k * n_out > 6e6:
        n = 200
    rng = np.random.default_rng([n, k, n_out])
    rows = n * k + 3
    H, D = rounded(rng.standard_normal((rows, n_out)), dtype), rounded(rng.standard_normal((n, n_out)), dtype)
    place = rng.permutation(rows)[:n * k].reshape(n, k).astype(np.int32)
    place[rng.random((n, k)) < 0.1] = -1
    if n > 5:
        place[2] = -1
        place[3, 0], place[4, 0] = rows + 5, -7   # out of range: no part
    gate = rounded(rng.standard_normal((n, k)), bp.BP_F32)
    Hd, Dd, pd, gd = dev(H, dtype), dev(D, dtype), dev(place), dev(gate)
    Y, dH, dg = empty((n, n_out), dtype), empty((rows, n_out), dtype, 5.0), empty((n, k), bp.BP_F32)
    bp.bp_mix(Hd, rows, pd, gd, n, k, n_out, dtype, Y)
    bp.bp_mix_backward(Dd, Hd, rows, pd, gd, n, k, n_out, dtype, dH, dg)
    dH2 = empty((rows, n_out), dtype, 5.0)
    bp.bp_mix_backward(Dd, None, rows, pd, gd, n, k, n_out, dtype, dH2)   # without the gates' gradient
    torch.cuda.synchronize()
    half = BF16 if dtype == bp.BP_BF16 else 2.0 ** -24
    want, mag = O.mix(H, place, gate), O.mix(np.abs(H), place, np.abs(gate))
    assert (np.abs(host(Y) - want) <= half * np.abs(want) + 2.0 ** -20 * mag).all()
    dHw = np.full(H.shape, 5.0)
    dgw = O.mix_backward(D, H, place, gate, dHw)
    dgm = O.mix_backward(np.abs(D), np.abs(H), place, gate, np.zeros(H.shape))
    assert (np.abs(host(dH) - dHw) <= (half + 2.0 ** -23) * np.abs(dHw)).all()
    assert torch.equal(dH, dH2)
    assert (np.abs(host(dg) - dgw) <= SUM * dgm).all()
    bp.bp_mix(Hd, rows, pd, None, n, k, n_out, dtype, Y)   # gates of 1
    want, mag = O.mix(H, place, np.ones((n, k))), O.mix(np.abs(H), place, np.ones((n, k)))
    assert (np.abs(host(Y) - want) <= half * np.abs(want) + 2.0 ** -20 * mag).all()


def test_mix_rows_off_16_bytes():
    """float32 buffers on a 4-byte boundary."""
    rng = np.random.default_rng(3)
    n, k, N = 9, 2, 64
    H = rounded(rng.standard_normal((n * k, N)), bp.BP_F32)
    place, gate = rng.permutation(n * k).reshape(n, k).astype(np.int32), rounded(rng.random((n, k)), bp.BP_F32)
    buf = torch.zeros(n * k * N + 1, device="cuda")
    buf[1:] = dev(H).view(-1)
    Y = empty((n, N), bp.BP_F32)
    bp.bp_mix(buf[1:], n * k, dev(place), dev(gate), n, k, N, bp.BP_F32, Y)
    want = O.mix(H, place, gate)
    np.testing.assert_allclose(host(Y), want, atol=1e-6)
