"""Gradients of the stream's weights, biases and gates over very many rows: the error of a sum does not grow with them.

A worker adds up at most 128 rows in float32 (127 roundings of 2^-24) and goes on in float64, which is rounded once; workers and blocks add
16 + 76 + 32 more at most; a row's own term is within 2^-18 of its magnitude.  So 2^-16 + 2^-18 of the magnitudes bounds
all of it.  Rows that are all alike are the worst: every addition to a plain sum would be rounded the same way.
"""
import numpy as np
import pytest

from expert_cases import dev, empty, host, rounded
from oracle import blocks_oracle as O
from paper_1801_01554_gb300 import bp

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BOUND, EPS = 2.0 ** -16 + 2.0 ** -18, float(np.float32(1e-5))
SIZES = [(bp.BP_F32, 1, 4_000_003), (bp.BP_F32, 8, 3_000_001), (bp.BP_F32, 203, 600_007), (bp.BP_F32, 516, 200_000),
         (bp.BP_F32, 4100, 50_000), (bp.BP_BF16, 8, 3_000_001), (bp.BP_BF16, 264, 300_000), (bp.BP_BF16, 4104, 60_000),
         (bp.BP_F32, 8192, 20_003)]


def close(got, want, mag, what):
    err = np.abs(host(got) - want)
    assert (err <= BOUND * mag + 1e-37).all(), (what, float(np.max(err / (BOUND * mag + 1e-37))))


@pytest.mark.parametrize("dtype,width,n", SIZES)
@pytest.mark.parametrize("out,into", [(O.RMS, O.RMS), (O.LAYER, O.LAYER)])
@pytest.mark.parametrize("ranges", ["one", "some", "short"])
def test_equal_rows(ranges, out, into, dtype, width, n):
    """n times one row, whose sums are n times that row's; gates for all rows, by a few ranges, and by ranges of a few rows."""
    rng = np.random.default_rng([n, width, out])
    def values(at=0.0, t=dtype):
        return rounded(rng.standard_normal((1, width)) + at, t)
    s = dict(X=values(), F=values(), dY=values(0.7), dH=values(1.1))
    w = {x: values(1.0, bp.BP_F32)[0] for x in ("wo", "wi")}
    if out == O.LAYER:
        w["bo"] = values(0.0, bp.BP_F32)[0]
    if ranges == "one":
        offsets, gate = None, values(1.0, bp.BP_F32)
    elif ranges == "some":
        offsets, gate = np.array([0, n // 5, n // 5, n - 77, n]), rounded(rng.standard_normal((4, width)), bp.BP_F32)
    else:
        gates = min(n // 3, 70_000_000 // width)
        offsets = np.concatenate([np.arange(gates) * 3, [n]])
        gate = np.repeat(values(1.0, bp.BP_F32), gates, 0)
    m = len(gate)
    X, F, dY, dH = (dev(x, dtype).expand(n, width).contiguous() for x in s.values())
    k = dict({x: dev(v) for x, v in w.items()}, gate=dev(gate), offsets=None if offsets is None else dev(offsets), n_gates=m, scale=0.5)
    got = {"G" + x: empty((width,), bp.BP_F32) for x in ("wo", "wi") + (("bo", "bi") if out == O.LAYER else ())}
    got["Ggate"] = empty((m, width), bp.BP_F32)
    Y, stats = empty((n, width), dtype), empty((n, 4), bp.BP_F32)
    with bp.Residual(width, dtype, n, out, into, EPS, max_gates=m) as layer:
        layer.forward(X, F, n, Y, None, stats, **k)
        layer.backward(Y, F, n, stats, dY, dH, **k, **got)
        layer.check()
    counts = np.array([n]) if offsets is None else np.diff(offsets)
    sums = {}
    alike = [0, m - 1] if ranges == "short" else range(m)   # the last range takes the rows that are left
    for i in alike:
        row = host(Y[0 if offsets is None else min(int(offsets[i]), n - 1)][None])
        one = O.residual_backward(row, s["F"], w["wo"], w.get("bo"), gate[i:i + 1], None, 0.5, w["wi"], s["dY"], s["dH"], out, into, EPS)
        close(got["Ggate"][i][None], counts[i] * one["Ggate"][0], counts[i] * one["Ggate"][1], ("Ggate", i))
        rows = n if ranges == "short" else counts[i]
        for x in got:
            if x != "Ggate":
                a, b = sums.get(x, (0.0, 0.0))
                sums[x] = a + rows * one[x][0], b + rows * one[x][1]
        if ranges == "short":
            break
    for x, (want, mag) in sums.items():
        close(got[x], want, mag, x)


@pytest.mark.parametrize("ranges", [False, True])
def test_any_rows(ranges):
    """Rows of their own, against sums in 64 bits of the same stream: biases and weights of both norms."""
    n, width = 500_000, 40
    g = torch.Generator(device="cuda").manual_seed(3)
    X, F, dY, dH = (torch.randn(n, width, generator=g, device="cuda") for _ in range(4))
    gate = torch.randn(3 if ranges else 1, width, generator=g, device="cuda")
    offsets = torch.tensor([0, 70_001, 70_002, n], dtype=torch.int32, device="cuda") if ranges else None
    got = {x: empty((width,), bp.BP_F32) for x in ("Gwo", "Gbo", "Gwi", "Gbi")}
    Y, stats = empty((n, width), bp.BP_F32), empty((n, 4), bp.BP_F32)
    k = dict(gate=gate, offsets=offsets, n_gates=len(gate), scale=1.0)
    with bp.Residual(width, bp.BP_F32, n, O.LAYER, O.LAYER, EPS, max_gates=3) as layer:
        layer.forward(X, F, n, Y, None, stats, **k)
        layer.backward(Y, F, n, stats, dY, dH, **k, **got)
        first = {x: v.clone() for x, v in got.items()}
        layer.backward(Y, F, n, stats, dY, dH, **k, **got)
        layer.check()
    assert all(torch.equal(first[x], got[x]) for x in got)
    norm = lambda x: (x - x.mean(1, keepdim=True)) / (x.var(1, correction=0, keepdim=True) + EPS).sqrt()
    y, f, d, h = norm(Y.double()), norm(F.double()), dY.double(), dH.double()
    r = 1 / (Y.double().var(1, correction=0, keepdim=True) + EPS).sqrt()
    d = d + r * (h - h.mean(1, keepdim=True) - y * (h * y).mean(1, keepdim=True))
    rows = gate.double()[torch.searchsorted(offsets[1:].long(), torch.arange(n, device="cuda"), right=True)] if ranges else gate.double()
    u = d * rows
    for x, terms in (("Gwo", u * f), ("Gbo", u), ("Gwi", h * y), ("Gbi", h)):
        err, mag = (got[x].double() - terms.sum(0)).abs(), terms.abs().sum(0)
        assert bool((err <= BOUND * 4 * mag).all()), (x, float((err / mag).max()))
