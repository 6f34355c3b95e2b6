"""The residual stream against the float64 oracle.

Sums over a row take at most 16 values a thread, 5 and 16 additions: 37 * 2^-24 of the magnitudes, for a root half as
much of itself; with the few operations around them 2^-18 of a result's magnitudes going forward, where the oracle's magnitudes
count a mean beside what it is taken from.  A gradient has two such sums behind one another, and those by column add at most as many
rows as a test has per block and 50: 2^-16.  Rows are rounded once more to bfloat16: 2^-8 of themselves.
"""
import numpy as np
import pytest

from expert_cases import BF16, SUM, dev, empty, host, ragged, rounded
from oracle import blocks_oracle as O
from paper_1801_01554_gb300 import bp

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

NORM, EPS = 2.0 ** -18, float(np.float32(1e-5))
WEIGHTS = {O.NONE: "", O.RMS: "w", O.LAYER: "wb"}


def make(rng, n, width, dtype, out, into, gates, mean=0.0):
    def values(*shape, scale=1.0, at=0.0, t=dtype):
        return rounded(rng.standard_normal(shape) * scale + at, t)
    s = dict(X=values(n, width, scale=2.0, at=mean), F=values(n, width, scale=0.7, at=mean), dY=values(n, width))
    for name, kind in (("o", out), ("i", into)):
        if "w" in WEIGHTS[kind]:
            s["w" + name] = values(width, scale=0.3, at=1.0, t=bp.BP_F32)
        if "b" in WEIGHTS[kind]:
            s["b" + name] = values(width, scale=0.3, t=bp.BP_F32)
    if into != O.NONE:
        s["dH"] = values(n, width)
    if gates:
        s["gate"] = values(gates, width, t=bp.BP_F32)
    if gates > 1:
        s["offsets"] = np.arange(n + 1).astype(np.int32) if gates == n else ragged(rng, n, gates)
    return s


def way(s, scale, gates, device=True):
    return {x: dev(s.get(x)) for x in ("wo", "bo", "gate", "offsets", "wi")} | dict(n_gates=gates, scale=scale)


def close(got, want, mag, tol, half, what):
    err, bound = np.abs(host(got) - want), tol * mag + half * np.abs(want) + 1e-37
    assert (err <= bound).all(), (what, float(np.max(err / bound)))


def check_forward(s, Y, H, stats, scale, dtype, out, into):
    half = BF16 if dtype == bp.BP_BF16 else 0.0
    y, mag = O.residual(s["X"], s.get("F"), s.get("wo"), s.get("bo"), s.get("gate"), s.get("offsets"), scale, out, EPS)
    close(Y, y, mag + np.abs(s["X"]) * 2.0 ** -5, NORM, half, "Y")
    stored = host(Y)
    if H is not None:
        close(H, *O.norm_in(stored, s.get("wi"), s.get("bi"), into, EPS), NORM, half, "H")
    if stats is not None:
        for i, (x, kind) in enumerate(((s.get("F"), out), (stored, into))):
            if x is None or kind == O.NONE:
                want_mean, want_r, size = 0.0, 1.0, 0.0
            else:
                _, want_mean, want_r, _ = O.normed(x, kind, EPS)
                size = np.abs(x).mean(1, keepdims=True)
            got = host(stats)
            assert (np.abs(got[:, 2 * i:2 * i + 1] - want_mean) <= NORM * size).all()
            assert (np.abs(got[:, 2 * i + 1:2 * i + 2] / want_r - 1) <= NORM * (1 + size * want_r)).all()
    return stored


def check_backward(s, stored, got, scale, dtype, out, into, before=0.0):
    half = BF16 if dtype == bp.BP_BF16 else 0.0
    want = O.residual_backward(stored, s.get("F"), s.get("wo"), s.get("bo"), s.get("gate"), s.get("offsets"), scale, s.get("wi"),
                               s.get("dY"), s.get("dH"), out, into, EPS)
    for name, x in got.items():
        g, mag = want[name]
        if name[0] == "G":
            close(x, g + before, mag + abs(before), SUM, 0.0, name)
        else:
            close(x, g, mag, SUM, half, name)


def run(s, n, width, dtype, out, into, gates, scale, rows=None):
    k = way(s, scale, gates)
    X, F = dev(s["X"], dtype), dev(s["F"], dtype)
    Y, stats = empty((n, width), dtype), empty((n, 4), bp.BP_F32)
    H = empty((n, width), dtype) if into != O.NONE else None
    got = dict(dX=empty((n, width), dtype), dF=empty((n, width), dtype))
    for name in ("wo", "bo", "wi", "bi", "gate"):
        if name in s:
            got["G" + name] = empty(s[name].shape, bp.BP_F32)
    with bp.Residual(width, dtype, rows or n, out, into, EPS, max(gates, 1)) as layer:
        layer.forward(X, F, n, Y, H, stats, bi=dev(s.get("bi")), **k)
        layer.backward(Y, F, n, stats, dev(s["dY"], dtype), dev(s.get("dH"), dtype), **k, **got)
        layer.check()
        again = {x: g.clone() for x, g in got.items()}
        layer.backward(Y, F, n, stats, dev(s["dY"], dtype), dev(s.get("dH"), dtype), **k, **got)
        for x in got:
            assert torch.equal(again[x], got[x]), x
        stored = check_forward(s, Y, H, stats, scale, dtype, out, into)
        check_backward(s, stored, got, scale, dtype, out, into)
        # added to what is there
        for x in got:
            got[x].fill_(2.0)
        layer.backward(Y, F, n, stats, dev(s["dY"], dtype), dev(s.get("dH"), dtype), accumulate=True, **k, **got)
        torch.cuda.synchronize()
        check_backward(s, stored, got, scale, dtype, out, into, before=2.0)


SIZES = [(bp.BP_F32, 1), (bp.BP_F32, 3), (bp.BP_F32, 203), (bp.BP_F32, 256), (bp.BP_F32, 519), (bp.BP_F32, 2049), (bp.BP_F32, 2052),
         (bp.BP_F32, 4100), (bp.BP_F32, 8191), (bp.BP_F32, 8192), (bp.BP_BF16, 8), (bp.BP_BF16, 264), (bp.BP_BF16, 2048),
         (bp.BP_BF16, 4104), (bp.BP_BF16, 8192)]


@pytest.mark.parametrize("dtype,width", SIZES)
@pytest.mark.parametrize("out,into", [(O.RMS, O.RMS), (O.LAYER, O.LAYER), (O.NONE, O.LAYER), (O.RMS, O.NONE)])
@pytest.mark.parametrize("n,gates", [(1, 1), (7, 3), (13, 13)])
def test_few_rows(n, gates, out, into, dtype, width):
    rng = np.random.default_rng([n, width, out, into])
    run(make(rng, n, width, dtype, out, into, gates), n, width, dtype, out, into, gates, 0.625)


@pytest.mark.parametrize("out", [O.NONE, O.RMS, O.LAYER])
@pytest.mark.parametrize("into", [O.NONE, O.RMS, O.LAYER])
@pytest.mark.parametrize("dtype,width,n,gates", [(bp.BP_F32, 37, 5000, 0), (bp.BP_F32, 136, 999, 1), (bp.BP_BF16, 16, 6007, 17),
                                                 (bp.BP_BF16, 520, 1500, 1500), (bp.BP_BF16, 1032, 700, 5)])
def test_many_rows(out, into, dtype, width, n, gates):
    rng = np.random.default_rng([n, width, out, into])
    run(make(rng, n, width, dtype, out, into, gates), n, width, dtype, out, into, gates, -0.5, rows=n + 3)


@pytest.mark.parametrize("dtype,width", [(bp.BP_F32, 77), (bp.BP_F32, 1024), (bp.BP_BF16, 2048)])
def test_rows_far_from_zero(dtype, width):
    """A mean of 100 standard deviations and more does not cancel the variance."""
    rng = np.random.default_rng(3)
    s = make(rng, 20, width, dtype, O.LAYER, O.LAYER, 1, mean=200.0)
    run(s, 20, width, dtype, O.LAYER, O.LAYER, 1, 1.0)


@pytest.mark.parametrize("dtype", [bp.BP_F32, bp.BP_BF16])
def test_constant_rows_and_rows_of_zeros(dtype):
    rng = np.random.default_rng(3)
    s = make(rng, 9, 48, dtype, O.LAYER, O.RMS, 0)
    s["F"][2], s["F"][4], s["X"][4], s["X"][5], s["F"][5] = 3.0, 0.0, 0.0, 1.0, -1.0
    s["bo"][:] = 0.0
    run(s, 9, 48, dtype, O.LAYER, O.RMS, 0, 1.0)


@pytest.mark.parametrize("dtype,width", [(bp.BP_F32, 50), (bp.BP_BF16, 264)])
def test_parts_left_out(dtype, width):
    """No block before, no norm's output, and gradients from one side only; in place where that is allowed."""
    rng = np.random.default_rng(5)
    n = 40
    for out, into in ((O.RMS, O.RMS), (O.LAYER, O.LAYER)):
        s = make(rng, n, width, dtype, out, into, 3)
        k = way(s, 0.5, 3)
        with bp.Residual(width, dtype, n, out, into, EPS, max_gates=3) as layer:
            X, F, Y, H, stats = (dev(s["X"], dtype), dev(s["F"], dtype), empty((n, width), dtype), empty((n, width), dtype),
                                 empty((n, 4), bp.BP_F32))
            bi = dev(s.get("bi"))
            # no block before
            first = dict(X=s["X"], wi=s["wi"], bi=s.get("bi"))
            layer.forward(X, None, n, Y, H, stats, bi=bi, **k)
            check_forward(first, Y, H, stats, 0.5, dtype, out, into)
            assert torch.equal(Y, X)
            layer.forward(X, None, n, None, H, bi=bi, **k)
            check_forward(first, X, H, None, 0.5, dtype, out, into)
            dX, Gwi = empty((n, width), dtype), empty((width,), bp.BP_F32)
            layer.backward(X, None, n, stats, dev(s["dY"], dtype), dev(s["dH"], dtype), dX=dX, Gwi=Gwi, **k)
            check_backward(dict(first, dY=s["dY"], dH=s["dH"]), s["X"], dict(dX=dX, Gwi=Gwi), 0.5, dtype, out, into)
            # the sum alone, over X; then both in place
            layer.forward(X, F, n, X, None, stats, bi=bi, **k)
            check_forward(s, X, None, stats, 0.5, dtype, out, into)
            X = dev(s["X"], dtype)
            layer.forward(X, F, n, X, F, stats, bi=bi, **k)
            stored = check_forward(s, X, F, stats, 0.5, dtype, out, into)
            # one side only
            F = dev(s["F"], dtype)
            for dY, dH in ((s["dY"], None), (None, s["dH"]), (None, None)):
                got = dict(dX=empty((n, width), dtype), dF=empty((n, width), dtype), Gwo=empty((width,), bp.BP_F32),
                           Ggate=empty((3, width), bp.BP_F32))
                layer.backward(X if dH is not None else None, F, n, stats, dev(dY, dtype), dev(dH, dtype), **k, **got)
                check_backward(dict(s, dY=dY, dH=dH), stored, got, 0.5, dtype, out, into)
            Gwi = empty((width,), bp.BP_F32)
            layer.backward(None, F, n, stats, dev(s["dY"], dtype), None, Gwi=Gwi, **k)
            assert (Gwi == 0).all()
            dY, dH = dev(s["dY"], dtype), dev(s["dH"], dtype)
            layer.backward(X, F, n, stats, dY, dH, dX=dY, dF=dH, **k)
            check_backward(s, stored, dict(dX=dY, dF=dH), 0.5, dtype, out, into)
            layer.check()


def test_float_rows_off_16_bytes():
    n, width, rng = 30, 64, np.random.default_rng(6)
    s = make(rng, n, width, bp.BP_F32, O.RMS, O.RMS, 1)

    def off(x):
        b = torch.full((n * width + 1,), float("nan"), device="cuda")
        if x is not None:
            b[1:] = dev(x).view(-1)
        return b[1:].view(n, width)
    k = way(s, 1.0, 1)
    with bp.Residual(width, bp.BP_F32, n, O.RMS, O.RMS, EPS) as layer:
        X, F, Y, H, stats = off(s["X"]), off(s["F"]), off(None), off(None), empty((n, 4), bp.BP_F32)
        layer.forward(X, F, n, Y, H, stats, **k)
        stored = check_forward(s, Y, H, stats, 1.0, bp.BP_F32, O.RMS, O.RMS)
        got = dict(dX=off(None), dF=off(None), Gwo=empty((width,), bp.BP_F32), Ggate=empty((1, width), bp.BP_F32))
        layer.backward(Y, F, n, stats, off(s["dY"]), off(s["dH"]), **k, **got)
        check_backward(s, stored, got, 1.0, bp.BP_F32, O.RMS, O.RMS)


def test_rows_outside_every_range_and_bad_offsets():
    n, width, rng = 50, 24, np.random.default_rng(7)
    s = make(rng, n, width, bp.BP_F32, O.RMS, O.RMS, 4)
    s["offsets"] = np.array([3, 10, 10, 30, 45], dtype=np.int32)
    run(s, n, width, bp.BP_F32, O.RMS, O.RMS, 4, 1.0)
    X, F, Y, stats, g = (dev(s["X"]), dev(s["F"]), empty((n, width), bp.BP_F32), empty((n, 4), bp.BP_F32), empty((4, width), bp.BP_F32))
    with bp.Residual(width, bp.BP_F32, n, O.RMS, O.RMS, EPS, max_gates=4) as layer:
        for bad in ([0, 10, 9, 30, 50], [-1, 10, 20, 30, 50], [0, 10, 20, 30, 51], [0, 2 ** 31 - 1, 20, -2 ** 31, 50]):
            k = dict(wo=dev(s["wo"]), gate=dev(s["gate"]), offsets=dev(np.array(bad)), n_gates=4)
            layer.forward(X, F, n, Y, None, stats, **k)
            with pytest.raises(bp.BPError) as e:
                layer.check()
            assert e.value.status == bp.BP_ESTATE and "offsets" in str(e.value)
            layer.backward(None, F, n, stats, X, None, Ggate=g, **k)
            with pytest.raises(bp.BPError):
                layer.check()
        layer.check()


def test_no_rows():
    w = torch.full((8,), 5.0, device="cuda")
    with bp.Residual(8, bp.BP_F32, 4, O.RMS, O.RMS) as layer:
        layer.forward(None, None, 0, None)
        layer.backward(None, None, 0, None, None, None, Gwi=w, accumulate=True)
        assert (w == 5).all()
        layer.backward(None, None, 0, None, None, None, Gwi=w)
        assert (w == 0).all()


def test_replayed_for_other_rows():
    n, width, dtype, rng = 333, 264, bp.BP_BF16, np.random.default_rng(8)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s = make(rng, n, width, dtype, O.RMS, O.RMS, 5)
    k = way(s, 1.0, 5)
    X, F, dY, dH = (dev(s[x], dtype) for x in ("X", "F", "dY", "dH"))
    Y, H, stats = empty((n, width), dtype), empty((n, width), dtype), empty((n, 4), bp.BP_F32)
    got = dict(dX=empty((n, width), dtype), dF=empty((n, width), dtype), Gwo=empty((width,), bp.BP_F32), Gwi=empty((width,), bp.BP_F32),
               Ggate=empty((5, width), bp.BP_F32))
    with bp.Residual(width, dtype, n, O.RMS, O.RMS, EPS, max_gates=5) as layer:
        with torch.cuda.graph(graph, stream=stream):
            layer.forward(X, F, n, Y, H, stats, stream=stream, **k)
            layer.backward(Y, F, n, stats, dY, dH, stream=stream, **k, **got)
        for _ in range(2):
            t = make(rng, n, width, dtype, O.RMS, O.RMS, 5)
            for name, x in (("X", X), ("F", F), ("dY", dY), ("dH", dH)):
                x.copy_(dev(t[name], dtype))
            k["offsets"].copy_(dev(t["offsets"]))
            s.update(X=t["X"], F=t["F"], dY=t["dY"], dH=t["dH"], offsets=t["offsets"])
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                graph.replay()
            stream.synchronize()
            stored = check_forward(s, Y, H, stats, 1.0, dtype, O.RMS, O.RMS)
            check_backward(s, stored, got, 1.0, dtype, O.RMS, O.RMS)
        layer.check(stream)
        del graph


def test_residual_refuses():
    n, w = 4, 8
    x, v, i, st = torch.zeros(n + 1, w, device="cuda"), torch.zeros(w, device="cuda"), dev(np.array([0, 4])), torch.zeros(n, 4, device="cuda")
    y = torch.zeros(n + 1, w, device="cuda")

    def refused(call, word):
        with pytest.raises(bp.BPError) as e:
            call()
        assert e.value.status == bp.BP_EINVAL and word in str(e.value), str(e.value)
    with bp.Residual(w, bp.BP_F32, n, O.RMS, O.RMS) as a, bp.Residual(w, bp.BP_F32, n, O.NONE, O.NONE) as b:
        refused(lambda: a.forward(x, x, n + 1, y), "n must be")
        refused(lambda: a.forward(x, x, n, y, gate=x[:2].contiguous(), offsets=dev(np.array([0, 2, 4])), n_gates=2), "n_gates must be")
        refused(lambda: a.forward(x, x, n, y, gate=v), "d_gate and n_gates")
        refused(lambda: a.forward(x, x, n, y, n_gates=1), "d_gate and n_gates")
        refused(lambda: a.forward(x, x, n, y, offsets=i), "d_offsets")
        refused(lambda: a.forward(x, x, n, y, scale=float("inf")), "scale")
        refused(lambda: a.forward(x, x, n, y, bo=v), "weight or bias")
        refused(lambda: a.forward(x, x, n, y, bi=v), "weight or bias")
        refused(lambda: b.forward(x, x, n, y, wo=v), "weight or bias")
        refused(lambda: b.forward(x, x, n, y, wi=v), "weight or bias")
        refused(lambda: b.forward(x, x, n, y, y), "d_H")
        refused(lambda: a.forward(x, x, n, None, y), "d_Y")
        refused(lambda: a.forward(None, x, n, y), "d_X")
        refused(lambda: a.forward(x.data_ptr() + 2, x, n, y), "aligned")
        refused(lambda: a.backward(None, x, n, st, x, x), "d_Y")
        refused(lambda: a.backward(x, x, n, None, x, x), "d_stats")
        refused(lambda: b.backward(x, x, n, st, x, x), "d_dH")
        refused(lambda: a.backward(x, None, n, st, x, x, dF=y), "without d_F")
        refused(lambda: a.backward(x, x, n, st, x, x, Gbo=v), "do not have")
        refused(lambda: b.backward(x, x, n, st, x, None, Gwo=v), "do not have")
        refused(lambda: a.backward(x, x, n, st, x, x, Ggate=v), "d_Ggate")
        for call in (lambda: a.forward(x[:3], x, n, y), lambda: a.forward(x, x.bfloat16(), n, y), lambda: a.forward(x, x, n, y, wo=v[:7]),
                     lambda: a.forward(x, x, n, y, stats=st[:3]), lambda: a.forward(x, x, n, y, gate=v, offsets=i.long(), n_gates=1),
                     lambda: a.forward(x, x, n, y, gate=v, offsets=i[:1], n_gates=1), lambda: a.backward(x, x, n, st, x, x[:3])):
            with pytest.raises(ValueError):
                call()
        a.check()
