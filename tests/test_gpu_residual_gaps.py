"""Rows that no range of gates has (places behind the last sequence, or between two): the block's output is not theirs, whatever
lies there, and has no part in any gradient.  A call with such rows is compared, bit for bit, with one whose rows there are ordinary."""
import numpy as np
import pytest

from expert_cases import dev, empty, rounded
from oracle import blocks_oracle as O
from paper_1801_01554_gb300 import bp

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,width", [(bp.BP_F32, 24), (bp.BP_F32, 203), (bp.BP_F32, 3001), (bp.BP_F32, 4100), (bp.BP_BF16, 8),
                                         (bp.BP_BF16, 264), (bp.BP_BF16, 4104)])
@pytest.mark.parametrize("out,into", [(O.RMS, O.RMS), (O.LAYER, O.LAYER), (O.NONE, O.RMS), (O.NONE, O.NONE)])
@pytest.mark.parametrize("n", [9, 61, 40000])
def test_rows_of_no_range(n, out, into, dtype, width):
    if n * width > 12_000_000:
        n = 12_000_000 // width   # some rows of each worker of the backward pass
    rng = np.random.default_rng([n, width, out])
    gates = 3
    offsets = np.array([2, n // 3, n // 3 + 1 + n // 8, n - 2])   # the second range begins where the first ends
    where = torch.zeros(n, dtype=torch.bool, device="cuda")
    where[:2], where[n - 2:] = True, True
    g = torch.Generator(device="cuda").manual_seed(n)
    t = torch.bfloat16 if dtype == bp.BP_BF16 else torch.float32
    X, F, dY, dH = (torch.randn(n, width, generator=g, device="cuda").to(t) for _ in range(4))
    w = {x: dev(rounded(rng.standard_normal(width), bp.BP_F32)) for x, kind in (("wo", out), ("wi", into)) if kind != O.NONE}
    if out == O.LAYER:
        w["bo"] = dev(rounded(rng.standard_normal(width), bp.BP_F32))
    k = dict(w, gate=torch.randn(gates, width, generator=g, device="cuda"), offsets=dev(offsets), n_gates=gates, scale=0.5)

    def run(F, dY):
        Y, stats = empty((n, width), dtype), empty((n, 4), bp.BP_F32)
        H = empty((n, width), dtype) if into != O.NONE else None
        got = dict(dX=empty((n, width), dtype), dF=empty((n, width), dtype), Ggate=empty((gates, width), bp.BP_F32))
        for x in w:
            got["G" + x] = empty((width,), bp.BP_F32)
        with bp.Residual(width, dtype, n, out, into, 1e-5, max_gates=gates) as layer:
            layer.forward(X, F, n, Y, H, stats, **k)
            layer.backward(Y, F, n, stats, dY, dH if H is not None else None, **k, **got)
            layer.check()
        return dict(got, Y=Y) | ({} if H is None else dict(H=H))

    want = run(F, dY)
    assert torch.equal(want["Y"][where], X[where]) and (want["dF"][where] == 0).all()
    assert all(bool(x.isfinite().all()) for x in want.values())
    for bad in (float("nan"), float("inf"), -float("inf")):
        f = F.clone()
        f[where] = bad
        f[0, 1:] = 1.0   # one bad value of a row
        got = run(f, dY)
        for x in want:
            assert torch.equal(got[x], want[x]), (x, bad)
        d = dY.clone()
        d[where] = bad
        got = run(f, d)
        for x in want:
            rows = slice(None) if x != "dX" else ~where   # the stream's own gradient there is what came
            assert torch.equal(got[x][rows], want[x][rows]), (x, bad)
