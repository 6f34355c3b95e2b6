"""Handles of expert and adapter layers beside a busy default stream: a new layer, or one whose errors were
just reported, is ready for a call on any stream.  The bound is that of expert_cases."""
import numpy as np
import pytest

from expert_cases import assert_sum, dev, empty, host, rounded
from oracle import experts_oracle as O
from paper_1801_01554_gb300 import bp

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def busy_default_stream():
    """Some 100 ms of work, queued."""
    x = torch.ones(64 << 20, device="cuda")
    for _ in range(500):
        x.mul_(1.0)
    return x


@pytest.mark.parametrize("dtype", [bp.BP_F32, bp.BP_BF16])
def test_new_layers_on_a_side_stream(dtype):
    """Changes whose rows are shared out, by a layer that was made behind queued work."""
    rng = np.random.default_rng(1)
    rows, n_in, n_out, rank = 6000, 64, 32, 16
    X, D = rounded(rng.standard_normal((rows, n_in)), dtype), rounded(rng.standard_normal((rows, n_out)), dtype)
    U, B = rounded(rng.standard_normal((rows, rank)), bp.BP_F32), rounded(rng.standard_normal((1, rank, n_out)), dtype)
    _, (ww, mw), (wb, mb) = O.experts_backward(np.zeros((2, n_out, n_in)), X, None, [0, 2500, rows], D, False)
    _, (wa, ma), (wg, mg) = O.adapters_backward(np.zeros((n_out, n_in)), np.zeros((1, rank, n_in)), B, None, X, U, [0, rows],
                                                [0], D, False)
    Xd, Dd, Ud, Bd = dev(X, dtype), dev(D, dtype), dev(U), dev(B, dtype)
    cut, off, ad = dev(np.array([0, 2500, rows])), dev(np.array([0, rows])), dev(np.array([0]))
    outs = [(empty((2, n_out, n_in), bp.BP_F32), empty((2, n_out), bp.BP_F32), empty((1, rank, n_in), bp.BP_F32),
             empty((1, rank, n_out), bp.BP_F32)) for _ in range(2)]
    s = torch.cuda.Stream()
    for GW, Gb, GA, GB in outs:
        torch.cuda.synchronize()
        kept = busy_default_stream()
        with bp.Experts(2, n_in, n_out, dtype, max_rows=rows) as layer:
            layer.backward(None, Xd, rows, None, cut, rows, Dd, GW=GW, Gb=Gb, stream=s)
            layer.check(s)
        kept = busy_default_stream()
        with bp.Adapters(1, rank, n_in, n_out, dtype, max_rows=rows, max_requests=1) as layer:
            layer.backward(None, None, Bd, None, Xd, Ud, off, ad, 1, rows, Dd, GA=GA, GB=GB, stream=s)
            layer.check(s)
        del kept
    for GW, Gb, GA, GB in outs:
        for got, want, mag in ((GW, ww, mw), (Gb, wb, mb), (GA, wa, ma), (GB, wg, mg)):
            assert_sum(host(got), want, mag, bp.BP_F32)


@pytest.mark.parametrize("dtype", [bp.BP_F32, bp.BP_BF16])
def test_errors_are_cleared_before_the_next_call(dtype):
    """An error that is reported beside queued work is gone, and the next one is not."""
    rows, n = 40, 16
    W, X, Y = (torch.zeros(s, device="cuda") for s in ((2, n, n), (rows, n), (rows, n)))
    if dtype == bp.BP_BF16:
        W, X, Y = W.bfloat16(), X.bfloat16(), Y.bfloat16()
    good, bad = dev(np.array([0, 20, rows])), dev(np.array([0, 20, rows + 1]))
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    with bp.Experts(2, n, n, dtype, max_rows=rows) as layer:
        torch.cuda.synchronize()
        for i in range(6):
            kept = busy_default_stream()
            layer.forward(W, None, X, rows, None, bad, rows, Y, stream=streams[i % 2])
            with pytest.raises(bp.BPError) as e:
                layer.check(streams[i % 2])
            assert e.value.status == bp.BP_ESTATE
            layer.forward(W, None, X, rows, None, good, rows, Y, stream=streams[1 - i % 2])
            layer.check(streams[1 - i % 2])
        torch.cuda.synchronize()
        del kept
