"""Adapter layers: calls without requests and without adapters' weights, and what long lists of requests
report.  The bound is that of expert_cases."""
import numpy as np
import pytest

from expert_cases import assert_sum, dev, empty, host, rounded
from oracle import experts_oracle as O
from paper_1801_01554_gb300 import bp

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [bp.BP_F32, bp.BP_BF16])
@pytest.mark.parametrize("rows", [3, 70, 300])
def test_no_requests_need_no_adapters(dtype, rows):
    rng = np.random.default_rng(rows)
    n_in, n_out = 72, 136
    X, D = rounded(rng.standard_normal((rows, n_in)), dtype), rounded(rng.standard_normal((rows, n_out)), dtype)
    W, b = rounded(rng.standard_normal((n_out, n_in)), dtype), rounded(rng.standard_normal(n_out), bp.BP_F32)
    Wd, Xd, Dd = dev(W, dtype), dev(X, dtype), dev(D, dtype)
    U, Y, dX = empty((rows, 4), bp.BP_F32), empty((rows, n_out), dtype), empty((rows, n_in), dtype)
    GA, GB = empty((2, 4, n_in), bp.BP_F32), empty((2, 4, n_out), bp.BP_F32)
    with bp.Adapters(2, 4, n_in, n_out, dtype, max_rows=rows, max_requests=1) as layer:
        layer.forward(Wd, dev(b), None, None, None, Xd, None, None, 0, rows, U, Y)
        layer.backward(Wd, None, None, None, Xd, None, None, None, 0, rows, Dd, dX=dX, GA=GA, GB=GB)
        layer.check()
    (wy, my), _ = O.adapters_forward(W, b, np.zeros((2, 4, n_in)), np.zeros((2, 4, n_out)), None, X, np.zeros(1, int), [])
    assert_sum(host(Y), wy, my, dtype, what="Y")
    assert_sum(host(dX), D @ W, np.abs(D) @ np.abs(W), dtype, what="dX")
    for z in (U, GA, GB):
        assert (host(z) == 0).all()


@pytest.mark.parametrize("dtype", [bp.BP_F32, bp.BP_BF16])
@pytest.mark.parametrize("requests,bad", [(700, 650), (700, 3), (513, 512)])
def test_a_bad_adapter_of_many_requests_is_reported_by_a_change_alone(dtype, requests, bad):
    rows = 2 * requests
    rng = np.random.default_rng(bad)
    D, U = rounded(rng.standard_normal((rows, 32)), dtype), rounded(rng.standard_normal((rows, 8)), bp.BP_F32)
    off, adapter = np.arange(requests + 1) * 2, np.arange(requests) % 3 - 1
    GB = empty((2, 8, 32), bp.BP_F32)
    with bp.Adapters(2, 8, 64, 32, dtype, max_rows=rows, max_requests=requests) as layer:
        def change():
            layer.backward(None, None, None, None, None, dev(U), dev(off), dev(adapter), requests, rows, dev(D, dtype), GB=GB)
            layer.check()
        adapter[bad] = 2
        with pytest.raises(bp.BPError) as e:
            change()
        assert e.value.status == bp.BP_ESTATE
        adapter[bad] = -1   # and as one without it is treated
        kept = host(GB)
        change()
        np.testing.assert_array_equal(host(GB), kept)
