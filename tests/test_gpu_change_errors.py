"""Float32 results of bfloat16 layers are as exact as float32: changes of weights and adapters and the
low-rank sums, by the 2-norm of their error against 64 bits.

The bound.  The tensor cores accumulate by truncation to 24 bits, 2^-24 of the running sum a step on
average, and the running sum of products of random signs is on average 2/3 of the last one; sums are cut
into parts of at most 32 steps of 16 products, whose sums are added by rounding to nearest.  So the error is
at most 32 * 2/3 * 2^-24 of the sums' 2-norm, 1.3e-6.  A float32 factor taken in three bfloat16 terms
loses 2^-25 of itself; in two it loses 2^-17 at most and 2.5e-6 in the 2-norm, which these tests tell.
"""
import numpy as np
import pytest

from expert_cases import dev, empty, host, rounded
from oracle import experts_oracle as O
from paper_1801_01554_gb300 import bp

torch = pytest.importorskip("torch")

NORM = 32 * 2 / 3 * 2.0 ** -24
BF = bp.BP_BF16


def error(got, want):
    return float(np.linalg.norm(got - want) / np.linalg.norm(want))


def terms(x, n):
    """x as the sum of n bfloat16 terms."""
    total, rest = np.zeros_like(x), x
    for _ in range(n):
        t = rounded(rest, BF)
        total, rest = total + t, rest - t
    return total


@pytest.mark.parametrize("rank", [16, 100])
def test_the_bound_tells_two_terms_from_three(rank):
    rng = np.random.default_rng(rank)
    u = rounded(rng.standard_normal((1024, rank)), bp.BP_F32)
    d = rounded(rng.standard_normal((1024, 64)), BF)
    want = u.T @ d
    assert error(terms(u, 2).T @ d, want) > NORM > 10 * error(terms(u, 3).T @ d, want)


@pytest.mark.gpu
@pytest.mark.parametrize("rank", [5, 16, 32, 48, 64, 65, 100, 128])
@pytest.mark.parametrize("offsets", [[0, 4096], [0, 1000, 1777, 3000]])
def test_adapters_changes(rank, offsets):
    """v is a sum of 64 products, four steps: 4 * 2/3 * 2^-24 more for its change."""
    rng = np.random.default_rng([rank, len(offsets)])
    n, n_in, n_out, rows, requests = 2, 200, 64, offsets[-1], len(offsets) - 1
    X, D = rounded(rng.standard_normal((rows, n_in)), BF), rounded(rng.standard_normal((rows, n_out)), BF)
    U = rounded(rng.standard_normal((rows, rank)), bp.BP_F32)
    W, A = rounded(rng.standard_normal((n_out, n_in)), BF), rounded(rng.standard_normal((n, rank, n_in)), BF)
    B, scale = rounded(rng.standard_normal((n, rank, n_out)), BF), rounded(rng.uniform(0.5, 2.0, n), bp.BP_F32)
    off, adapter = np.array(offsets), np.arange(requests) % n
    GA, GB = empty((n, rank, n_in), bp.BP_F32), empty((n, rank, n_out), bp.BP_F32)
    with bp.Adapters(n, rank, n_in, n_out, BF, max_rows=rows, max_requests=requests) as layer:
        layer.backward(None, None, dev(B, BF), dev(scale), dev(X, BF), dev(U), dev(off), dev(adapter), requests, rows,
                       dev(D, BF), GA=GA, GB=GB)
        layer.check()
    _, (wa, _), (wb, _) = O.adapters_backward(W, A, B, scale, X, U, off, adapter, D, False)
    assert error(host(GA), wa) <= NORM + 4 * 2 / 3 * 2.0 ** -24
    assert error(host(GB), wb) <= NORM


@pytest.mark.gpu
@pytest.mark.parametrize("rank", [8, 32, 64, 100])
@pytest.mark.parametrize("requests", [1, 30])
def test_low_rank_sums(rank, requests):
    rng = np.random.default_rng([rank, requests])
    n_in, n_out, rows = 1024, 64, 300
    X, W = rounded(rng.standard_normal((rows, n_in)), BF), rounded(rng.standard_normal((n_out, n_in)), BF)
    A, B = rounded(rng.standard_normal((1, rank, n_in)), BF), rounded(rng.standard_normal((1, rank, n_out)), BF)
    off, adapter = np.linspace(0, rows, requests + 1).astype(np.int32), np.zeros(requests, dtype=np.int32)
    U, Y = empty((rows, rank), bp.BP_F32), empty((rows, n_out), BF)
    with bp.Adapters(1, rank, n_in, n_out, BF, max_rows=rows, max_requests=requests) as layer:
        layer.forward(dev(W, BF), None, dev(A, BF), dev(B, BF), None, dev(X, BF), dev(off), dev(adapter), requests, rows, U, Y)
        layer.check()
    assert error(host(U), X @ A[0].T) <= NORM


@pytest.mark.gpu
@pytest.mark.parametrize("rows,n_in,n_out", [(4096, 264, 136), (3000, 512, 512)])
def test_experts_changes(rows, n_in, n_out):
    rng = np.random.default_rng(rows)
    offsets = np.array([0, rows - 1000, rows])
    X, D = rounded(rng.standard_normal((rows, n_in)), BF), rounded(rng.standard_normal((rows, n_out)), BF)
    GW, Gb = empty((2, n_out, n_in), bp.BP_F32), empty((2, n_out), bp.BP_F32)
    with bp.Experts(2, n_in, n_out, BF, max_rows=rows) as layer:
        layer.backward(None, dev(X, BF), rows, None, dev(offsets), rows, dev(D, BF), GW=GW, Gb=Gb)
        layer.check()
    _, (ww, _), (wb, _) = O.experts_backward(np.zeros((2, n_out, n_in)), X, None, offsets, D, False)
    assert error(host(GW), ww) <= NORM and error(host(Gb), wb) <= NORM
