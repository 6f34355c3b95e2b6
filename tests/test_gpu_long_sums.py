"""Sums over very many units, in bfloat16: outputs and hidden deltas of layers whose inputs or units are
tens of thousands, against sums in 64 bits.

The tensor cores truncate as they accumulate, so that a sum of positive products comes out too small, by
more the longer one accumulator runs.  The bound of expert_cases holds for sums that are cut into parts of
at most 128 steps: 2^-16 of a sum of positive products.  A bfloat16 result hides that behind its rounding,
2^-8 at most; but the rounding goes either way, so that the mean of N values' relative errors has a standard
deviation of at most 2^-8 / sqrt(3 N), of which five are allowed.  (For that the values must not lie on one
spot of bfloat16's grid, as sums of so many alike products do: rows and units have factors of their own,
their logarithms spread over an octave.)
"""
import math

import numpy as np
import pytest

from expert_cases import SUM, dev, empty
from paper_1801_01554_gb300 import bp

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF = bp.BP_BF16


def positive(seed, *shape):
    """Products' factors [.., rows, K], every row with a factor of its own."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.rand(*shape, generator=g, device="cuda").add_(0.25)
    return x.mul_(torch.rand(*shape[:-1], 1, generator=g, device="cuda").exp2_()).to(torch.bfloat16)


def assert_unbiased(got, want):
    e = (got.double() - want) / want
    bound = SUM + 5 * 2.0 ** -8 / math.sqrt(3 * e.numel())
    assert e.numel() >= 2 ** 16 and abs(float(e.mean())) <= bound, (float(e.mean()), bound)


@pytest.mark.parametrize("gather", [False, True])
def test_experts_outputs(gather):
    K, N, rows = 2 ** 18, 128, 512
    X, W, Y = positive(1, rows, K), positive(2, 1, N, K), empty((rows, N), BF)
    source = torch.randperm(rows, device="cuda").int() if gather else None
    with bp.Experts(1, K, N, BF, max_rows=rows) as layer:
        layer.forward(W, None, X, rows, source, dev(np.array([0, rows])), rows, Y)
        layer.check()
    x = X if source is None else X[source.long()]
    assert_unbiased(Y, x.double() @ W[0].double().t())


def test_experts_hidden_deltas():
    K, N, rows = 2 ** 18, 128, 512
    D, W, dX = positive(3, rows, K), positive(4, N, K).t().contiguous().unsqueeze(0), empty((rows, N), BF)
    with bp.Experts(1, N, K, BF, max_rows=rows) as layer:
        layer.backward(W, None, rows, None, dev(np.array([0, rows])), rows, D, dX=dX)
        layer.check()
    assert_unbiased(dX, D.double() @ W[0].double())


# tiles of one request, of several whose sums are taken apart, and of rows taken one by one
@pytest.mark.parametrize("rank,offsets", [(16, [0, 512]), (16, [0, 50, 300, 512]), (2, [0, 50, 60, 90, 300, 301, 302, 512])])
def test_adapters_outputs_and_hidden_deltas(rank, offsets):
    K, N, rows, n = 2 ** 18, 128, 512, 3
    requests = len(offsets) - 1
    adapter = np.arange(requests) % n
    off, ad = dev(np.array(offsets)), dev(adapter)
    of_row = np.repeat(adapter, np.diff(offsets))
    X, W, Y, U = positive(5, rows, K), positive(6, N, K), empty((rows, N), BF), empty((rows, rank), bp.BP_F32)
    A, B = positive(7, n, rank, K) / K, positive(8, n, rank, N)
    with bp.Adapters(n, rank, K, N, BF, max_rows=rows, max_requests=requests) as layer:
        layer.forward(W, None, A, B, None, X, off, ad, requests, rows, U, Y)
        layer.check()
    want = X.double() @ W.double().t()
    for a in range(n):
        mine = torch.tensor(of_row == a, device="cuda")
        want[mine] += (X[mine].double() @ A[a].double().t()) @ B[a].double()
    assert_unbiased(Y, want)
    D, W, dX = positive(9, rows, K), positive(10, N, K).t().contiguous(), empty((rows, N), BF)
    A, B = positive(11, n, rank, N), positive(12, n, rank, K) / K
    with bp.Adapters(n, rank, N, K, BF, max_rows=rows, max_requests=requests) as layer:
        layer.backward(W, A, B, None, None, None, off, ad, requests, rows, D, dX=dX)
        layer.check()
    want = D.double() @ W.double()
    for a in range(n):
        mine = torch.tensor(of_row == a, device="cuda")
        want[mine] += (D[mine].double() @ B[a].double().t()) @ A[a].double()
    assert_unbiased(dX, want)


def test_outputs_of_a_few_rows():
    K, N, rows = 2 ** 20, 1024, 64
    X, W, Y = positive(13, rows, K), positive(14, 1, N, K), empty((rows, N), BF)
    with bp.Experts(1, K, N, BF, max_rows=rows) as layer:
        layer.forward(W, None, X, rows, None, dev(np.array([0, rows])), rows, Y)
        layer.check()
    assert_unbiased(Y, X.double() @ W[0].double().t())


# few rows a request, each width of the rank's products; many, whose product is another kernel's
@pytest.mark.parametrize("rank", [8, 24, 40, 100])
@pytest.mark.parametrize("rows,requests", [(16, 16), (96, 3), (300, 1)])
def test_low_rank_sums(rank, rows, requests):
    K, N, n = 2 ** 17, 8, 2
    off = torch.linspace(0, rows, requests + 1, device="cuda").int()
    ad = torch.zeros(requests, dtype=torch.int32, device="cuda")
    X, W, A, B = positive(15, rows, K), positive(16, N, K), positive(17, n, rank, K), positive(18, n, rank, N)
    U, Y = empty((rows, rank), bp.BP_F32), empty((rows, N), BF)
    with bp.Adapters(n, rank, K, N, BF, max_rows=rows, max_requests=requests) as layer:
        layer.forward(W, None, A, B, None, X, off, ad, requests, rows, U, Y)
        layer.check()
    want = X.double() @ A[0].double().t()
    assert float(((U.double() - want) / want).abs().max()) <= SUM + 2.0 ** -23
