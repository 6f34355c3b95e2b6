"""Changes of tokens that come very often: the error of a sum does not grow with its rows.

At most 32 rows are added to a piece (31 roundings of 2^-24), pieces 32 at a time (31 for each time over, three for up to 32,768
pieces), and the scale and what was there before add two: 128 * 2^-24 of the magnitudes bounds that.  Calls of up to 4,096 ids
add their 128 pieces one after another: 31 + 127 + 2, 160 * 2^-24; with few tokens 4 pieces a warp and then the 32
warps' sums: 31 + 4 + 32 + 2, 72 * 2^-24 bounds that.
Rows that are all alike are the worst: every addition to a plain sum would be rounded the same way.
"""
import numpy as np
import pytest

from expert_cases import empty, host
from paper_1801_01554_gb300 import bp

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32 = 2.0 ** -24


def rows(n, width, dtype, kind):
    t = torch.bfloat16 if dtype == bp.BP_BF16 else torch.float32
    if kind == "any":
        g = torch.Generator(device="cuda").manual_seed(n + width)
        return torch.rand(n, width, generator=g, device="cuda").to(t)
    return torch.full((n, width), kind, device="cuda").to(t)


@pytest.mark.parametrize("kind", [0.7, 1.1, "any"])
@pytest.mark.parametrize("dtype,width", [(bp.BP_F32, 1), (bp.BP_F32, 36), (bp.BP_F32, 133), (bp.BP_BF16, 8), (bp.BP_BF16, 264)])
@pytest.mark.parametrize("n,V,bound", [(1 << 20, 3, 128), (300001, 40000, 128), (4096, 5000, 160), (4096, 3, 72)])
def test_one_token_for_all(n, V, bound, dtype, width, kind):
    D, G, token = rows(n, width, dtype, kind), empty((V, width), bp.BP_F32), V // 2
    ids = torch.full((n,), token, dtype=torch.int32, device="cuda")
    with bp.Embedding(V, width, dtype, max_ids=n) as layer:
        layer.backward(ids, n, D, G, scale=0.75)
        layer.check()
        want = 0.75 * D.sum(0, dtype=torch.float64).cpu().numpy()
        assert (np.abs(host(G[token]) - want) <= bound * F32 * want).all()   # (all rows are positive)
        assert (G[:token] == 0).all() and (G[token + 1:] == 0).all()
        G.fill_(5.0)
        layer.backward(ids, n, D, G, scale=0.75, accumulate=True)
        layer.check()
        assert (np.abs(host(G[token]) - want - 5.0) <= bound * F32 * (want + 5.0)).all()


@pytest.mark.parametrize("n", [2048, 200000])
def test_infinite_rows_stay_infinite(n):
    """An infinity in a long run of rows is the sum, and a NaN stays one."""
    V, width = 2000, 8
    D = torch.ones(n, width, device="cuda")
    D[n // 2, 1], D[n - 1, 2], D[5, 3] = float("inf"), float("-inf"), float("nan")
    D[7, 4], D[n - 7, 4] = float("inf"), float("-inf")
    G, ids = empty((V, width), bp.BP_F32), torch.full((n,), 1, dtype=torch.int32, device="cuda")
    with bp.Embedding(V, width, bp.BP_F32, max_ids=n) as layer:
        layer.backward(ids, n, D, G)
        layer.check()
    got = host(G[1])
    assert got[1] == np.inf and got[2] == -np.inf and np.isnan(got[3]) and np.isnan(got[4])
    assert (got[[0, 5, 6, 7]] == n).all()
