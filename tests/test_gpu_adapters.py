"""Adapter layers (a shared layer and each request's low-rank change) against the float64 oracle:
requests of one row and of many, without rows, without adapters, adapters shared by requests.
The bound is that of expert_cases."""
import numpy as np
import pytest

from expert_cases import assert_sum, dev, empty, host, ragged, rounded
from oracle import experts_oracle as O
from paper_1801_01554_gb300 import bp

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def problem(n, rank, n_in, n_out, rows, requests, dtype, squash, seed, offsets=None):
    rng = np.random.default_rng([seed, n, rank, n_in, n_out, rows, requests])
    offsets = ragged(rng, rows, requests) if offsets is None else np.asarray(offsets, dtype=np.int32)
    adapter = rng.integers(-1, n, requests).astype(np.int32)
    x = rng.standard_normal((max(rows, 1), n_in))
    return dict(X=rounded(O.logistic(x) if squash else x, dtype),
                W=rounded(rng.standard_normal((n_out, n_in)) / np.sqrt(n_in), dtype),
                b=rounded(rng.uniform(-0.3, 0.3, n_out), bp.BP_F32),
                A=rounded(rng.standard_normal((n, rank, n_in)) / np.sqrt(n_in), dtype),
                B=rounded(rng.standard_normal((n, rank, n_out)) / np.sqrt(rank), dtype),
                scale=rounded(rng.uniform(0.5, 2.0, n), bp.BP_F32),
                D=rounded(rng.standard_normal((max(rows, 1), n_out)) * 0.25, dtype), offsets=offsets, adapter=adapter)


def check(n, rank, n_in, n_out, rows, requests, dtype, squash=False, seed=0, offsets=None, p=None):
    p = problem(n, rank, n_in, n_out, rows, requests, dtype, squash, seed, offsets) if p is None else p
    X, D = p["X"][:rows], p["D"][:rows]
    v = {k: dev(p[k], dtype) for k in ("X", "W", "A", "B", "D")}
    scale, b, off, ad = dev(p["scale"]), dev(p["b"]), dev(p["offsets"]), dev(p["adapter"])
    U, Y, dX = empty((rows, rank), bp.BP_F32), empty((rows, n_out), dtype), empty((rows, n_in), dtype)
    GA, GB = empty((n, rank, n_in), bp.BP_F32), empty((n, rank, n_out), bp.BP_F32)
    with bp.Adapters(n, rank, n_in, n_out, dtype, max_rows=max(rows, 1), max_requests=max(requests, 1)) as layer:
        where = (off, ad, requests, rows)
        layer.forward(v["W"], b, v["A"], v["B"], scale, v["X"], *where, U, Y, squash=squash)
        layer.check()
        (wy, my), (wu, mu) = O.adapters_forward(p["W"], p["b"], p["A"], p["B"], p["scale"], X, p["offsets"], p["adapter"])
        assert_sum(host(Y), wy, my, dtype, squash, "Y")
        assert_sum(host(U), wu, mu, bp.BP_F32, what="U")
        u = host(U)   # the backward pass takes it as an input
        layer.backward(v["W"], v["A"], v["B"], scale, v["X"], U, *where, v["D"], dX=dX, GA=GA, GB=GB, squash=squash)
        layer.check()
        (wx, mx), (wa, ma), (wb, mb) = O.adapters_backward(p["W"], p["A"], p["B"], p["scale"], X, u, p["offsets"],
                                                          p["adapter"], D, squash)
        assert_sum(host(dX), wx, mx, dtype, what="dX")
        assert_sum(host(GA), wa, ma, bp.BP_F32, what="GA")
        assert_sum(host(GB), wb, mb, bp.BP_F32, what="GB")
        if rows:   # without scale and bias; changes added up
            layer.backward(v["W"], v["A"], v["B"], scale, v["X"], U, *where, v["D"], GA=GA, GB=GB, accumulate=True)
            layer.forward(v["W"], None, v["A"], v["B"], None, v["X"], *where, U, Y)
            layer.check()
            assert_sum(host(GA), 2 * wa, 2 * ma, bp.BP_F32, what="2 GA")
            assert_sum(host(GB), 2 * wb, 2 * mb, bp.BP_F32, what="2 GB")
            (wy, my), _ = O.adapters_forward(p["W"], None, p["A"], p["B"], None, X, p["offsets"], p["adapter"])
            assert_sum(host(Y), wy, my, dtype, what="Y without scale")


@pytest.mark.parametrize("n,rank,n_in,n_out,rows,requests", [
    (1, 1, 1, 1, 1, 1), (3, 4, 203, 120, 100, 5), (5, 16, 64, 64, 300, 3), (2, 100, 33, 17, 65, 9), (40, 8, 96, 26, 64, 64),
    (4, 128, 120, 130, 200, 2)])
@pytest.mark.parametrize("squash", [False, True])
def test_f32_matches_oracle(n, rank, n_in, n_out, rows, requests, squash):
    check(n, rank, n_in, n_out, rows, requests, bp.BP_F32, squash)


# tiles of 128 with one request and with several; changes of long requests shared out
@pytest.mark.parametrize("n,rank,n_in,n_out,rows,requests", [
    (3, 24, 64, 1280, 2048, 3), (3, 24, 1280, 64, 2048, 3), (2, 8, 64, 48, 3000, 2)])
def test_f32_large_tiles_and_shares(n, rank, n_in, n_out, rows, requests):
    check(n, rank, n_in, n_out, rows, requests, bp.BP_F32, True, 3)


@pytest.mark.parametrize("n,rank,n_in,n_out,rows,requests", [
    (1, 100, 256, 192, 3000, 2), (2, 17, 512, 64, 4000, 3), (1, 64, 64, 4096, 2500, 1)])
def test_bf16_changes_shared_out(n, rank, n_in, n_out, rows, requests):
    check(n, rank, n_in, n_out, rows, requests, bp.BP_BF16, False, 4)


@pytest.mark.parametrize("dtype", [bp.BP_F32, bp.BP_BF16])
def test_a_bad_adapter_is_reported_by_a_change_alone(dtype):
    rows = 40
    p = problem(2, 8, 64, 32, rows, 2, dtype, False, 4, [0, 20, 40])
    U, GB = torch.zeros(rows, 8, device="cuda"), empty((2, 8, 32), bp.BP_F32)
    with bp.Adapters(2, 8, 64, 32, dtype, max_rows=rows, max_requests=2) as layer:
        layer.backward(None, None, None, None, None, U, dev(p["offsets"]), dev(np.array([0, 2])), 2, rows, dev(p["D"], dtype),
                       GB=GB)
        with pytest.raises(bp.BPError) as e:
            layer.check()
        assert e.value.status == bp.BP_ESTATE


@pytest.mark.parametrize("n,rank,n_in,n_out,rows,requests", [
    (1, 1, 8, 8, 1, 1), (7, 16, 256, 128, 1, 1), (50, 16, 1024, 264, 61, 61), (9, 8, 128, 64, 16, 16), (6, 32, 512, 392, 700, 11),
    (5, 64, 264, 520, 1025, 7), (3, 5, 72, 136, 130, 4), (2, 128, 320, 256, 400, 3), (4, 100, 136, 72, 257, 5),
    (200, 12, 256, 192, 300, 300), (3, 33, 2048, 64, 150, 2), (4, 16, 64, 2056, 90, 30), (1, 24, 512, 512, 3000, 1)])
@pytest.mark.parametrize("squash", [False, True])
def test_bf16_matches_oracle(n, rank, n_in, n_out, rows, requests, squash):
    check(n, rank, n_in, n_out, rows, requests, bp.BP_BF16, squash)


@pytest.mark.parametrize("dtype", [bp.BP_F32, bp.BP_BF16])
@pytest.mark.parametrize("offsets", [
    [0, 0, 0], [0, 0, 5, 5, 5, 9], [0, 1, 2, 3, 4], [0, 64, 128, 192], [0, 127, 128, 129, 256, 300], [0, 15, 16, 17, 33],
    [0, 300], [0, 100, 100, 101, 290]])
def test_request_edges(offsets, dtype):
    check(3, 16, 96, 72, offsets[-1], len(offsets) - 1, dtype, True, 21, offsets)


def test_no_requests_is_the_shared_layer():
    for dtype in (bp.BP_F32, bp.BP_BF16):
        check(2, 8, 64, 48, 70, 0, dtype, False, 5, [0])


def test_rows_outside_requests_get_the_shared_layer():
    for dtype in (bp.BP_F32, bp.BP_BF16):
        p = problem(2, 8, 64, 48, 150, 2, dtype, False, 6, [20, 70, 140])
        p["adapter"][:] = [1, 0]
        check(2, 8, 64, 48, 150, 2, dtype, p=p)


def test_larger_layer_of_many_tiles():
    check(5, 48, 1024, 1536, 5000, 6, bp.BP_BF16, True, 2)


@pytest.mark.parametrize("dtype", [bp.BP_F32, bp.BP_BF16])
def test_more_requests_than_a_table_holds(dtype):
    """700 requests in 1,500 rows: blocks of rows with many requests, and the long list of them."""
    check(3, 16, 128, 64, 1500, 700, dtype, True, 31)


def test_few_adapters_of_many_rows_and_many_without_any():
    """Changes whose rows are shared out, beside adapters that nobody asks for."""
    p = problem(40, 40, 192, 136, 5000, 4, bp.BP_BF16, False, 17)
    p["adapter"][:] = [7, -1, 7, 39]
    check(40, 40, 192, 136, 5000, 4, bp.BP_BF16, p=p)


def test_one_long_request_among_single_rows():
    offsets = list(range(0, 90)) + [700] + list(range(701, 760))
    check(9, 24, 264, 136, offsets[-1], len(offsets) - 1, bp.BP_BF16, True, 18, offsets)


def test_other_requests_do_not_leak():
    """NaN rows and an infinite adapter of one request stay in it."""
    for dtype in (bp.BP_F32, bp.BP_BF16):
        n, rank, n_in, n_out, rows = 3, 24, 128, 72, 150
        offsets = np.array([0, 37, 101, 150], dtype=np.int32)
        p = problem(n, rank, n_in, n_out, rows, 3, dtype, False, 8, offsets)
        p["adapter"][:] = [0, 1, 2]
        p["X"][37:101], p["D"][37:101], p["A"][1], p["B"][1] = np.nan, np.nan, np.inf, np.inf
        v = {k: dev(p[k], dtype) for k in ("X", "W", "A", "B", "D")}
        U, Y, dX = empty((rows, rank), bp.BP_F32), empty((rows, n_out), dtype), empty((rows, n_in), dtype)
        GA, GB = empty((n, rank, n_in), bp.BP_F32), empty((n, rank, n_out), bp.BP_F32)
        with bp.Adapters(n, rank, n_in, n_out, dtype, max_rows=rows, max_requests=3) as layer:
            where = (dev(p["offsets"]), dev(p["adapter"]), 3, rows)
            layer.forward(v["W"], dev(p["b"]), v["A"], v["B"], dev(p["scale"]), v["X"], *where, U, Y)
            layer.backward(v["W"], v["A"], v["B"], dev(p["scale"]), v["X"], U, *where, v["D"], dX=dX, GA=GA, GB=GB)
            layer.check()
        with np.errstate(invalid="ignore", over="ignore"):
            (wy, my), (wu, mu) = O.adapters_forward(p["W"], p["b"], p["A"], p["B"], p["scale"], p["X"], offsets, p["adapter"])
            (wx, mx), (wa, ma), (wb, mb) = O.adapters_backward(p["W"], p["A"], p["B"], p["scale"], p["X"], host(U), offsets,
                                                              p["adapter"], p["D"], False)
        for q in (slice(0, 37), slice(101, 150)):
            assert_sum(host(Y)[q], wy[q], my[q], dtype, what="Y")
            assert_sum(host(U)[q], wu[q], mu[q], bp.BP_F32, what="U")
            assert_sum(host(dX)[q], wx[q], mx[q], dtype, what="dX")
        for a in (0, 2):
            assert_sum(host(GA)[a], wa[a], ma[a], bp.BP_F32, what="GA")
            assert_sum(host(GB)[a], wb[a], mb[a], bp.BP_F32, what="GB")


@pytest.mark.parametrize("dtype", [bp.BP_F32, bp.BP_BF16])
def test_bad_indexes_are_reported(dtype):
    rows = 40
    p = problem(2, 8, 64, 32, rows, 2, dtype, False, 4, [0, 20, 40])
    p["adapter"][:] = [0, 1]
    v = {k: dev(p[k], dtype) for k in ("X", "W", "A", "B")}
    U, Y = empty((rows, 8), bp.BP_F32), empty((rows, 32), dtype)
    with bp.Adapters(2, 8, 64, 32, dtype, max_rows=rows, max_requests=2) as layer:
        for off, ad in (([0, 20, 40], [0, 2]), ([0, 20, 40], [-2, 1]), ([0, 20, 44], [0, 1]), ([0, 45, 40], [0, 1])):
            layer.forward(v["W"], None, v["A"], v["B"], None, v["X"], dev(np.array(off)), dev(np.array(ad)), 2, rows, U, Y)
            with pytest.raises(bp.BPError) as e:
                layer.check()
            assert e.value.status == bp.BP_ESTATE
        layer.forward(v["W"], None, v["A"], v["B"], None, v["X"], dev(p["offsets"]), dev(p["adapter"]), 2, rows, U, Y)
        layer.check()
        (wy, my), _ = O.adapters_forward(p["W"], None, p["A"], p["B"], None, p["X"], p["offsets"], p["adapter"])
        assert_sum(host(Y), wy, my, dtype)


def test_refusals():
    with bp.Adapters(2, 4, 16, 8, bp.BP_BF16, max_rows=4, max_requests=2) as layer:
        W, A, B = (torch.zeros(s, device="cuda").bfloat16() for s in ((8, 16), (2, 4, 16), (2, 4, 8)))
        X, U, Y = torch.zeros(6, 16, device="cuda").bfloat16(), torch.zeros(6, 4, device="cuda"), torch.zeros(6, 8, device="cuda").bfloat16()
        off, ad = torch.tensor([0, 2, 4, 5], dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
        for requests, rows, word in ((3, 4, "n_requests"), (2, 5, "n_rows"), (-1, 4, "n_requests")):
            with pytest.raises(bp.BPError) as e:
                layer.forward(W, None, A, B, None, X, off, ad, requests, rows, U, Y)
            assert e.value.status == bp.BP_EINVAL and word in str(e.value)
        with pytest.raises(bp.BPError):
            layer.forward(W, None, A, None, None, X, off, ad, 2, 4, U, Y)
        with pytest.raises(bp.BPError):   # its change needs U
            layer.backward(W, A, B, None, X, None, off, ad, 2, 4, Y, GB=torch.zeros(2, 4, 8, device="cuda"))
        with pytest.raises(ValueError):
            layer.forward(W, None, A, B, None, X, off, ad, 2, 4, U[:2], Y)
        layer.forward(W, None, A, B, None, X, off, ad, 2, 4, U, Y)
        layer.check()


def test_same_bits_on_a_side_stream_and_in_a_graph():
    rows, requests, n, rank, n_in, n_out = 600, 9, 4, 16, 256, 192
    p = problem(n, rank, n_in, n_out, rows, requests, bp.BP_BF16, True, 6)
    v = {k: dev(p[k], bp.BP_BF16) for k in ("X", "W", "A", "B", "D")}
    scale, b, where = dev(p["scale"]), dev(p["b"]), (dev(p["offsets"]), dev(p["adapter"]), requests, rows)

    def outs():
        return [empty((rows, rank), bp.BP_F32), empty((rows, n_out), bp.BP_BF16), empty((rows, n_in), bp.BP_BF16),
                empty((n, rank, n_in), bp.BP_F32), empty((n, rank, n_out), bp.BP_F32)]
    s = torch.cuda.Stream()
    with bp.Adapters(n, rank, n_in, n_out, bp.BP_BF16, max_rows=rows, max_requests=requests) as layer:
        def step(o, stream):
            layer.forward(v["W"], b, v["A"], v["B"], scale, v["X"], *where, o[0], o[1], squash=True, stream=stream)
            layer.backward(v["W"], v["A"], v["B"], scale, v["X"], o[0], *where, v["D"], dX=o[2], GA=o[3], GB=o[4],
                           squash=True, stream=stream)
        a, c, d = outs(), outs(), outs()
        torch.cuda.synchronize()
        step(a, None)
        torch.cuda.synchronize()
        step(c, s)
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            step(d, s)
        g.replay()
        torch.cuda.synchronize()
        layer.check()
    for x, y, z in zip(a, c, d):
        assert torch.equal(x, y) and torch.equal(x, z)
