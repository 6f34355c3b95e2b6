"""Expert layers (products grouped by expert) against the float64 oracle: ragged groups, empty
ones, gathered inputs, both dtypes and directions.  The bound is that of expert_cases."""
import numpy as np
import pytest

from expert_cases import assert_sum, dev, empty, host, ragged, rounded
from oracle import experts_oracle as O
from paper_1801_01554_gb300 import bp

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def problem(E, n_in, n_out, rows, dtype, gather, squash, seed, offsets=None):
    rng = np.random.default_rng([seed, E, n_in, n_out, rows])
    offsets = ragged(rng, rows, E) if offsets is None else np.asarray(offsets, dtype=np.int32)
    n_x = max(1, rows // 2) if gather else max(rows, 1)
    x = rng.standard_normal((n_x, n_in))
    X = rounded(O.logistic(x) if squash else x, dtype)
    W = rounded(rng.standard_normal((E, n_out, n_in)) / np.sqrt(n_in), dtype)
    b = rounded(rng.uniform(-0.3, 0.3, (E, n_out)), bp.BP_F32)
    D = rounded(rng.standard_normal((rows, n_out)) * 0.25, dtype)
    source = rng.integers(0, n_x, rows).astype(np.int32) if gather else None
    return X, W, b, D, source, offsets


def check(E, n_in, n_out, rows, dtype, gather=True, squash=False, seed=0, offsets=None):
    X, W, b, D, source, offsets = problem(E, n_in, n_out, rows, dtype, gather, squash, seed, offsets)
    Xd, Wd, bd, Dd, sd, od = dev(X, dtype), dev(W, dtype), dev(b), dev(D, dtype), dev(source), dev(offsets)
    Y, dX = empty((rows, n_out), dtype, 7.0), empty((rows, n_in), dtype, 7.0)
    GW, Gb = empty(W.shape, bp.BP_F32), empty(b.shape, bp.BP_F32)
    with bp.Experts(E, n_in, n_out, dtype, max_rows=max(rows, 1)) as layer:
        layer.forward(Wd, bd, Xd, len(X), sd, od, rows, Y, squash=squash)
        layer.backward(Wd, Xd, len(X), sd, od, rows, Dd, dX=dX, GW=GW, Gb=Gb, squash=squash)
        layer.check()
        inside = np.zeros(rows, dtype=bool)
        inside[offsets[0]:offsets[-1]] = True
        want, mag = O.experts_forward(W, b, X, source, offsets, rows)
        assert_sum(host(Y)[inside], want[inside], mag[inside], dtype, squash, "Y")
        (wx, mx), (ww, mw), (wb, mb) = O.experts_backward(W, X, source, offsets, D, squash)
        assert_sum(host(dX)[inside], wx[inside], mx[inside], dtype, what="dX")
        assert (host(Y)[~inside] == 7).all() and (host(dX)[~inside] == 7).all()   # rows in no group: left alone
        assert_sum(host(GW), ww, mw, bp.BP_F32, what="GW")
        assert_sum(host(Gb), wb, mb, bp.BP_F32, what="Gb")
        if rows:   # a second call adds, without biases and hidden deltas
            layer.backward(None, Xd, len(X), sd, od, rows, Dd, GW=GW, Gb=Gb, squash=squash, accumulate=True)
            layer.forward(Wd, None, Xd, len(X), sd, od, rows, Y)
            layer.check()
            assert_sum(host(GW), 2 * ww, 2 * mw, bp.BP_F32, what="2 GW")
            assert_sum(host(Gb), 2 * wb, 2 * mb, bp.BP_F32, what="2 Gb")
            want, mag = O.experts_forward(W, None, X, source, offsets, rows)
            assert_sum(host(Y)[inside], want[inside], mag[inside], dtype, what="Y without bias")


@pytest.mark.parametrize("E,n_in,n_out,rows", [
    (1, 1, 1, 1), (3, 203, 120, 100), (8, 17, 9, 1), (5, 120, 26, 333), (64, 33, 65, 200), (4, 64, 64, 1000),
    (512, 16, 8, 700), (2, 300, 130, 257)])
@pytest.mark.parametrize("gather,squash", [(True, False), (False, True)])
def test_f32_matches_oracle(E, n_in, n_out, rows, gather, squash):
    check(E, n_in, n_out, rows, bp.BP_F32, gather, squash)


# tiles of 128 in each of the three products, rows on 16-byte boundaries and not; long groups shared out
@pytest.mark.parametrize("E,n_in,n_out,rows", [
    (1, 64, 1280, 2048), (1, 65, 1281, 2047), (1, 1280, 64, 2048), (1, 1281, 63, 2050), (1, 1280, 2048, 300),
    (1, 1281, 2047, 300), (2, 64, 32, 5000), (3, 33, 130, 3000)])
def test_f32_large_tiles_and_shares(E, n_in, n_out, rows):
    check(E, n_in, n_out, rows, bp.BP_F32, True, True, 2)


@pytest.mark.parametrize("dtype", [bp.BP_F32, bp.BP_BF16])
def test_changes_off_32_bytes(dtype):
    """G on a 16-byte boundary that is no 32-byte one (and, float32, inputs on a 4-byte one)."""
    E, n_in, n_out, rows = 2, 264, 136, 300
    X, W, b, D, _, offsets = problem(E, n_in, n_out, rows, dtype, False, False, 13)
    buf = torch.full((E * n_out * n_in + 4,), float("nan"), device="cuda")
    GW, Xd = buf[4:].view(E, n_out, n_in), dev(X, dtype)
    assert GW.data_ptr() % 32 == 16
    if dtype == bp.BP_F32:
        shifted = torch.zeros(X.size + 1, device="cuda")[1:].view(rows, n_in)
        Xd = shifted.copy_(Xd)
    with bp.Experts(E, n_in, n_out, dtype, max_rows=rows) as layer:
        layer.backward(None, Xd, rows, None, dev(offsets), rows, dev(D, dtype), GW=GW)
        layer.check()
    _, (ww, mw), _ = O.experts_backward(W, X, None, offsets, D, False)
    assert_sum(host(GW), ww, mw, bp.BP_F32, what="GW")
    assert torch.isnan(buf[:4]).all()


# rows that end on, before and after 16-, 64- and 128-row blocks; widths off the tiles' 64 and 128
@pytest.mark.parametrize("E,n_in,n_out,rows", [
    (1, 8, 8, 1), (4, 64, 32, 3), (16, 1024, 256, 10), (3, 72, 264, 129), (7, 320, 520, 500), (32, 128, 72, 1000),
    (2, 2048, 136, 300), (5, 136, 2312, 260), (8, 512, 384, 2500), (512, 64, 40, 900), (1, 256, 256, 4097)])
@pytest.mark.parametrize("gather,squash", [(True, False), (True, True), (False, True)])
def test_bf16_matches_oracle(E, n_in, n_out, rows, gather, squash):
    check(E, n_in, n_out, rows, bp.BP_BF16, gather, squash)


@pytest.mark.parametrize("dtype", [bp.BP_F32, bp.BP_BF16])
@pytest.mark.parametrize("offsets,rows", [
    ([0, 0, 0, 0, 0], 0), ([0, 0, 300, 300, 300], 300), ([0, 1, 2, 3, 4], 4), ([0, 64, 128, 192, 193], 193),
    ([0, 127, 255, 383, 512], 512), ([0, 15, 31, 47, 48], 48), ([5, 5, 20, 90, 110], 130),   # rows in no group
    ([0, 1000, 1001, 1001, 1024], 1024)])
def test_group_edges(offsets, rows, dtype):
    check(4, 96, 48, rows, dtype, True, True, 11, offsets)


def test_a_larger_layer_of_many_tiles():
    """More tiles than SMs, rows in the thousands, in both directions."""
    check(6, 1024, 1536, 5000, bp.BP_BF16, True, True, 3)


def test_foreign_rows_do_not_leak():
    """Infinities and NaN in another group's rows, weights and in rows of no group stay there."""
    for dtype in (bp.BP_F32, bp.BP_BF16):
        E, n_in, n_out, rows = 3, 72, 40, 150
        offsets = [0, 37, 101, 140]
        X, W, b, D, _, offsets = problem(E, n_in, n_out, rows, dtype, False, False, 8, offsets)
        bad = slice(37, 101)
        X[bad], D[bad], W[1], b[1] = np.nan, np.inf, np.inf, np.nan
        X[140:], D[140:] = np.inf, np.nan
        Y, dX = empty((rows, n_out), dtype, 7.0), empty((rows, n_in), dtype, 7.0)
        GW, Gb = empty(W.shape, bp.BP_F32), empty(b.shape, bp.BP_F32)
        with bp.Experts(E, n_in, n_out, dtype, max_rows=rows) as layer:
            args = (dev(X, dtype), rows, None, dev(offsets), rows)
            layer.forward(dev(W, dtype), dev(b), *args, Y)
            layer.backward(dev(W, dtype), *args, dev(D, dtype), dX=dX, GW=GW, Gb=Gb)
            layer.check()
        with np.errstate(invalid="ignore", over="ignore"):
            want, mag = O.experts_forward(W, b, X, None, offsets, rows)
            (wx, mx), (ww, mw), (wb, mb) = O.experts_backward(W, X, None, offsets, D, False)
        for part in (slice(0, 37), slice(101, 140)):
            assert_sum(host(Y)[part], want[part], mag[part], dtype, what="Y")
            assert_sum(host(dX)[part], wx[part], mx[part], dtype, what="dX")
        for e in (0, 2):
            assert_sum(host(GW)[e], ww[e], mw[e], bp.BP_F32, what="GW")
            assert_sum(host(Gb)[e], wb[e], mb[e], bp.BP_F32, what="Gb")
        assert not np.isfinite(host(GW)[1]).any()
        assert (host(Y)[140:] == 7).all() and (host(dX)[140:] == 7).all()


@pytest.mark.parametrize("dtype", [bp.BP_F32, bp.BP_BF16])
def test_bad_indexes_are_reported_and_the_layer_stays_usable(dtype):
    E, n_in, n_out, rows = 2, 64, 32, 40
    X, W, b, D, source, offsets = problem(E, n_in, n_out, rows, dtype, True, False, 4, [0, 20, 40])
    args = dev(W, dtype), dev(b), dev(X, dtype), len(X)
    Y = empty((rows, n_out), dtype)
    with bp.Experts(E, n_in, n_out, dtype, max_rows=rows) as layer:
        for bad_source, bad_offsets in ((np.where(np.arange(rows) == 3, len(X), source), offsets),
                                        (np.where(np.arange(rows) == 30, -1, source), offsets),
                                        (source, [0, 20, 41]), (source, [0, 30, 20]), (source, [-5, 20, 40])):
            layer.forward(*args, dev(bad_source), dev(np.asarray(bad_offsets)), rows, Y)
            with pytest.raises(bp.BPError) as e:
                layer.check()
            assert e.value.status == bp.BP_ESTATE
        layer.forward(*args, dev(source), dev(offsets), rows, Y)
        layer.check()
        want, mag = O.experts_forward(W, b, X, source, offsets, rows)
        assert_sum(host(Y), want, mag, dtype)


def test_refusals():
    with bp.Experts(2, 16, 8, bp.BP_BF16, max_rows=4) as layer:
        W, X = torch.zeros(2, 8, 16, device="cuda").bfloat16(), torch.zeros(6, 16, device="cuda").bfloat16()
        Y, off = torch.zeros(6, 8, device="cuda").bfloat16(), torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
        with pytest.raises(bp.BPError) as e:
            layer.forward(W, None, X, 6, None, off, 5, Y)
        assert e.value.status == bp.BP_EINVAL and "n_rows" in str(e.value)
        with pytest.raises(bp.BPError):   # fewer inputs than rows
            layer.forward(W, None, X, 3, None, off, 4, Y)
        with pytest.raises(bp.BPError):   # off a 16-byte boundary
            layer.forward(W, None, X.view(-1)[4:], 5, None, off, 4, Y)
        with pytest.raises(bp.BPError):   # changes need the inputs
            layer.backward(W, None, 4, None, off, 4, Y, GW=torch.zeros(2, 8, 16, device="cuda"))
        with pytest.raises(ValueError):
            layer.forward(W, None, X, 6, None, off, 4, Y[:3])
        with pytest.raises(ValueError):
            layer.forward(W, None, X, 6, None, off.long(), 4, Y)
        layer.forward(W, None, X, 6, None, off, 4, Y)
        layer.check()


def test_same_bits_on_a_side_stream_and_in_a_graph():
    E, n_in, n_out, rows = 5, 256, 192, 700
    X, W, b, D, source, offsets = problem(E, n_in, n_out, rows, bp.BP_BF16, True, True, 6)
    Xd, Wd, bd, Dd = dev(X, bp.BP_BF16), dev(W, bp.BP_BF16), dev(b), dev(D, bp.BP_BF16)
    sd, od = dev(source), dev(offsets)

    def outs():
        return [empty((rows, n_out), bp.BP_BF16, 7.0), empty((rows, n_in), bp.BP_BF16, 7.0), empty(W.shape, bp.BP_F32),
                empty(b.shape, bp.BP_F32)]
    s = torch.cuda.Stream()
    with bp.Experts(E, n_in, n_out, bp.BP_BF16, max_rows=rows) as layer:
        def step(o, stream):
            layer.forward(Wd, bd, Xd, len(X), sd, od, rows, o[0], squash=True, stream=stream)
            layer.backward(Wd, Xd, len(X), sd, od, rows, Dd, dX=o[1], GW=o[2], Gb=o[3], squash=True, stream=stream)
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
