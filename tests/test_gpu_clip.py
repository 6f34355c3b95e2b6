"""Clipping against the float64 oracle.

Squares are added up 32 at a time in float32 (33 roundings of 2^-24 of a positive sum), beyond that in float64: 17 * 2^-24 of the
norm, one more for its float32 value; a value is multiplied by a factor that is as far off and rounded, and
rounded: 20 * 2^-24 of itself, and half a unit of bfloat16.
"""
import numpy as np
import pytest

from expert_cases import BF16, dev, host, rounded
from oracle import blocks_oracle as O
from paper_1801_01554_gb300 import bp

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

NORM, VALUE = 18 * 2.0 ** -24, 20 * 2.0 ** -24


def check(values, dtypes, max_norm, outputs=None, offset=0, twice=True):
    """values: float64 arrays that the types hold; outputs None: in place, else offset of the outputs in their memory."""
    def memory(i, shift, fill):
        size = values[i].size
        t = torch.full((size + 32,), fill, device="cuda", dtype=torch.bfloat16 if dtypes[i] == bp.BP_BF16 else torch.float32)
        return t, t[shift:shift + size]
    buf, ins = zip(*(memory(i, offset if outputs is None else (i * 3) % 7, 7.0) for i in range(len(values))))
    for x, v, t in zip(ins, values, dtypes):
        x.copy_(dev(v, t).view(-1))
    outbuf, outs = (None, None) if outputs is None else zip(*(memory(i, (i * 5 + outputs) % 8, 9.0) for i in range(len(values))))
    norm = torch.full((1,), -1.0, device="cuda")
    with bp.Clip(ins, outs) as clip:
        clip.run(max_norm, norm)
        clip.check()
        want, clipped = O.clip(values, max_norm)
        assert abs(float(norm) - want) <= NORM * want + 1e-45
        for i, (x, w, v) in enumerate(zip(ins if outs is None else outs, clipped, values)):
            half = BF16 if dtypes[i] == bp.BP_BF16 else 0.0
            if want > max_norm:
                assert (np.abs(host(x) - w.ravel()) <= (VALUE + half) * np.abs(w.ravel()) + 1e-38).all()
            elif np.isfinite(max_norm) or outs is None:
                assert (host(x) == v.ravel()).all()
            else:
                assert (x == 9).all()   # the norm alone
        for b, x, fill in [(b, x, 7) for b, x in zip(buf, ins)] + ([] if outs is None else [(b, x, 9) for b, x in zip(outbuf, outs)]):
            rest = torch.ones_like(b, dtype=torch.bool)
            at = (x.data_ptr() - b.data_ptr()) // b.element_size() if x.numel() else 0
            rest[at:at + x.numel()] = False
            assert (b[rest] == fill).all()   # what lies around
        if outs is not None and twice:
            kept = [x.clone() for x in outs]
            for x in outs:
                x.fill_(0)
            clip.run(max_norm, norm)
            torch.cuda.synchronize()
            for a, b in zip(kept, outs):
                assert torch.equal(a, b) or max_norm == np.inf
    return float(norm)


def make(rng, sizes, kind):
    dtypes = [bp.BP_F32 if kind == "f32" or (kind == "both" and i % 2) else bp.BP_BF16 for i in range(len(sizes))]
    return [rounded(rng.standard_normal(s) * 10.0 ** rng.uniform(-3, 0), t) for s, t in zip(sizes, dtypes)], dtypes


SIZES = [[1], [0, 3], [5, 0, 1, 33], [8192], [8191, 8193], [27000, 120, 3120, 26], [70001, 7, 64000, 1, 2, 3, 300000], [1] * 300,
         [9] * 2000, [1500007, 999]]


@pytest.mark.parametrize("kind", ["f32", "bf16", "both"])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{sum(s)}")
def test_clip_matches_oracle(sizes, kind):
    rng = np.random.default_rng([len(sizes), sum(sizes)])
    values, dtypes = make(rng, sizes, kind)
    norm = O.clip(values, np.inf)[0]
    for max_norm in (norm / 3, norm * 3, 0.0, np.inf):
        for outputs in (None, 0, 3) if len(sizes) < 100 else (None,) if max_norm == norm * 3 else (3,):
            check(values, dtypes, max_norm, outputs, offset=1)
    check(values, dtypes, norm / 3, None, offset=0)


@pytest.mark.parametrize("scale", [1e-42, 3e-39, 1e-30, 1e-19, 1e18, 1e30, 1e36])
def test_squares_beyond_float32(scale):
    """Squares that vanish or overflow in float32, alone and beside others."""
    rng = np.random.default_rng(1)
    a = rounded(rng.standard_normal(10001) * scale, bp.BP_F32)
    b = rounded(rng.standard_normal(9000), bp.BP_BF16)
    norm = O.clip([a], np.inf)[0]
    check([a], [bp.BP_F32], float(np.float32(norm / 4)), 0)
    check([a, b], [bp.BP_F32, bp.BP_BF16], 0.5, 0)
    a[::7] = 0.0
    a[1::3] *= 2.0 ** -30   # large and small ones beside one another
    a = rounded(a, bp.BP_F32)
    check([a], [bp.BP_F32], np.inf, None)
    check([np.zeros(777), a], [bp.BP_F32, bp.BP_F32], np.inf, 0)


def test_zeros():
    assert check([np.zeros(10000), np.zeros(3)], [bp.BP_F32, bp.BP_BF16], 0.0, 0) == 0.0


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("sizes", [[100, 50], [300000, 50]])
def test_values_that_are_not_finite_clip_nothing(bad, sizes):
    for where in (0, 1):
        x = [torch.ones(s, device="cuda") for s in sizes]
        x[where][-1] = bad
        out = [torch.zeros_like(t) for t in x]
        norm = torch.zeros(1, device="cuda")
        with bp.Clip(x, out) as clip:
            clip.run(1.0, norm)
            with pytest.raises(bp.BPError) as e:
                clip.check()
            assert e.value.status == bp.BP_ENONFINITE and not np.isfinite(float(norm))
            for a, b in zip(x, out):
                assert torch.equal(a.nan_to_num(1e9), b.nan_to_num(1e9))
            x[where][-1] = 1.0
            clip.run(1.0, norm)
            clip.check()
            assert abs(float(norm) - sum(sizes) ** 0.5) < 1e-3


def test_one_input_twice():
    """A change that two places share may be counted twice, with outputs of their own."""
    x, o = torch.full((1000,), 3.0, device="cuda"), [torch.zeros(1000, device="cuda") for _ in range(2)]
    norm = torch.zeros(1, device="cuda")
    with bp.Clip([x, x], o) as clip:
        clip.run(1.0, norm)
        clip.check()
    want = np.sqrt(2000 * 9.0)
    assert abs(float(norm) - want) <= NORM * want
    assert all(np.abs(host(y) - 3.0 / want).max() <= VALUE * 3.0 / want for y in o)


@pytest.mark.parametrize("sizes", [[300, 20], [400000, 77, 900000]])
def test_replayed_for_other_values(sizes):
    rng = np.random.default_rng(2)
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    x, norm = [torch.zeros(n, device="cuda") for n in sizes], torch.zeros(1, device="cuda")
    with bp.Clip(x) as clip:
        with torch.cuda.graph(graph, stream=s):
            clip.run(2.0, norm, stream=s)
        for scale in (1.0, 1e-4, 5.0):
            values = [rounded(rng.standard_normal(n) * scale, bp.BP_F32) for n in sizes]
            for a, b in zip(x, values):
                a.copy_(dev(b))
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                graph.replay()
            clip.check(s)
            want, out = O.clip(values, 2.0)
            assert abs(float(norm) - want) <= NORM * want
            for a, b in zip(x, out):
                assert (np.abs(host(a) - b) <= VALUE * np.abs(b) + 1e-38).all()
        del graph


def test_clip_refuses():
    x = torch.ones(10, device="cuda")
    with bp.Clip([x]) as clip:
        for bad in (-1.0, float("nan")):
            with pytest.raises(bp.BPError) as e:
                clip.run(bad)
            assert e.value.status == bp.BP_EINVAL and "max_norm" in str(e.value)
        with pytest.raises(ValueError):
            clip.run(1.0, x.double())
    for tensors, outputs in (([x.double()], None), ([x], [x.bfloat16()]), ([x], [x[:9]]), ([x, x], [x]), ([x[::2]], None), ([x.cpu()], None)):
        with pytest.raises(ValueError):
            bp.Clip(tensors, outputs)
    with pytest.raises(bp.BPError):
        bp.Clip([x, x])   # in place, twice
    with pytest.raises(bp.BPError):
        bp.Clip([x[:5]], [x[1:6]])
