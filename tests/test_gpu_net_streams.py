"""A net beside a busy default stream: one that was just made, or whose errors were just reported, is ready for a
call on any stream.  Weight changes against the float64 oracle, 1e-5 (float32) and 2e-2 (bfloat16) of the
largest, as the other tests of one update."""
import numpy as np
import pytest

from oracle import bp_oracle as O
from paper_1801_01554_gb300 import bp, synth

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,sizes,bar", [(bp.BP_F32, (203, 60, 26), 1e-5), (bp.BP_BF16, (64, 128, 32), 2e-2)])
def test_new_nets_on_a_side_stream(dtype, sizes, bar):
    batch = 300
    X, T = synth.nettalk_patterns(batch, seed=3) if dtype == bp.BP_F32 else \
        synth.gaussian_patterns(batch, sizes[0], sizes[-1], 0.3, seed=3)
    t = torch.float32 if dtype == bp.BP_F32 else torch.bfloat16
    if dtype == bp.BP_BF16:
        X, T = synth.round_to(X, "bf16"), synth.round_to(T, "bf16")
    Xd, Td = (torch.tensor(v, dtype=torch.float32, device="cuda").to(t) for v in (X, T))
    st = O.State(sizes, np.zeros(O.pack(*O.unpack(sizes, synth.init_uniform(sizes, -0.3, 0.3, 1))).size), lr=0.1, momentum=0.9)
    O.train_batch(st, X, T)
    s = torch.cuda.Stream()
    for _ in range(3):
        torch.cuda.synchronize()
        x = torch.ones(64 << 20, device="cuda")
        torch.cuda.synchronize()
        for _ in range(300):   # some 60 ms, queued
            x.mul_(1.0)
        with bp.Net(sizes, lr=0.1, momentum=0.9, dtype=dtype, max_batch=batch) as net:   # its weights are 0
            net.train_batch(Xd, Td, batch, None, stream=s)
            net.check(stream=s)
            got = net.get_weights()
        assert np.max(np.abs(got - st.theta)) <= bar * np.max(np.abs(st.theta))


def test_an_error_is_cleared_before_the_next_call():
    sizes, batch = (203, 60, 26), 64
    X, T = synth.nettalk_patterns(batch, seed=4)
    bad = X.copy()
    bad[3, 5] = np.nan
    Xd, Bd, Td = (torch.tensor(v, dtype=torch.float32, device="cuda") for v in (X, bad, T))
    theta = synth.round_to(synth.init_uniform(sizes, -0.3, 0.3, 2), "f32")
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    sse = torch.zeros(1, device="cuda")
    x = torch.ones(64 << 20, device="cuda")
    with bp.Net(sizes, lr=0.1, momentum=0.9, max_batch=batch) as net:
        for i in range(4):
            net.set_weights(theta)
            torch.cuda.synchronize()
            for _ in range(300):
                x.mul_(1.0)
            a, b = streams[i % 2], streams[1 - i % 2]
            net.train_batch(Bd, Td, batch, sse, stream=a)
            with pytest.raises(bp.BPError) as e:
                net.check(stream=a)
            assert e.value.status == bp.BP_ENONFINITE
            net.set_weights(theta)
            net.train_batch(Xd, Td, batch, sse, stream=b)
            net.check(stream=b)
