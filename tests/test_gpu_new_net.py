"""A new net's weights are zero until they are set: every unit's output is the logistic of 0, exactly 1/2 in
both types, whatever its memory held before."""
import numpy as np
import pytest

from paper_1801_01554_gb300 import bp

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [bp.BP_F32, bp.BP_BF16])
@pytest.mark.parametrize("before", [64, 300])
def test_weights_start_at_zero(dtype, before):
    sizes = (64, 128, 32)
    t = torch.float32 if dtype == bp.BP_F32 else torch.bfloat16
    X, Y = torch.rand(40, sizes[0], device="cuda").to(t), torch.empty(40, sizes[-1], device="cuda", dtype=t)
    # memory that other nets leave behind, full of other weights, beside nets that keep the driver's blocks in use
    junk = [bp.Net(sizes, lr=0.1, momentum=0.9, dtype=dtype, max_batch=before) for _ in range(24)]
    for net in junk:
        net.set_weights(np.full(net.num_params, 0.5, dtype=np.float32))
        net.forward(X, 40, Y)
        net.train_batch(X, Y, 40)
    torch.cuda.synchronize()
    for net in (net for i, net in enumerate(junk) if i % 3):
        net.close()
    nets = [bp.Net(sizes, lr=0.1, momentum=0.9, dtype=dtype, max_batch=300) for _ in range(16)]
    for net in nets:
        net.forward(X, 40, Y)
        net.check()
        torch.cuda.synchronize()
        assert (net.get_weights() == 0).all() and (Y.float() == 0.5).all()
