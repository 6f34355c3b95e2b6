"""A handle for which there is no memory is refused, and the next call on another handle is not: the error is reported
once."""
import numpy as np
import pytest

from expert_cases import dev, empty
from paper_1801_01554_gb300 import bp

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

MANY = 2 ** 31 - 1024
TOO_LARGE = {   # terabytes of scratch or parameters
    "embedding": lambda: bp.Embedding(1 << 24, 1 << 20, bp.BP_F32, max_ids=1 << 26),
    "residual": lambda: bp.Residual(8192, bp.BP_F32, 4, bp.BP_NORM_LAYER, bp.BP_NORM_LAYER, max_gates=MANY),
    "experts": lambda: bp.Experts(1, 1 << 20, 8, bp.BP_BF16, max_rows=MANY),
    "net": lambda: bp.Net([1 << 17] * 9, 0.1, 0.9, bp.BP_BF16, max_batch=128),
}


@pytest.mark.parametrize("large", sorted(TOO_LARGE))
def test_a_refused_handle_leaves_no_error_behind(large):
    table, ids, y = torch.ones(10, 16, device="cuda"), dev(np.arange(8)), empty((8, 16), bp.BP_F32)
    with bp.Embedding(10, 16, bp.BP_F32, max_ids=8) as layer:
        with pytest.raises(bp.BPError) as e:
            TOO_LARGE[large]()
        assert e.value.status == bp.BP_ENOMEM
        layer.forward(table, ids, 8, y)
        layer.check()
        assert (y == 1).all()
