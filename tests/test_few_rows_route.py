"""Which forward calls of bfloat16 experts the kernel of few rows takes (host code, no GPU): those that it is
faster at, by the times beside the rule."""
import os

import pytest

from paper_1801_01554_gb300 import bp, build


@pytest.fixture(scope="module")
def few():
    if not os.path.exists(bp.lib_path()):
        build.build()
    return bp.load().bp_internal_few_experts


@pytest.mark.parametrize("rows,experts,n_in,n_out,want", [
    (1, 16, 4096, 4096, 1), (8, 16, 1024, 1024, 1), (8, 64, 4096, 4096, 1), (12, 16, 1024, 2048, 1),
    (16, 4, 1024, 1024, 1), (32, 8, 512, 512, 1), (16, 16, 2048, 2048, 0), (32, 8, 4096, 256, 1), (64, 16, 4096, 256, 1), (65, 17, 4096, 8, 0), (32, 8, 1024, 2048, 0),
    (48, 16, 2048, 2048, 0), (100, 16, 2048, 2048, 0), (256, 64, 512, 512, 0), (512, 128, 512, 512, 0),
    (1, 1, 256, 4096, 1), (32, 1, 4096, 4096, 1), (64, 1, 4096, 4096, 0), (8, 2, 16384, 64, 1), (8, 2, 16392, 64, 0)])
def test_rule(few, rows, experts, n_in, n_out, want):
    assert few(rows, experts, n_in, n_out) == want
