"""What one launch writes and the next one reads: kernels that start while the launch before them still runs (they
wait for it inside) read its results with ordinary loads or from L2, not through the read-only cache, which is for data
that stays as it is for as long as the kernel runs."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1801_01554_gb300", "csrc")
# scratch that a launch leaves for the next one: ids in order, counts, partial sums
WRITTEN = {"bp_embed.cu": ("keys", "g.ids_in_order", "g.partial", "g.arrived"),
           "bp_route.cu": ("h", "g.hist", "g.expert"),
           "bp_residual.cu": ("from", "from2", "g.A", "g.B", "g.C", "g.D", "g.W", "g.WB"),
           "bp_clip.cu": ("g.partial", "g.total", "g.arrived")}


def test_the_files_are_there():
    assert set(WRITTEN) <= {os.path.basename(f) for f in glob.glob(os.path.join(CSRC, "*.cu"))}


@pytest.mark.parametrize("name", sorted(WRITTEN))
def test_results_of_an_earlier_launch_are_not_read_as_constants(name):
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    assert "pdl_wait()" in text
    reads = re.findall(r"__ldg\(\s*([\w.]+)", text)
    assert reads == [] or not set(reads) & set(WRITTEN[name]), sorted(set(reads) & set(WRITTEN[name]))
