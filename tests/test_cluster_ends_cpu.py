"""A block of a cluster may end only when no other reads its shared memory any more: read in the sources, no GPU needed."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2501_17086_b200", "csrc")


def test_cluster_barriers_order_the_reads_before_them():
    """A relaxed arrival orders nothing: a read of another block's shared memory may still be under way when that block ends."""
    for name in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, name)) as f:
            assert not re.search(r"barrier\.cluster\.arrive\.relaxed", f.read()), name
