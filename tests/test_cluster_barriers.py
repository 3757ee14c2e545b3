"""Barriers of a cluster in their aligned form are for warps that come to them as one: what the sources show of it."""
import glob
import os

from paper_2202_05008_b200 import build as B


def test_a_warp_is_brought_together_in_front_of_every_aligned_cluster_barrier():
    found = 0
    for path in sorted(glob.glob(os.path.join(B.CSRC, "*.cu*"))):
        with open(path) as f:
            lines = f.read().splitlines()
        for n, line in enumerate(lines):
            if "barrier.cluster." in line and ".aligned" in line:
                found += 1
                assert line.strip().startswith("asm volatile") and lines[n - 1].strip().startswith("__syncwarp();"), (os.path.basename(path), n + 1, lines[n - 1])
    assert found >= 7
