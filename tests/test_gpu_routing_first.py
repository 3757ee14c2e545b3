"""Routes whose launch is a process's first of its kernel: nothing that an earlier call has set up is there."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

# counters that, with the 128 bytes that a kernel has beside them, are just above what a launch has without asking: pairs and members for one block (one and four pairs a
# lane), a cluster (the same) and the three launches
PROGRAM = """
import torch
from paper_2202_05008_b200 import route_rows
for pairs, groups in ((100, 2042), (2000, 360), (5000, 360), (20000, 360), (40000, 1225)):
    members = torch.randint(-1, groups + 1, (pairs,), device="cuda")
    routes = route_rows(members, groups)
    key = torch.where((members >= 0) & (members < groups), members, groups)
    order = torch.argsort(key, stable=True)
    live = int((key < groups).sum())
    assert routes.offsets[-1] == live and torch.equal(routes.source[:live].long(), order[:live]) and bool((routes.source[live:] == -1).all())
    assert torch.equal(routes.place[order[:live]].long(), torch.arange(live, device="cuda"))
print("all routes")
"""


def test_a_launch_asks_for_its_shared_memory_whatever_ran_before():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    run = subprocess.run([sys.executable, "-c", PROGRAM], cwd=root, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "all routes" in run.stdout, run.stderr[-2000:]
