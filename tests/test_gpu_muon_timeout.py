"""A device-side wait of the Muon step that runs out: reported, NaN in the whole matrix that depends on it, everything else as ever."""
import pytest
import torch

from paper_2202_05008_b200 import Solver, workloads as W
from paper_2202_05008_b200.binding import DEBUG_DROP_COMPLETION

pytestmark = pytest.mark.gpu

# the first matrix in one block, in clusters of 2, 4 and 8, and one that takes a launch per product
SIZES = [(28, 128, 128, 8), (150, 100, 5), (120, 300, 3), (100, 700, 64, 8), (300, 200, 3)]


def _workload(sizes):
    return W.Workload("timeout", 16, W.mlp_param_count(sizes), seed=3, lr=0.02, policy_kind=W.POLICY_MLP, layer_sizes=sizes, optimizer=W.OPT_MUON)


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "-".join(map(str, s)))
def test_a_wait_that_runs_out_leaves_nan_in_its_matrix_and_nowhere_else(sizes):
    """With EVO_DEBUG_DROP_COMPLETION the first block of a launch never hears of its first product, and with a limit of 2^23 clocks gives up after some
    four milliseconds; it and, in a cluster, the blocks that it shares a matrix with return by themselves."""
    w = _workload(sizes)
    first = sizes[0] * sizes[1]
    plain, s = Solver(w), Solver(w, wait_cycles_log2=23, debug_flags=DEBUG_DROP_COMPLETION)
    fitness = torch.tensor(W.synthetic_fitness(w.seed, 0, w.pop_size), device="cuda")
    for x in (plain, s):
        x.ask()
        x.tell(fitness)
    assert plain.sync_status() == 0
    assert s.sync_status() == 6 and s.sync_status() == 0          # EVO_ERR_TIMEOUT, once
    assert s.center()[:first].isnan().all() and torch.equal(s.center()[first:], plain.center()[first:])
    assert all(torch.equal(x, y) for x, y in zip(s.moments(), plain.moments())) and s.counters() == (1, 1)
    s.close()
    # the device is as it was
    plain.ask()
    plain.tell(fitness)
    assert plain.sync_status() == 0 and plain.center().isfinite().all()
    plain.close()
