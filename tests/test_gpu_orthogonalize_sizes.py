"""Newton-Schulz orthogonalisation and the Muon step at the sizes where another kernel, or another number of blocks of a cluster, takes
over, against the formulas in 64 bits with the tolerances of test_gpu_orthogonalize."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2202_05008_b200 import muon_step, orthogonalize
from test_gpu_orthogonalize import check, exact, matrix, muon_exact

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# up to 16 rows and 17 to 32 long ones (registers), up to 128 (shared memory), in 1, 2, 4 and 8 blocks; and the first sizes beyond
REGISTERS_16 = [(16, 1024), (9, 1025), (3000, 16), (16, 8192), (4097, 7), (1, 8000)]
REGISTERS_32 = [(31, 129), (17, 144), (30, 145), (24, 200), (192, 32), (20, 193), (32, 512), (513, 18), (700, 20), (32, 2000), (2049, 25), (17, 4000), (4096, 32)]
SHARED = [(33, 600), (100, 1000), (1024, 48), (128, 513), (257, 65)]
BEYOND = [(33, 1025), (1100, 40), (24, 4097), (8200, 5)]


@pytest.mark.parametrize("rows,cols", REGISTERS_16 + REGISTERS_32 + SHARED + BEYOND)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_every_kernel_and_cluster(rows, cols, dtype):
    g = matrix(rows, cols, 3, dtype=dtype)
    check(orthogonalize(g), g)


@pytest.mark.parametrize("rows,cols", [(24, 200), (700, 20), (17, 4000), (9, 5000), (100, 1000)])
def test_batches_strides_in_place_and_what_has_no_direction(rows, cols):
    base = torch.full((5, rows, cols + 3), 7.0, device="cuda")
    x = base[:, :, 1:cols + 1]
    for k in range(5):
        x[k] = matrix(rows, cols, k)
    x[1] = 0.0
    x[2, rows // 2, cols - 1] = float("nan")
    x[3, rows - 1, 0] = float("-inf")
    keep = x.clone()
    got = orthogonalize(x)
    assert (got[1] == 0).all() and got[2].isnan().all() and got[3].isnan().all()
    for k in (0, 4):
        check(got[k], keep[k])
        assert torch.equal(orthogonalize(keep[k]), got[k])
    orthogonalize(x, out=x)
    assert torch.equal(x[[0, 1, 4]], got[[0, 1, 4]]) and x[2:4].isnan().all()
    assert (base[:, :, 0] == 7).all() and (base[:, :, cols + 1:] == 7).all()


@pytest.mark.parametrize("nesterov", [True, False])
def test_muon_steps_of_long_matrices(nesterov):
    sizes, at, matrices = [(24, 200), (700, 20), (32, 2000), (17, 4000), (5000, 9), (1000, 100), (18, 150)], 3, []
    for rows, cols in sizes:
        matrices.append((at, rows, cols))
        at += rows * cols + 1
    gen = torch.Generator(device="cuda").manual_seed(at)
    c, m, v, g = (torch.randn(at, generator=gen, device="cuda") * s for s in (0.3, 1e-3, 1.0, 1e-2))
    v = v.square() * 1e-5
    got = muon_step(c, m, v, g, matrices, 2, lr=0.02, momentum=0.9, nesterov=nesterov, weight_decay=0.1)
    want = muon_exact(c, m, v, g, matrices, 2, 0.02, 0.9, nesterov, 0.1)
    for o, r, k in matrices:
        part = slice(o, o + r * k)
        assert ((got[1][part].double() - want[1][part]).abs() <= 2.0 ** -22 * (m.abs() + g.abs())[part]).all()
        assert torch.equal(got[2][part], v[part])
        # full-rank matrices: 64 x 2^-22 of the step, and 3.4445^5 2^-22 against |O| >= 2; the centre's own rounding
        move = want[3][part]
        err = (got[0][part].double() - want[0][part]).norm()
        assert float(err) <= 2.0 ** -22 * (64 + 243) * float(move.norm()) + 2.0 ** -23 * float(c[part].norm()), (r, k)


@pytest.mark.parametrize("rows,cols", [(20, 160), (192, 17)])
def test_the_first_call_of_a_process_may_be_of_any_size(rows, cols):
    """Kernel attributes that a launch needs are set by that launch, not by one of another size before it."""
    code = ("import torch\nfrom paper_2202_05008_b200 import orthogonalize\n"
            f"x = torch.randn({rows}, {cols}, device='cuda')\nassert orthogonalize(x).isfinite().all()\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-800:]


def test_orthogonal_matrices_of_17_to_32_rows_stay_close_to_orthogonal():
    """The definition itself: the singular values that the steps make of those of G, with G's singular vectors."""
    g = matrix(24, 300, 5)
    u, s, vt = torch.linalg.svd(g.double(), full_matrices=False)
    t = s / (g.double().norm() + 1e-7)
    for _ in range(5):
        t = t * (3.4445 + t * t * (-4.7750 + 2.0315 * t * t))
    want = (u * t) @ vt
    assert float((exact(g) - want).norm() / want.norm()) < 1e-12
    check(orthogonalize(g), g)


@pytest.mark.parametrize("count,rows,cols", [(40, 20, 300), (100, 24, 700), (30, 18, 600), (200, 513, 32), (200, 100, 300), (300, 12, 1500)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_more_matrices_than_run_at_once(count, rows, cols, dtype):
    x = torch.stack([matrix(rows, cols, k, dtype=dtype) for k in range(count)])
    got = orthogonalize(x)
    for k in (0, 1, count // 2, count - 1):
        check(got[k], x[k])
    assert torch.equal(orthogonalize(x), got)
