"""Newton-Schulz orthogonalisation and the Muon step against the same formulas in 64 bits.

Tolerances (2-norm of the difference over that of the result).  A step rounds its operands to 22 bits (2^-23 relative, drops
products below 2^-22) and sums in fp32; what a step loses is relative to its own X, and X grows by at most a = 3.4445 a step.  Errors
in the span of X stay relative to it: a few 2^-22 for each of the 3 products of 5 steps, 64 x 2^-22 in all.  Errors in the null space of X
grow by a each step and are not held down there: a^5 2^-22 |X0|_F (= 1) against |O|_F.  The result is rounded once to its type."""
import math

import pytest
import torch

from paper_2202_05008_b200 import EvoError, muon_step, orthogonalize

pytestmark = pytest.mark.gpu
ABC = (3.4445, -4.7750, 2.0315)


def exact(g, steps=5, abc=ABC, eps=1e-7):
    a, b, c = abc
    x = g.double()
    x = x / (x.norm() + eps)
    flip = x.shape[0] < x.shape[1]
    x = x.t() if flip else x
    eye = torch.eye(x.shape[1], dtype=torch.float64, device=x.device)
    for _ in range(steps):
        s = x.t() @ x
        x = x @ (a * eye + s @ (b * eye + c * s))
    return x.t() if flip else x


def tolerance(want, dtype):
    return 2.0 ** -22 * (64 + 3.4445 ** 5 / max(float(want.norm()), 1e-30)) + (0 if dtype == torch.float32 else torch.finfo(dtype).eps / 2)


def check(got, g, **kw):
    want = exact(g, **kw)
    err = float((got.double() - want).norm() / want.norm())
    assert err <= tolerance(want, got.dtype), (tuple(g.shape), g.dtype, err)


def matrix(rows, cols, seed=0, dtype=torch.float32, scale=0.01):
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + rows * 31 + cols)
    return (torch.randn(rows, cols, generator=gen, device="cuda") * scale).to(dtype)


SMALL = [(1, 1), (1, 7), (9, 1), (2, 3), (15, 17), (16, 16), (33, 31), (64, 64), (28, 128), (128, 128), (128, 129), (127, 257), (256, 128),
         (12, 512), (1, 3000), (2047, 9)]
LARGE = [(129, 129), (128, 300), (130, 1000), (300, 200), (257, 513), (640, 640), (1000, 130)]


@pytest.mark.parametrize("rows,cols", SMALL + LARGE)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_sizes_and_types(rows, cols, dtype):
    g = matrix(rows, cols, dtype=dtype)
    got = orthogonalize(g)
    assert got.dtype == dtype and got.shape == g.shape
    check(got, g)


@pytest.mark.parametrize("rows,cols", [(48, 96), (200, 260)])
def test_steps_coefficients_and_eps(rows, cols):
    g = matrix(rows, cols, 1)
    for steps in (1, 2, 7):
        check(orthogonalize(g, steps=steps), g, steps=steps)
    for abc in ((1.5, -0.5, 0.0), (2.0, -1.5, 0.5), (3.4445, -4.7750, 2.0315)):
        check(orthogonalize(g, coefficients=abc, steps=6), g, abc=abc, steps=6)
    check(orthogonalize(g, eps=0.5), g, eps=0.5)          # an eps that matters


@pytest.mark.parametrize("rows,cols", [(40, 24), (150, 400)])
def test_batches_strides_and_in_place(rows, cols):
    base = torch.empty(3, rows + 2, cols + 5, device="cuda").fill_(7.0)
    x = base[:, 1:rows + 1, 3:cols + 3]
    for k in range(3):
        x[k] = matrix(rows, cols, k, scale=10.0 ** (3 * k - 3))
    before = base.clone()
    got = orthogonalize(x)
    out = torch.full((3, rows, cols + 9), -3.0, device="cuda")
    view = out[:, :, 4:cols + 4]
    assert orthogonalize(x, out=view) is view
    assert torch.equal(view, got) and torch.equal(base, before)
    assert (out[:, :, :4] == -3.0).all() and (out[:, :, cols + 4:] == -3.0).all()
    for k in range(3):
        check(got[k], x[k])
        assert torch.equal(orthogonalize(x[k]), got[k])
    orthogonalize(x, out=x)
    assert torch.equal(x, got)
    x.copy_(before[:, 1:rows + 1, 3:cols + 3])
    assert torch.equal(base, before)                    # nothing beside the matrices was written


@pytest.mark.parametrize("rows,cols", [(20, 50), (140, 260)])
def test_what_has_no_direction(rows, cols):
    x = torch.stack([matrix(rows, cols, k) for k in range(6)])
    x[1] = 0.0
    x[2, 3, 4] = float("nan")
    x[3, 0, 0] = float("inf")
    x[4] *= 1e30                                          # squares beyond fp32
    x[5] = torch.where(torch.arange(cols, device="cuda") < 2, x[5], torch.zeros(()).cuda())      # rank 2
    got = orthogonalize(x)
    assert (got[1] == 0).all() and got[2].isnan().all() and got[3].isnan().all()
    for k in (0, 4, 5):
        check(got[k], x[k])


def test_a_matrix_near_the_smallest_numbers():
    x = matrix(30, 30) * 1e-42
    got, want = orthogonalize(x), exact(x)                # far below eps: stays small
    assert float((got.double() - want).abs().max()) <= 2.0 ** -20 * float(want.abs().max()) + 1e-38


@pytest.mark.parametrize("rows,cols", [(64, 64), (256, 300)])
def test_streams_graphs_and_repetition(rows, cols):
    x, y = matrix(rows, cols, 1), matrix(rows, cols, 2)
    a, b = orthogonalize(x), orthogonalize(y)
    for _ in range(3):
        assert torch.equal(orthogonalize(x), a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c = orthogonalize(y, stream=side)
    d = orthogonalize(x)                                   # both at once
    side.synchronize()
    torch.cuda.current_stream().synchronize()
    assert torch.equal(c, b) and torch.equal(d, a)
    static, graphs, outs = x.clone(), [], []
    for _ in range(2):                                     # two graphs, each with a workspace of its own pool
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(orthogonalize(static))
        graphs.append(g)
    for value, want in ((y, b), (x, a)):
        static.copy_(value)
        for g in graphs:
            g.replay()
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


def test_python_refusals():
    x = matrix(8, 8)
    for bad in (x.cpu(), x.double(), x[0], x.t(), x[None, None], matrix(8, 16)[:, ::2]):
        with pytest.raises(EvoError):
            orthogonalize(bad)
    for kw in (dict(steps=0), dict(steps=65), dict(eps=0.0), dict(coefficients=(0, 0, 0)), dict(out=torch.empty(8, 9, device="cuda")),
               dict(out=x.bfloat16()), dict(coefficients=(9.0, 9.0, 9.0))):
        with pytest.raises(EvoError):
            orthogonalize(x, **kw)
    assert orthogonalize(torch.empty(0, 4, 4, device="cuda")).shape == (0, 4, 4)


def muon_exact(c, m, v, g, matrices, step, lr, mu=0.95, nesterov=True, decay=0.0, b1=0.9, b2=0.999, eps=1e-8):
    c, m, v, g = (x.double() for x in (c, m, v, g))
    nm, nv = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    nc = (1 - lr * decay) * c + lr * (nm / (1 - b1 ** step)) / ((nv / (1 - b2 ** step)).sqrt() + eps)
    change = torch.zeros_like(c)                           # what the tolerance of the matrices' steps is relative to
    for at, r, k in matrices:
        s = slice(at, at + r * k)
        nm[s] = mu * m[s] + (1 - mu) * g[s]
        nv[s] = v[s]
        u = (mu * nm[s] + (1 - mu) * g[s]) if nesterov else nm[s]
        o = exact(u.view(r, k)).reshape(-1) * (lr * 0.2 * math.sqrt(max(r, k)))
        nc[s] = (1 - lr * decay) * c[s] + o
        change[s] = o
    return nc, nm, nv, change


LISTS = [
    (100, [], "no matrices"),
    (385, [(0, 16, 5), (96, 16, 16), (368, 1, 16)], "the smallest policy"),
    (21256, [(0, 128, 28), (3712, 128, 128), (20224, 8, 128)], "the large control policy"),
    (5994, [(0, 8, 25), (208, 16, 200), (3424, 10, 256)], "the convolutions"),
    (300 * 200 + 64 * 64 + 50, [(7, 300, 200), (300 * 200 + 20, 64, 64)], "large and small"),
    (40 * 12 * 9 + 3, [(i * 12 * 9 + 1, 12, 9) for i in range(40)], "more than a launch lists"),
    (33 * 140 * 150 + 90, [(i * 140 * 150 + 2 * i, 140, 150) for i in range(33)], "more large ones than a launch lists"),
]


@pytest.mark.parametrize("dim,matrices,what", LISTS, ids=[x[2] for x in LISTS])
@pytest.mark.parametrize("nesterov", [True, False])
def test_muon_step(dim, matrices, what, nesterov):
    gen = torch.Generator(device="cuda").manual_seed(dim)
    c, m, v, g = (torch.randn(dim, generator=gen, device="cuda") * s for s in (0.3, 1e-3, 1.0, 1e-2))
    v = v.square() * 1e-5
    kw = dict(lr=0.02, nesterov=nesterov, weight_decay=0.1)
    got = muon_step(c, m, v, g, matrices, 3, momentum=0.9, **kw)
    want = muon_exact(c, m, v, g, matrices, 3, 0.02, 0.9, nesterov, 0.1)
    # sums of two or three rounded products: 4 x 2^-24 of the largest term; the centre adds the step's own error
    for x, y, size in zip(got[1:], want[1:3], (m.abs() + g.abs(), v + g * g)):
        assert ((x.double() - y).abs() <= 2.0 ** -22 * size).all()
    err = (got[0].double() - want[0]).abs()
    inside = torch.zeros(dim, dtype=torch.bool, device="cuda")
    for at, r, k in matrices:
        s = slice(at, at + r * k)
        inside[s] = True
        o = want[3][s]
        scale = 0.02 * 0.2 * math.sqrt(max(r, k))
        rel = 2.0 ** -22 * (64 + 3.4445 ** 5 / max(float(o.norm()) / scale, 1e-30))
        assert float((err[s] - 2.0 ** -22 * (c[s].abs() + o.abs())).clamp_min(0).norm()) <= rel * float(o.norm()), (at, r, k)
    # Adam's ratio: m' and v' as above, one division and one root: 16 x 2^-24 of the quotient's terms
    rest = ~inside
    denom = (want[2] / (1 - 0.999 ** 3)).sqrt() + 1e-8
    size = c.abs() + 0.02 * (m.abs() + g.abs()) / (1 - 0.9 ** 3) / denom * (1 + (v + g * g) / denom.square())
    assert (err[rest] <= 2.0 ** -20 * size[rest]).all()
    # in place: the same bits, and the gradient is left alone
    c2, m2, v2, g2 = (x.clone() for x in (c, m, v, g))
    muon_step(c2, m2, v2, g2, matrices, 3, momentum=0.9, out=(c2, m2, v2), **kw)
    assert torch.equal(g2, g) and all(torch.equal(x, y) for x, y in zip((c2, m2, v2), got))


def test_muon_refusals_in_python():
    x = [torch.zeros(100, device="cuda") for _ in range(4)]
    for bad in ([(0, 10, 11)], [(0, 5, 5), (20, 5, 5)], [(-1, 2, 2)], [(0, 0, 3)]):
        with pytest.raises(EvoError):
            muon_step(*x, bad, 1, lr=0.1)
    with pytest.raises(EvoError):
        muon_step(*x, [], 0, lr=0.1)
    with pytest.raises(EvoError):
        muon_step(x[0], x[1], x[2], torch.zeros(99, device="cuda"), [], 1, lr=0.1)
    with pytest.raises(EvoError):
        muon_step(*x, [], 1, lr=0.1, out=(x[1], x[0], x[2]))
    with pytest.raises(EvoError):
        muon_step(*x, [], 1, lr=0.1, momentum=1.0)


def test_muon_steps_in_place_keep_their_order():
    """The launches of a step overlap; steps after one another, and what writes their inputs, do not."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    sizes, at = [(128, 28), (128, 128), (100, 700), (12, 300), (200, 160), (8, 128), (40, 40)], 5
    matrices = []
    for rows, cols in sizes:
        matrices.append((at, rows, cols))
        at += rows * cols + rows
    first = [torch.randn(at, generator=gen, device="cuda") for _ in range(3)]
    first[2].square_()
    gradients = torch.randn(24, at, generator=gen, device="cuda")
    results = []
    for wait in (False, True):
        state, g = [x.clone() for x in first], torch.empty(at, device="cuda")
        for step in range(1, 25):
            torch.mul(gradients[step - 1], state[0].abs() + 0.5, out=g)
            if wait:
                torch.cuda.synchronize()
            muon_step(*state, g, matrices, step, lr=0.05, weight_decay=0.01, out=tuple(state))
            if wait:
                torch.cuda.synchronize()
        results.append(state)
    for x, y in zip(*results):
        assert torch.isfinite(x).all() and torch.equal(x, y)
