"""Gradients of products whose scale has no square in fp32, against the formulas in 64 bits.

Tolerances as for other scales: dz comes of six roundings of fp32, operands count with 21 bits or more, a sum of k products is off by k + 32 units of 2^-24, the result by its rounding."""
import math

import pytest
import torch

from paper_2202_05008_b200 import grouped_linear_backward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [1e-30, -3e-25, 1e25, -1e30])
@pytest.mark.parametrize("act", ["tanh", "relu"])
@pytest.mark.parametrize("lengths,n_in,n_out", [([3, 0, 5], 40, 24), ([2] * 50, 300, 7), ([70, 200, 9], 136, 200), ([3000], 20, 16)])
def test_scales_that_have_no_square(scale, act, lengths, n_in, n_out):
    gen = torch.Generator(device="cuda").manual_seed(n_in)
    rows, groups = sum(lengths), len(lengths)
    x, dy = torch.randn(rows, n_in, generator=gen, device="cuda"), torch.randn(rows, n_out, generator=gen, device="cuda")
    w = torch.randn(groups, n_out, n_in, generator=gen, device="cuda") / math.sqrt(n_in)
    z = torch.randn(rows, n_out, generator=gen, device="cuda")
    y = scale * (torch.tanh(z) if act == "tanh" else z.relu())
    edges = [0]
    for n in lengths:
        edges.append(edges[-1] + n)
    offsets = torch.tensor(edges, device="cuda")
    s, yy, d = torch.tensor(scale, dtype=torch.float32).double().item(), y.double(), dy.double()
    dz = d * (s - yy * yy / s) if act == "tanh" else d * s * (yy / s > 0)
    for wanted in ((True, True, True), (False, False, True)):
        dx, dw, db = grouped_linear_backward(dy, x, w, offsets, y, activation=act, scale=scale, wanted=wanted)
        for g, (p, q) in enumerate(zip(edges[:-1], edges[1:])):
            a, b, ww = dz[p:q], x[p:q].double(), w[g].double()
            for got, want, size, k in ((None if dx is None else dx[p:q], a @ ww, a.abs() @ ww.abs(), n_out), (None if dw is None else dw[g], a.t() @ b, a.abs().t() @ b.abs(), q - p),
                                       (db[g], a.sum(0), a.abs().sum(0), q - p)):
                if got is not None:
                    bound = (6 * 2.0 ** -24 + 2.0 ** -20 + (k + 32) * 2.0 ** -24) * size + 2.0 ** -24 * want.abs() + 1e-44
                    assert ((got.double() - want).abs() <= bound).all()
