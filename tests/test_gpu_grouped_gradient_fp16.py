"""Gradients of products of fp16 with tanh, for gradients as small as a mean over many rows gives them, against the formulas in 64 bits.

dz / scale is two numbers of fp16, the second 2^11 times as large as what the first leaves: off by 2^-22 of itself, or by 2^-36 where that is more.  The scale takes the results
to where fp16 has all of its bits, so that their own rounding hides nothing.  For the rest: dz comes of six roundings of fp32, a sum of k products is off by k + 32 units of 2^-24, and the
result is rounded to its type."""
import math

import pytest
import torch

from paper_2202_05008_b200 import grouped_linear_backward

pytestmark = pytest.mark.gpu
F16 = torch.float16


def make(lengths, n_in, n_out, size, scale, lead=0, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed + n_in * 31 + n_out)
    rows, groups = lead + sum(lengths), len(lengths)
    x = torch.randn(rows, n_in, generator=gen, device="cuda").half()
    w = (torch.randn(groups, n_out, n_in, generator=gen, device="cuda") / math.sqrt(n_in)).half()
    dy = (torch.randn(rows, n_out, generator=gen, device="cuda") * size).half()
    y = (torch.tanh(torch.randn(rows, n_out, generator=gen, device="cuda")) * scale).half()
    edges = [lead]
    for n in lengths:
        edges.append(edges[-1] + n)
    return dy, x, w, torch.tensor(edges, dtype=torch.int32, device="cuda"), y


def check(dy, x, w, offsets, y, scale, shared=False, **kw):
    got = grouped_linear_backward(dy, x, w, offsets, y, activation="tanh", scale=scale, **kw)
    d, xx, ww, yy = dy.double(), x.double(), w.double(), y.double()
    dz = d * (scale - yy * yy / scale)
    off_dz = dz.abs() * (6 * 2.0 ** -24 + 2.0 ** -22) + 2.0 ** -36 * scale
    edges = offsets.tolist()
    sets = [(edges[0], edges[-1])] if shared else list(zip(edges[:-1], edges[1:]))

    def close(g, want, off, s, k, what):
        off = off + (k + 32) * 2.0 ** -24 * s
        err, bound = (g.double() - want).abs(), off + 2.0 ** -11 * (want.abs() + off) + 2.0 ** -25
        assert (err <= bound).all(), (what, float((err / bound).max()))
    for n, (p, q) in enumerate(zip(edges[:-1], edges[1:])):
        if q > p and got[0] is not None:
            close(got[0][p:q], dz[p:q] @ ww[n], off_dz[p:q] @ ww[n].abs(), dz[p:q].abs() @ ww[n].abs(), w.shape[1], "dx")
    for n, (p, q) in enumerate(sets):
        d, o, z = dz[p:q], off_dz[p:q], xx[p:q]
        if got[1] is not None:
            close(got[1][n], d.t() @ z, o.t() @ z.abs(), d.abs().t() @ z.abs(), q - p, "dW")
        close(got[2][n], d.sum(0), o.sum(0), d.abs().sum(0), q - p, "db")


@pytest.mark.parametrize("size", [3e-6, 1e-4, 1.0])
@pytest.mark.parametrize("lengths,n_in,n_out", [
    ([3, 0, 1, 5], 40, 24), ([2, 9] * 40, 200, 136), ([7, 12, 0, 30] * 20, 159, 902), ([1, 2], 1001, 2000),       # dx of few rows: 8 and 16 at a time, weight rows split
    ([64, 300, 17, 0, 128], 264, 128), ([129, 65, 700], 130, 70), ([513, 40], 520, 1032),                         # both on the tensor cores, whole and laid out
    ([40, 70], 136, 4500), ([100], 264, 9000),                                                                    # weight rows of more than one sum
    ([9000, 300], 40, 24), ([5000, 8200, 31] + [64] * 40, 264, 520), ([4097] * 3, 300, 130),                      # rows of more than one sum, split and in one block
    ([300, 40] * 60, 20, 200), ([2000, 5], 300, 7),
])
def test_small_gradients_keep_their_bits(size, lengths, n_in, n_out):
    scale = 1024.0 if size < 1.0 else 2.0
    check(*make(lengths, n_in, n_out, size, scale, lead=2), scale)


@pytest.mark.parametrize("lengths,n_in,n_out", [([40, 3, 0, 5], 40, 24), ([300, 500], 264, 128), ([9000, 700, 2], 136, 72)])
def test_of_shared_weights_and_one_by_one(lengths, n_in, n_out):
    dy, x, w, offsets, y = make(lengths, n_in, n_out, 3e-6, 1024.0)
    check(dy, x, w[:1].expand_as(w), offsets, y, 1024.0, shared=True, shared_bias=True)
    check(dy, x, w, offsets, y, 1024.0, wanted=(False, True, True))
    check(dy, x, w, offsets, y, 1024.0, wanted=(True, False, True))
    check(dy, x, w, offsets, y, 1024.0, wanted=(False, False, True))
