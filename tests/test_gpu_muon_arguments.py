"""The Muon step's constants at the ends of their ranges: what the caller passes is what the step uses."""
import pytest
import torch

from paper_2202_05008_b200 import muon_step
from test_gpu_orthogonalize import muon_exact

pytestmark = pytest.mark.gpu


def _state(dim=500):
    gen = torch.Generator(device="cuda").manual_seed(dim)
    c, m, v, g = (torch.randn(dim, generator=gen, device="cuda") * s for s in (0.3, 1e-2, 1.0, 1e-2))
    return c, m, v.square() * 1e-4 + 1e-6, g


@pytest.mark.parametrize("kw", [dict(beta1=0.0), dict(beta2=0.0), dict(adam_eps=0.0), dict(beta1=0.0, beta2=0.0, adam_eps=0.0), dict(beta1=0.5, beta2=0.25, adam_eps=1e-3)])
@pytest.mark.parametrize("step", [1, 9])
def test_a_zero_is_a_zero(kw, step):
    c, m, v, g = _state()
    got = muon_step(c, m, v, g, [], step, lr=0.02, weight_decay=0.1, **kw)
    b1, b2, eps = kw.get("beta1", 0.9), kw.get("beta2", 0.999), kw.get("adam_eps", 1e-8)
    want = muon_exact(c, m, v, g, [], step, 0.02, decay=0.1, b1=b1, b2=b2, eps=eps)
    # sums of two rounded products: 4 x 2^-24 of the largest term
    assert ((got[1].double() - want[1]).abs() <= 2.0 ** -22 * (m.abs() + g.abs())).all()
    assert ((got[2].double() - want[2]).abs() <= 2.0 ** -22 * (v + g * g)).all()
    # the quotient: m' and v' as above, one root and one division, 16 x 2^-24 of its terms
    denom = (want[2] / (1 - b2 ** step)).sqrt() + eps
    size = c.abs() + 0.02 * (m.abs() + g.abs()) / (1 - b1 ** step) / denom * (1 + (v + g * g) / ((1 - b2 ** step) * denom.square()))
    assert ((got[0].double() - want[0]).abs() <= 2.0 ** -20 * size).all()
