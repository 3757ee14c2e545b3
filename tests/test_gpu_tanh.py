"""The tanh of the grouped products and of the policy's actions, by itself."""
import pytest
import torch

from paper_2202_05008_b200 import mlp_actions

pytestmark = pytest.mark.gpu


def test_tanh_by_itself():
    """A policy of one weight, 1: numbers of up to 22 bits pass through the product as they are.  Beyond 1/2 the result is
    1 - 2 r, r = 1 / (e + 1), e = 2^(2 log2(e) x).  Relative to e: 2 x (2^-24 + 2^-25) from the argument (its product and its constant) and 2^-22 from the
    exponential; relative to r: e / (e + 1) of that, 2^-24 from the sum and 2^-23 from the reciprocal; 2 r / tanh = 2 / (e - 1) of that reaches the
    result, which is rounded once.  Below 1/2: 1e-7 left out of the series, and 1.25 x 2^-24 of rounding twice."""
    k = torch.cat([torch.arange(1, 1 << 22, device="cuda"), torch.arange(1, 1 << 12, device="cuda") * 2.0 ** -10])
    x = (k.double() * 2.0 ** -18).float()
    x = torch.cat([x, -x])[:, None]
    theta = torch.tensor([[1.0, 0.0, 0.0, 0.0]], device="cuda")
    got = mlp_actions(theta, (1, 1), x, torch.tensor([0, x.shape[0]], device="cuda"))[:, 0].double()
    a = x[:, 0].double().abs()
    want = torch.tanh(a)
    e = torch.exp(2 * a)
    far = (e / (e + 1) * (2 * a * 1.5 * 2.0 ** -24 + 2.0 ** -22) + 1.5 * 2.0 ** -23) * 2 / (e - 1) + 2.0 ** -24
    bound = torch.where(a < 0.5, torch.full_like(a, 1e-7 + 2.5 * 2.0 ** -24), far)
    err = (got.abs() - want).abs() / want
    print("largest error of tanh, relative:", float(err.max()), "at", float(a[err.argmax()]), "bound there", float(bound[err.argmax()]))
    assert torch.equal(got.sign(), x[:, 0].double().sign()) and (err <= bound).all()
    assert float(far[a >= 0.5].max()) < 5.5e-7
