"""The clipped policy loss where it is far from the policy that acted or from the reference, and exactly on the border of the clipping, against the definition in 64 bits.

Tolerances are those of the ordinary rows, which go by the logarithms' size, and one more: an exponential below fp32's smallest normal number, 2^-126, is 0 (the instruction's form flushes
it), so a probability is off by 2^-126 and a number of the gradient by 2^-126 G, where G is what its factor c is made of.  (e^-95 is 2^-137: the numbers that
this is about are 1e-38 of the row's largest.)"""
import math

import pytest
import torch

from paper_2202_05008_b200 import policy_loss
from test_gpu_policy_loss import definition

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def check(logits, actions, old, adv, ref=None, weights=None, clip=(0.2, 0.3), kl=0.0):
    got = policy_loss(logits, actions, old, adv, ref_logp=ref, weights=weights, clip=clip, kl=kl)
    loss, size, lp, gradient, g, far = definition(logits, actions, old, adv, ref, weights, clip, kl)
    n, x = logits.shape[1], logits.double()
    reach = x.amax(1) - torch.where(x.isfinite(), x, torch.full_like(x, math.inf)).amin(1)
    e = 2.0 ** -22 + reach * 2.25 * 2.0 ** -24
    d = e + reach * 2.0 ** -26 + (min(n, 512) + n / 512 + 16) * 2.0 ** -24
    c = d + 2.0 ** -21 + far * 2.0 ** -24
    assert ((got.logp.double() - lp).abs() <= d + 2.0 ** -24 * (lp.abs() + d)).all()
    assert abs(float(got.loss) - float(loss)) <= float((c * g).sum()) + 2.0 ** -24 * abs(float(loss)) + 1e-12 * float(size)
    p, half = torch.softmax(x, 1), torch.finfo(logits.dtype).eps / 2
    hot = torch.zeros_like(p).scatter_(1, actions[:, None], 1.0)
    off = g[:, None] * (c[:, None] * (hot - p).abs() + (e + d)[:, None] * p + 2.0 ** -126) + 2.0 ** -23 * gradient.abs()
    bound = off + half * (gradient.abs() + off) + 2.0 ** -126
    err = (got.gradient.double() - gradient).abs()
    assert (err <= bound).all(), float((err / bound).max())
    return got


@pytest.mark.parametrize("n", [3, 40, 100, 200, 300, 3000, 40000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_ratios_beyond_fp32_whose_products_are_not(n, dtype):
    """An action of probability e^-95 that the acting policy, or the reference, took for likely: e^95 is no fp32 number, e^95 times a weight of 1e-9 is."""
    rows = 6
    logits = torch.zeros(rows, n, device="cuda")
    logits[:, 0], logits[:, 2] = 95.0, -math.inf            # (a forbidden action: its gradient is 0, not 0 times infinity)
    logits = logits.to(dtype)
    actions = torch.ones(rows, dtype=torch.int64, device="cuda")
    weights = torch.full((rows,), 1e-9, device="cuda")
    actions[4:] = 0                                          # (log probability 0)
    logp = torch.tensor([-float(logits[0, 0])] * 4 + [0.0] * 2, device="cuda")
    old = logp - torch.tensor([0.1, 95.0, 90.0, -95.0, 95.0, -95.0], device="cuda")
    ref = logp + torch.tensor([95.0, 0.1, 91.0, -95.0, 93.0, 0.0], device="cuda")
    adv = torch.tensor([1.0, -1.0, -1e-3, -2.0, -0.5, 1.0], device="cuda")
    for kw in (dict(ref=ref, kl=0.05), dict()):
        got = check(logits, actions, old, adv, weights=weights, **kw)
        assert got.loss.isfinite() and got.gradient.isfinite().all() and (got.gradient[:, 2] == 0).all()
        if dtype == F32:
            assert got.gradient[1, 1] > 1e20


@pytest.mark.parametrize("n", [2, 40, 300, 5000])
def test_a_ratio_exactly_on_the_border_is_not_clipped(n):
    """One action has all of the probability, to the last bit of fp32: its log probability is 0, and the ratio to an old one of 0 is 1, the border of clip 0."""
    logits = torch.full((6, n), -40.0, device="cuda")
    logits[:, 0] = 0.0
    actions = torch.zeros(6, dtype=torch.int64, device="cuda")
    adv = torch.tensor([1.0, -1.0, 1.0, -1.0, 1.0, -1.0], device="cuda")
    old = torch.tensor([0.0, 0.0, -1e-6, 1e-6, 1e-6, -1e-6], device="cuda")     # on it; beyond it, clipped; inside, not
    got = policy_loss(logits, actions, old, adv, clip=(0.0, 0.0))
    assert (got.logp == 0).all()
    assert (got.gradient[[0, 1, 4, 5], 1] != 0).all() and (got.gradient[[2, 3]] == 0).all()
    assert got.gradient[0, 1] > 0 > got.gradient[1, 1]       # descending it takes from the other actions where the first did well


@pytest.mark.parametrize("n", [7, 40, 100, 200, 300, 1029, 5000, 40000])
@pytest.mark.parametrize("shift", [0, 1])
def test_small_probabilities_of_fp32_logits_have_their_bits(n, shift):
    """One logit far above the others, all of them multiples of 2^-10 below 2^7: differences are exact, the sum is 1 to the last bit (n e^-50 is below 2^-25), the action's log probability is
    exact, and with the old one equal to it the ratio is 1.  A number of the gradient is then an exponential, off by 2^-22 (the instruction) and four roundings of its correction (2^-24 each),
    times a weight, with two roundings more."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    logits = -torch.randint(50 << 10, 85 << 10, (4, n), generator=gen, device="cuda").float() / 1024
    at = torch.randint(1, n, (4,), generator=gen, device="cuda")
    logits[torch.arange(4, device="cuda"), at] = 0.0
    actions = torch.zeros(4, dtype=torch.int64, device="cuda")
    old = logits[:, 0].clone()
    adv, weights = torch.tensor([1.0, -2.0, 4.0, -0.5], device="cuda"), torch.tensor([1.0, 0.5, 2.0, 0.25], device="cuda")
    out = torch.empty(4, n + shift, device="cuda")[:, shift:]          # (1: rows of the gradient that do not lie like the logits')
    got = policy_loss(logits, actions, old, adv, weights=weights, clip=(0.2, 0.2), out=out)
    assert torch.equal(got.logp, old)
    want = (weights * adv).double()[:, None] * torch.exp(logits.double())
    want[:, 0] = -(weights * adv).double() * -torch.expm1(old.double())
    assert ((got.gradient.double() - want).abs() <= (2.0 ** -22 + 6 * 2.0 ** -24) * want.abs()).all()
