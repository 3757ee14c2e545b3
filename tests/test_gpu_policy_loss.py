"""The clipped policy loss and its gradient, against the definition in 64 bits.

Tolerances.  With R the largest distance of a finite logit from the row's maximum, an exponential is off by E = 2^-22 + R (2 2^-24 + 2^-26) of itself (the
instruction; its argument (x - max) log2 e: the difference's rounding, the product's, log2 e's own), the sum by another (terms of a thread's chain and of the tree) 2^-24; logp by both, D, plus
R 2^-26.  With G = |A| ratio + kl e^(ref - logp) the factor c is off by D G, and by 2^-21 G for the functions in fp32 that it is made of (each two units of 2^-23 at most, of
arguments rounded to fp32, 2^-24 of the largest logarithm l), a probability by E + D; a number of the gradient is rounded once to fp32 and once to its type."""
import math

import pytest
import torch

from paper_2202_05008_b200 import EvoError, policy_loss

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def definition(logits, actions, old, adv, ref, weights, clip, kl):
    """(loss, sum |w L|, logp, gradient, G w) in 64 bits."""
    rows, n = logits.shape
    w = torch.full((rows,), 1.0 / max(rows, 1), dtype=torch.float64, device=logits.device) if weights is None else weights.double()
    live = (actions >= 0) & (actions < n) & (w != 0)
    a = actions.clamp(0, n - 1).long()[:, None]
    lp_all = logits.double() - torch.logsumexp(logits.double(), 1, keepdim=True)
    lp = lp_all.gather(1, a)[:, 0]
    adv, ratio = adv.double(), torch.exp(lp - old.double())
    clipped = torch.where(adv >= 0, ratio > 1 + clip[1], ratio < 1 - clip[0])
    bound = torch.where(adv >= 0, torch.full_like(ratio, 1 + clip[1]), torch.full_like(ratio, 1 - clip[0]))
    loss, c, size = -torch.where(clipped, bound, ratio) * adv, torch.where(clipped, torch.zeros_like(ratio), -ratio * adv), (ratio * adv).abs()
    if kl:
        d = ref.double() - lp
        loss, c, size = loss + kl * (torch.expm1(d) - d), c - kl * torch.expm1(d), size + kl * (torch.exp(d) + 1 + d.abs())
    p = torch.exp(lp_all)
    gradient = -(w * c)[:, None] * p
    gradient.scatter_(1, a, (-(w * c) * torch.expm1(lp))[:, None])
    zero = torch.zeros((), dtype=torch.float64, device=logits.device)
    pick = lambda x: torch.where(live, x, zero)
    reach = torch.maximum((lp - old.double()).abs(), (ref.double() - lp).abs()) if kl else (lp - old.double()).abs()
    return pick(w * loss).sum(), pick((w * loss).abs() + w.abs() * size).sum(), pick(lp), torch.where(live[:, None], gradient, zero), pick(w.abs() * size), pick(reach)


def make(rows, n, dtype, seed=0, masked=0.0, spread=2.0, padded=0.2, wide=True):
    gen = torch.Generator(device="cuda").manual_seed(seed + rows * 13 + n)
    logits = (torch.randn(rows, n, generator=gen, device="cuda") * spread).to(dtype)
    actions = torch.randint(0, n, (rows,), generator=gen, device="cuda")
    if masked:
        mask = (torch.rand(rows, n, generator=gen, device="cuda") < masked).scatter_(1, actions[:, None], False)
        logits[mask] = -math.inf
    lp = (logits.double() - torch.logsumexp(logits.double(), 1, keepdim=True)).gather(1, actions[:, None])[:, 0]
    jump = torch.randn(rows, generator=gen, device="cuda", dtype=torch.float64) * 0.3
    for border in (math.log(0.8), math.log(1.3)):          # (the borders used below; off them by more than rounding)
        jump = torch.where((jump - border).abs() < 1e-4, jump + 4e-4, jump)
    old, ref = (lp - jump).float(), (lp + torch.randn(rows, generator=gen, device="cuda") * 0.5).float()
    adv = torch.randn(rows, generator=gen, device="cuda")
    weights = torch.rand(rows, generator=gen, device="cuda")
    pad = torch.rand(rows, generator=gen, device="cuda")
    actions[pad < padded / 2] = -1
    actions[(pad >= padded / 2) & (pad < padded * 0.75)] = n
    weights[(pad >= padded * 0.75) & (pad < padded)] = 0.0
    return logits, actions if wide else actions.int(), old, adv, ref, weights


def check(logits, actions, old, adv, ref=None, weights=None, clip=(0.2, 0.3), kl=0.0, **kw):
    given = logits.clone()
    got = policy_loss(logits, actions, old, adv, ref_logp=ref, weights=weights, clip=clip, kl=kl, **kw)
    loss, size, lp, gradient, g, far = definition(given, actions, old, adv, ref, weights, clip, kl)
    n = given.shape[1]
    x = given.double()
    reach = x.amax(1) - torch.where(x.isfinite(), x, torch.full_like(x, math.inf)).amin(1)
    e = 2.0 ** -22 + reach * 2.25 * 2.0 ** -24
    d = e + reach * 2.0 ** -26 + (min(n, 512) + n / 512 + 16) * 2.0 ** -24
    half = torch.finfo(logits.dtype).eps / 2
    c = d + 2.0 ** -21 + far * 2.0 ** -24
    assert ((got.logp.double() - lp).abs() <= d + 2.0 ** -24 * (lp.abs() + d)).all()
    assert abs(float(got.loss) - float(loss)) <= float((c * g).sum()) + 2.0 ** -24 * abs(float(loss)) + 1e-12 * float(size)
    if got.gradient is not None:
        p = torch.softmax(x, 1)
        hot = torch.zeros_like(p)
        inside = (actions >= 0) & (actions < n)
        hot[inside, actions[inside].long()] = 1.0
        off = g[:, None] * (c[:, None] * (hot - p).abs() + (e + d)[:, None] * p) + 2.0 ** -23 * gradient.abs()
        tiny = torch.finfo(logits.dtype).smallest_normal * torch.finfo(logits.dtype).eps + 2.0 ** -126
        bound = off + half * (gradient.abs() + off) + tiny
        err = (got.gradient.double() - gradient).abs()
        assert (err <= bound).all(), float((err / bound).max())
        dead = ~inside if weights is None else ~inside | (weights == 0)
        assert (got.gradient[dead] == 0).all() and (got.logp[dead] == 0).all()
    return got


LENGTHS = [1, 2, 12, 31, 32, 33, 200, 256, 257, 512, 1000, 1024, 1025, 2049, 4097, 5003, 8192, 10001, 16385, 32000, 40001, 70000, 131073, 300000]


@pytest.mark.parametrize("n", LENGTHS)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_lengths_and_types(n, dtype):
    rows = 37 if n < 3000 else 9
    logits, actions, old, adv, ref, weights = make(rows, n, dtype, wide=n % 2 == 0)
    check(logits, actions, old, adv, ref, weights, kl=0.05)
    logits, actions, old, adv, ref, weights = make(rows, n, dtype, seed=1, masked=0.6, padded=0.0)
    check(logits, actions, old, adv, clip=(0.2, 0.3))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [5, 100, 300, 1029, 3001, 9000, 50000])
@pytest.mark.parametrize("shift,pitch,same", [(0, 3, True), (1, 0, True), (5, 8, True), (0, 8, False), (3, 1, False)])
def test_strides_and_alignment(dtype, n, shift, pitch, same):
    logits, actions, old, adv, ref, weights = make(11, n, dtype)
    room = torch.full((11, shift + n + pitch), float("nan"), dtype=dtype, device="cuda")
    x = room[:, shift:shift + n]
    x.copy_(logits)
    target = torch.full((11, shift + n + pitch if same else n + 2), 7.0, dtype=dtype, device="cuda")
    out = target[:, shift:shift + n] if same else target[:, 1:1 + n]
    check(x, actions, old, adv, ref, weights, kl=0.1, out=out)
    assert int((target == 7).sum()) >= target.numel() - out.numel()
    got = policy_loss(logits, actions, old, adv, ref_logp=ref, weights=weights, clip=(0.2, 0.3), kl=0.1)
    inside = policy_loss(x, actions, old, adv, ref_logp=ref, weights=weights, clip=(0.2, 0.3), kl=0.1, out=x)          # over the logits
    assert inside.gradient is x and (room[:, :shift].isnan()).all() and room[:, shift + n:].isnan().all()
    half = torch.finfo(dtype).eps
    assert ((x.double() - got.gradient.double()).abs() <= (2 * half + 1e-5) * got.gradient.double().abs() + 1e-7).all()


@pytest.mark.parametrize("n", [7, 300, 9000, 300000])
def test_rows_that_have_no_probabilities(n):
    logits, actions, old, adv, ref, weights = make(8, n, F32, padded=0.0)
    logits[0, n // 2], logits[1, 3], logits[2], logits[3] = float("nan"), float("inf"), -math.inf, -math.inf
    actions[3], weights[0] = -1, 0.0                       # padding, whatever it holds
    got = policy_loss(logits, actions, old, adv, ref_logp=ref, weights=weights, kl=0.1)
    assert got.loss.isnan() and (got.gradient[0] == 0).all() and (got.gradient[3] == 0).all()
    assert got.gradient[1:3].isnan().all() and got.logp[1:3].isnan().all() and got.logp[[0, 3]].eq(0).all()
    assert got.gradient[4:].isfinite().all() and got.logp[4:].isfinite().all()
    actions[:] = n
    got = policy_loss(logits, actions, old, adv, weights=weights)
    assert float(got.loss) == 0 and (got.gradient == 0).all() and (got.logp == 0).all()


@pytest.mark.parametrize("n", [3, 270, 40000])
def test_one_action_that_is_allowed_and_extremes(n):
    logits, actions, old, adv, ref, weights = make(6, n, F32, padded=0.0)
    keep = torch.zeros_like(logits, dtype=torch.bool).scatter_(1, actions[:, None], True)
    logits[~keep] = -math.inf
    got = policy_loss(logits, actions, torch.zeros_like(old), adv)
    assert (got.logp == 0).all() and (got.gradient == 0).all()
    logits[~keep] = torch.finfo(F32).min
    logits[keep] = 3e38
    got = policy_loss(logits, actions, torch.zeros_like(old), adv)
    assert (got.logp == 0).all() and got.gradient.isfinite().all()
    logits[:] = torch.finfo(F32).min                       # all alike: even probabilities
    got = policy_loss(logits, actions, torch.full_like(old, -math.log(n)), adv, clip=(0.5, 0.5))
    assert (got.logp + math.log(n)).abs().max() < 1e-5 and got.gradient.isfinite().all()


@pytest.mark.parametrize("n,each", [(12, 128), (50, 64), (100, 32), (200, 16)])
def test_rows_of_one_block_of_a_cluster_of_them_and_more(n, each):
    for rows in (1, each - 1, each, each + 1, 2 * each + 1, 4 * each, 5 * each + 3, 8 * each - 1, 8 * each, 8 * each + 1, 9 * each):
        logits, actions, old, adv, ref, weights = make(rows, n, F32, wide=rows % 2 == 0)
        got = check(logits, actions, old, adv, ref, weights, kl=0.05)
        again = policy_loss(logits, actions, old, adv, ref_logp=ref, weights=weights, clip=(0.2, 0.3), kl=0.05, gradient=False)
        assert torch.equal(got.loss, again.loss) and torch.equal(got.logp, again.logp)
        check(logits, actions, old, adv)


def test_no_rows_and_one():
    empty = torch.zeros(0, 9, device="cuda")
    none = torch.zeros(0, device="cuda")
    got = policy_loss(empty, none.int(), none, none)
    assert float(got.loss) == 0 and got.logp.shape == (0,) and got.gradient.shape == (0, 9)
    check(*make(1, 9, F32, padded=0.0)[:4])
    x = make(50, 1000, BF16, padded=0.0)
    a, b = check(*x[:4]), policy_loss(*x[:4], clip=(0.2, 0.3), gradient=False)
    assert b.gradient is None and torch.equal(a.loss, b.loss) and torch.equal(a.logp, b.logp)


def test_the_borders_belong_to_what_is_not_clipped():
    # a row of two equal logits: logp = log 1/2 exactly as the kernel has it; a ratio of 1 is on the border of clip 0
    logits = torch.zeros(4, 2, device="cuda")
    old = torch.full((4,), math.log(0.5), device="cuda")
    adv = torch.tensor([1.0, -1.0, 2.0, -2.0], device="cuda")
    old[2:] += torch.tensor([-0.1, 0.1], device="cuda")    # above for A > 0, below for A < 0: clipped
    got = policy_loss(logits, torch.zeros(4, dtype=torch.int64, device="cuda"), old, adv, clip=(0.01, 0.01))
    assert (got.gradient[2:] == 0).all() and (got.gradient[:2] != 0).all()
    assert got.gradient[0, 0] < 0 < got.gradient[1, 0]     # descending it raises the first action's probability where it did well


def test_the_gradient_is_the_difference_of_the_loss():
    logits, actions, old, adv, ref, weights = make(5, 40, F32, padded=0.0)
    got = policy_loss(logits, actions, old, adv, ref_logp=ref, weights=weights, clip=(0.2, 0.3), kl=0.2)
    step = 2.0 ** -9                                         # (a row close to a border may cross it: the nearest is 1e-4 off and steps move a ratio by at most 2e-3; rows are picked)
    picked = 0
    for r in range(5):
        lp = float(definition(logits, actions, old, adv, ref, weights, (0.2, 0.3), 0.2)[2][r])
        if min(abs(math.exp(lp - float(old[r])) - b) for b in (0.8, 1.3)) < 0.02:
            continue
        picked += 1
        for v in (0, 17, int(actions[r])):
            ends = []
            for sign in (1.0, -1.0):
                moved = logits.double()
                moved[r, v] += sign * step
                ends.append(float(definition(moved, actions, old, adv, ref, weights, (0.2, 0.3), 0.2)[0]))
            assert abs((ends[0] - ends[1]) / (2 * step) - float(got.gradient[r, v])) < 1e-4
    assert picked


def test_refusals():
    logits, actions, old, adv, ref, weights = make(6, 10, F32)
    for call in (lambda: policy_loss(logits.double(), actions, old, adv), lambda: policy_loss(logits, actions.float(), old, adv), lambda: policy_loss(logits, actions[:5], old, adv),
                 lambda: policy_loss(logits, actions, old.half(), adv), lambda: policy_loss(logits, actions, old, adv[:5]), lambda: policy_loss(logits, actions, old, adv, kl=0.1),
                 lambda: policy_loss(logits, actions, old, adv, clip=(1.5, 0.2)), lambda: policy_loss(logits, actions, old, adv, clip=(0.2, -0.1)),
                 lambda: policy_loss(logits, actions, old, adv, clip=(0.2, float("nan"))), lambda: policy_loss(logits, actions, old, adv, ref_logp=ref, kl=-1.0),
                 lambda: policy_loss(logits.t(), actions, old, adv), lambda: policy_loss(logits.cpu(), actions, old, adv), lambda: policy_loss(logits, actions, old, adv, out=logits[:5]),
                 lambda: policy_loss(logits[:, :0], actions, old, adv), lambda: policy_loss(logits, actions, old, adv, weights=weights[:2])):
        with pytest.raises(EvoError):
            call()
