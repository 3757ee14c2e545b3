"""Rows that lie beyond 2^31 numbers of an array: taken, brought back, with their gradient, and as logits, against the same rows by themselves."""
import pytest
import torch

from paper_2202_05008_b200 import combine_rows, combine_rows_backward, policy_loss, take_rows

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("cols,pitch", [(2048, 2048), (1001, 2050)])
def test_sorted_rows_beyond_32_bits(cols, pitch):
    total, rows = 1_100_000, 300
    gen = torch.Generator(device="cuda").manual_seed(cols)
    y = torch.empty(total, pitch, dtype=BF16, device="cuda")[:, :cols]
    place = torch.stack([torch.arange(rows, device="cuda"), total - 1 - torch.arange(rows, device="cuda")], 1).int()
    x, w = torch.randn(rows, cols, generator=gen, device="cuda").to(BF16), torch.randn(rows, 2, generator=gen, device="cuda")
    take_rows(x, place, w, out=y)
    want = (w[:, :, None] * x[:, None].float()).to(BF16)
    assert torch.equal(y[:rows], want[:, 0]) and torch.equal(y[total - rows:].flip(0), want[:, 1])
    near, at = torch.cat([y[:rows], y[total - rows:]]), torch.stack([torch.arange(rows, device="cuda"), 2 * rows - 1 - torch.arange(rows, device="cuda")], 1).int()
    assert torch.equal(combine_rows(y, place, w), combine_rows(near.contiguous(), at, w))
    dy, dw = combine_rows_backward(x, y, place, w, out=torch.empty(total, pitch, dtype=BF16, device="cuda")[:, :cols])
    assert torch.equal(dy[:rows], want[:, 0]) and torch.equal(dy[total - rows:].flip(0), want[:, 1])
    sums = torch.stack([(x.double() * y[place[:, j].long()].double()).sum(1) for j in (0, 1)], 1)
    sizes = torch.stack([(x.double() * y[place[:, j].long()].double()).abs().sum(1) for j in (0, 1)], 1)
    assert ((dw.double() - sums).abs() <= (cols + 1) * 2.0 ** -24 * sizes).all()


@pytest.mark.parametrize("rows,n,pitch", [(70_000, 33_000, 33_000), (1_100_000, 700, 2056), (17_000_000, 130, 130)])
def test_logits_beyond_32_bits(rows, n, pitch):
    gen = torch.Generator(device="cuda").manual_seed(n)
    last = 500
    room = torch.zeros(rows, pitch, dtype=BF16, device="cuda")[:, :n]
    room[-last:] = torch.randn(last, n, generator=gen, device="cuda").to(BF16)
    actions = torch.full((rows,), -1, device="cuda")
    actions[-last:] = torch.randint(0, n, (last,), generator=gen, device="cuda")
    old, adv = torch.full((rows,), -5.0, device="cuda"), torch.ones(rows, device="cuda")
    weights = torch.full((rows,), 1.0 / last, device="cuda")
    out = torch.full((rows, pitch), 7.0, dtype=BF16, device="cuda")[:, :n]
    got = policy_loss(room, actions, old, adv, weights=weights, clip=(0.9, 30.0), out=out)
    alone = policy_loss(room[-last:], actions[-last:], old[-last:], adv[-last:], weights=weights[-last:], clip=(0.9, 30.0), out=torch.empty(last, pitch, dtype=BF16, device="cuda")[:, :n])
    assert torch.equal(got.logp[-last:], alone.logp) and (got.logp[:-last] == 0).all()
    # (few rows may be a block of other threads', whose sums have another order: a unit of the type)
    assert ((got.gradient[-last:].float() - alone.gradient.float()).abs() <= 2.0 ** -7 * alone.gradient.float().abs()).all() and alone.gradient.abs().sum() > 0
    assert not got.gradient[:-last].any() and abs(float(got.loss) - float(alone.loss)) <= 1e-5 * abs(float(alone.loss))
