"""Products grouped by member where a group has many rows (fp32 and unaligned 16-bit operands are laid out for the tensor cores there), and
offsets that are out of order; formulas and tolerances of test_gpu_grouped."""
import pytest
import torch

from paper_2202_05008_b200 import Solver, grouped_linear, mlp_actions, workloads as W
from test_gpu_grouped import BF16, F16, F32, actions_exact, check, exact, make, theta_for

pytestmark = pytest.mark.gpu
LONG = [3, 0, 320, 191, 140]                # 131 rows a group: beyond every threshold


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n_in,n_out,shift", [(64, 48, 0), (64, 48, 1), (61, 49, 0), (256, 136, 3), (130, 200, 2)])
def test_long_groups_with_strides_alignment_and_shared_weights(dtype, n_in, n_out, shift):
    x, w, b, off = make(5, LONG, n_in, n_out, dtype, lead=2, tail=4)
    theta = torch.full((5, shift + n_out * n_in + n_out + 24), float("nan"), dtype=dtype, device="cuda")
    theta[:, shift:shift + n_out * n_in] = w.flatten(1)
    theta[:, shift + n_out * n_in:shift + n_out * n_in + n_out] = b
    wv = theta[:, shift:shift + n_out * n_in].unflatten(1, (n_out, n_in))
    bv = theta[:, shift + n_out * n_in:shift + n_out * n_in + n_out]
    xs = torch.full((x.shape[0], n_in + 11), float("nan"), dtype=dtype, device="cuda")
    xs[2:-4, 3:3 + n_in] = x[2:-4]                             # (rows that no group has stay NaN)
    ys = torch.full((x.shape[0], n_out + 9), 7.0, dtype=dtype, device="cuda")
    yv = ys[:, 5:5 + n_out]
    assert grouped_linear(xs[:, 3:3 + n_in], wv, off, bv, activation="tanh", scale=1.5, out=yv) is yv
    check(yv, x, w, off, b, "tanh", 1.5)
    assert (ys[:, :5] == 7).all() and (ys[:, 5 + n_out:] == 7).all() and (ys[:2] == 7).all() and (ys[-4:] == 7).all()
    shared, one_bias = w[:1].expand(5, n_out, n_in), b[:1].expand(5, n_out)
    check(grouped_linear(x, shared, off, one_bias), x, shared, off, one_bias)
    pitch = torch.full((5, n_out, n_in + 7), float("nan"), dtype=dtype, device="cuda")
    pitch[:, :, 2:2 + n_in] = w
    check(grouped_linear(x, pitch[:, :, 2:2 + n_in], off), x, w, off)


@pytest.mark.parametrize("n_in", [64, 1100])                   # one part of a sum, and three
@pytest.mark.parametrize("dtype", [F32, F16])
def test_infinities_and_nan_of_long_groups_stay_with_their_rows_and_groups(n_in, dtype):
    x, w, b, off = make(5, LONG, n_in, 80, dtype, tail=2)
    clean = grouped_linear(x, w, off, b)
    x2, w2 = x.clone(), w.clone()
    x2[5, 7] = float("nan")
    x2[60, n_in - 1] = float("inf")
    x2[-1] = float("nan")                                       # a row of no group
    w2[4, 11, 5] = float("-inf")
    w2[1] = float("nan")                                        # a group without rows
    got = grouped_linear(x2, w2, off, b)
    want = exact(x2, w2, off, b)[0]
    inside = slice(0, sum(LONG))
    bad = ~want[inside].isfinite()
    # (of fp32 operands an infinity may come out as NaN)
    assert not got[inside][bad].isfinite().any() and torch.equal(got[inside][~bad], clean[inside][~bad])
    assert int(bad.sum()) == 80 + 80 + LONG[4] and got[5].isnan().all()


def test_the_largest_finite_numbers_are_numbers_in_long_groups():
    x, w, b, off = make(2, [90, 80], 40, 24, F32)
    top = torch.finfo(F32).max
    x, w = x.clamp(-1, 1) * 2.0 ** -12, w.clamp(-1, 1)
    x[3, 7], x[100, 39], w[1, 5, 6] = top, -3.3975e38, -top
    w[:, :, 7], w[:, :, 39] = 2.0 ** -40, -2.0 ** -30
    x[90:, 6] = 2.0 ** -70
    got = grouped_linear(x, w, off, b)
    assert got.isfinite().all()
    check(got, x, w, off, b)


OFFSETS = [lambda n: [-7, 4, 5 * n, 1 << 30, 3, 9], lambda n: [0, n, 5, n, 0, n], lambda n: [n, n // 2, n // 3, 2, 1, 0], lambda n: [n + 50] * 6]


@pytest.mark.parametrize("dtype,n_in,rows", [(F32, 64, 12), (F32, 200, 300), (F32, 61, 400), (BF16, 64, 300), (BF16, 61, 300), (F16, 520, 40)])
@pytest.mark.parametrize("which", range(len(OFFSETS)))
def test_offsets_out_of_order_touch_nothing_outside(dtype, n_in, rows, which):
    gen = torch.Generator(device="cuda").manual_seed(which)
    w = torch.randn(5, 48, n_in, generator=gen, device="cuda").to(dtype)
    xs = torch.randn(rows + 8, n_in, generator=gen, device="cuda").to(dtype)
    for wide in (torch.int32, torch.int64):
        ys = torch.full((rows + 8, 60), 3.0, dtype=dtype, device="cuda")
        off = torch.tensor(OFFSETS[which](rows), dtype=wide, device="cuda")
        grouped_linear(xs[4:-4], w, off, out=ys[4:-4, 6:54])
        assert (ys[:4] == 3).all() and (ys[-4:] == 3).all() and (ys[:, :6] == 3).all() and (ys[:, 54:] == 3).all()


@pytest.mark.parametrize("sizes,rows", [((5, 16, 3), 60), ((28, 128, 128, 8), 200), ((20, 600, 3), 200), ((28, 128, 8), 9)])
@pytest.mark.parametrize("which", range(len(OFFSETS)))
def test_offsets_out_of_order_of_policies_touch_nothing_outside(sizes, rows, which):
    theta = theta_for(5, sizes)
    obs = torch.randn(rows + 8, sizes[0], device="cuda")
    ys = torch.full((rows + 8, sizes[-1] + 4), 3.0, device="cuda")
    mlp_actions(theta, sizes, obs[4:-4], torch.tensor(OFFSETS[which](rows), device="cuda"), out=ys[4:-4, 2:-2])
    assert (ys[:4] == 3).all() and (ys[-4:] == 3).all() and (ys[:, :2] == 3).all() and (ys[:, -2:] == 3).all()


def test_solver_actions_with_a_matrix_of_the_caller():
    w = W.CFG2
    s = Solver(w)
    theta = s.ask()
    off = torch.arange(0, 3 * w.pop_size + 1, 3, device="cuda")
    obs = torch.randn(3 * w.pop_size, 5, device="cuda")
    got = s.actions(obs, off)
    mine = torch.full((w.pop_size, theta.stride(0)), float("nan"), device="cuda")
    mine[:, :w.param_dim] = theta
    assert torch.equal(s.actions(obs, off, theta=mine), got)
    other = theta_for(w.pop_size, w.layer_sizes)
    want, bound = actions_exact(other, w.layer_sizes, obs, off, w.action_scale)
    assert ((s.actions(obs, off, theta=other).double() - want).abs() <= bound).all()
    assert s.sync_status() == 0
    s.close()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n_in", [8192, 8200, 20001, 65536, 262144])
@pytest.mark.parametrize("rows", [(1, 2), (33, 20), (150, 70)])
def test_sums_of_many_numbers_of_one_sign(n_in, rows, dtype):
    """The tensor core cuts up to 2^-23 of a running sum off with every 16 numbers of 16 bits (8 of tf32) that it adds.  Sums stay in it for at most 8,192 numbers,
    2^-14 of the result; longer ones are added up in fp32, a rounding of 2^-24 for every 64 or more numbers.  The result is rounded once.  (fp32: in it for
    512 numbers at most, 2^-17, and 2^-20 for the operands.)"""
    gen = torch.Generator(device="cuda").manual_seed(n_in)
    x = (torch.rand(sum(rows), n_in, generator=gen, device="cuda") * 0.5 + 0.5).to(dtype)
    w = ((torch.rand(2, 24, n_in, generator=gen, device="cuda") * 0.5 + 0.5) / n_in).to(dtype)
    off = torch.tensor([0, rows[0], sum(rows)], device="cuda")
    got = grouped_linear(x, w, off).double()
    want = exact(x, w, off, None)[0]
    lost = 2.0 ** -17 + 2.0 ** -20 if dtype == F32 else 2.0 ** -14
    bound = torch.finfo(dtype).eps / 2 * 1.001 + lost + n_in / 64 * 2.0 ** -24 + (2.0 ** -25 / want if dtype == F16 else 0)
    err = (got - want).abs() / want
    assert (err <= bound).all(), float((err / bound).max())


@pytest.mark.parametrize("groups,per,n_in,n_out", [(300, 2, 40, 64), (300, 5, 40, 64), (64, 1, 2048, 136), (200, 4, 512, 72), (1, 5, 1024, 264), (1, 40, 1024, 264), (900, 17, 104, 8)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_aligned_rows_of_few_and_many_a_group(groups, per, n_in, n_out, dtype):
    """16-bit operands that both kernels take as they lie, on either side of where the choice changes."""
    lengths = [per + (g % 3 - 1 if g + 1 < groups else 0) if per > 1 else g % 2 * 2 for g in range(groups)]
    x, w, b, off = make(groups, lengths, n_in, n_out, dtype, lead=1, tail=3)
    y = torch.full((x.shape[0], n_out), 7.0, dtype=dtype, device="cuda")
    check(grouped_linear(x, w, off, b, activation="tanh", scale=0.5, out=y), x, w, off, b, "tanh", 0.5)
    assert (y[:1] == 7).all() and (y[-3:] == 7).all()
