"""Gradients of the products grouped by member, against the formulas in 64 bits.

Tolerances, relative to S = the sum of the products' sizes: dz is made of y and dy by six roundings of fp32 and counts with 16 bits or more where the operands have 16
(two parts of 8: 2^-17), fp32 operands count with 21 bits or more, and a sum of k products is off by k + 32 units of 2^-24 (an addition in fp32
is off by half a unit of the sum so far, the tensor core cuts off up to a unit of 2^-23 of every 16).  The result is rounded to its type."""
import ctypes as C
import math

import pytest
import torch

from paper_2202_05008_b200 import EvoError, grouped_linear, grouped_linear_backward

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def slack(dtype, k):
    return 6 * 2.0 ** -24 + (2.0 ** -20 if dtype == F32 else 2.0 ** -17) + (k + 32) * 2.0 ** -24


def exact(dy, x, weight, offsets, y, act, scale):
    """((dx, S), (dweight, S), (dbias, S)); rows outside all groups are NaN."""
    dy, x, weight = dy.double(), x.double(), weight.double()
    y = None if y is None else y.double()
    dz = dy * scale if act == "none" else dy * (scale - y * y / scale) if act == "tanh" else dy * scale * (y / scale > 0)
    dx = torch.full_like(x, float("nan"))
    dw, db = torch.zeros_like(weight), torch.zeros(weight.shape[:2], dtype=torch.float64, device=x.device)
    sx, sw, sb = torch.zeros_like(x), torch.zeros_like(dw), torch.zeros_like(db)
    edges = offsets.tolist()
    for g, (p, q) in enumerate(zip(edges[:-1], edges[1:])):
        if q > p:
            d = dz[p:q]
            dx[p:q], sx[p:q] = d @ weight[g], d.abs() @ weight[g].abs()
            dw[g], sw[g] = d.t() @ x[p:q], d.abs().t() @ x[p:q].abs()
            db[g], sb[g] = d.sum(0), d.abs().sum(0)
    return (dx, sx), (dw, sw), (db, sb)


def close(got, want, s, k):
    inside = ~want.isnan()
    half = torch.finfo(got.dtype).eps / 2
    tiny = torch.finfo(got.dtype).smallest_normal * torch.finfo(got.dtype).eps
    off = slack(got.dtype, k) * s
    err, bound = (got.double() - want).abs(), off + half * (want.abs() + off) + tiny
    assert (err[inside] <= bound[inside]).all(), (float((err / bound)[inside].max()), got.shape)


def check(dy, x, weight, offsets, y=None, act="none", scale=1.0, longest=None, **kw):
    dx, dw, db = grouped_linear_backward(dy, x, weight, offsets, y, activation=act, scale=scale, **kw)
    (ex, sx), (ew, sw), (eb, sb) = exact(dy, x, weight, offsets, y, act, scale)
    edges = offsets.tolist()
    longest = max(q - p for p, q in zip(edges[:-1], edges[1:]))
    if dw.shape[0] < ew.shape[0]:
        ew, sw, longest = ew.sum(0, keepdim=True), sw.sum(0, keepdim=True), edges[-1] - edges[0]
    if db.shape[0] < eb.shape[0]:
        eb, sb, longest = eb.sum(0, keepdim=True), sb.sum(0, keepdim=True), edges[-1] - edges[0]
    close(dx, ex, sx, weight.shape[1])
    close(dw, ew, sw, longest)
    close(db, eb, sb, longest)
    return dx, dw, db


def make(groups, lengths, n_in, n_out, dtype, act="none", scale=1.0, seed=0, lead=0, tail=0, wide=False):
    gen = torch.Generator(device="cuda").manual_seed(seed + n_in * 31 + n_out)
    rows = lead + sum(lengths) + tail
    x = torch.randn(rows, n_in, generator=gen, device="cuda").to(dtype)
    w = (torch.randn(groups, n_out, n_in, generator=gen, device="cuda") / math.sqrt(n_in)).to(dtype)
    dy = torch.randn(rows, n_out, generator=gen, device="cuda").to(dtype)
    y = torch.randn(rows, n_out, generator=gen, device="cuda")
    y = (scale * (torch.tanh(y) if act == "tanh" else y.relu())).to(dtype)
    edges = [lead]
    for n in lengths:
        edges.append(edges[-1] + n)
    return dy, x, w, torch.tensor(edges, dtype=torch.int64 if wide else torch.int32, device="cuda"), (None if act == "none" else y)


SHAPES = [
    (1, [1], 1, 1), (3, [1, 0, 2], 5, 3), (4, [0, 0, 0, 7], 16, 16), (2, [8, 9], 17, 33), (5, [3, 40, 0, 1, 33], 28, 128),
    (3, [31, 32, 65], 64, 64), (2, [100, 1], 130, 70), (2, [5, 300], 1000, 90), (1, [17], 2048, 40), (6, [1] * 6, 512, 260),
    (70, [i % 5 for i in range(70)], 24, 40), (3, [129, 257, 40], 264, 264), (2, [513, 16], 72, 512), (1, [3000], 12, 20), (1, [1], 4096, 64), (1, [700], 300, 1),
    (9, [0] * 9, 40, 24), (2, [64, 128], 128, 256),
]


@pytest.mark.parametrize("groups,lengths,n_in,n_out", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_sizes_and_types(groups, lengths, n_in, n_out, dtype):
    for act, scale in (("none", 1.0), ("tanh", 2.5), ("relu", 0.5)):
        dy, x, w, off, y = make(groups, lengths, n_in, n_out, dtype, act, scale, wide=n_in % 2 == 0)
        check(dy, x, w, off, y, act, scale)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n_in,n_out", [(72, 130), (648, 500), (264, 1200), (1500, 1032)])
def test_groups_of_every_part_of_a_tile(n_in, n_out, dtype):
    lengths = [1, 31, 33, 0, 63, 65, 97, 129, 161, 191, 193, 225, 255, 257, 300, 511, 513, 7]
    for act, scale in (("tanh", -0.5), ("none", 3.0)):
        dy, x, w, off, y = make(18, lengths, n_in, n_out, dtype, act, scale, tail=3)
        dx = torch.full((x.shape[0], n_in), 7.0, dtype=dtype, device="cuda")
        check(dy, x, w, off, y, act, scale, out=(dx, None, None))
        assert (dx[-3:] == 7).all()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("groups,lengths,n_in,n_out", [
    (1, [2], 200, 2000), (1, [1], 4097, 129), (2, [9, 0], 36, 700), (3, [30, 0, 47], 26, 300), (4, [3, 2, 0, 5], 300, 1031),    # few blocks: the weight rows are split
    (2, [200, 7], 14, 260), (24, [0] * 23 + [150], 70, 66), (400, [3] * 398 + [90, 0], 50, 61),                               # one group has most of the rows
    (400, [1] * 200 + [0] * 200, 137, 66), (300, [i % 7 for i in range(300)], 138, 200), (60, [1] * 60, 1001, 64),            # rows of weights that start on 2, 4 and 16 bytes
])
def test_few_rows_whatever_the_groups_and_the_alignment(dtype, groups, lengths, n_in, n_out):
    for act, shift in (("none", 0), ("tanh", 1), ("relu", 2)):
        dy, x, w, off, y = make(groups, lengths, n_in, n_out, dtype, act, lead=1, tail=2, seed=shift)
        room = torch.full((groups, n_out * n_in + 8), float("nan"), dtype=dtype, device="cuda")         # (a NaN beside the weights would show)
        weight = room[:, shift:shift + n_out * n_in].unflatten(1, (n_out, n_in))
        weight.copy_(w)
        wide = torch.full((x.shape[0], n_in + 3), 7.0, dtype=dtype, device="cuda")
        check(dy, x, weight, off, y, act, 1.0, out=(wide[:, 1:n_in + 1], None, None))
        assert (wide[0] == 7).all() and (wide[-2:] == 7).all() and (wide[:, 0] == 7).all() and (wide[:, n_in + 1:] == 7).all()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n_in,n_out", [(300, 7), (65, 16), (512, 1), (137, 15), (12, 300), (16, 65), (1, 520), (7, 257)])
@pytest.mark.parametrize("lengths", [[i % 4 for i in range(40)], [0] * 30 + [2], [17, 40, 0, 3], [2000, 5]])
def test_few_outputs_and_few_inputs(dtype, n_in, n_out, lengths):
    for act, scale in (("none", -1.5), ("tanh", 1.0)):
        dy, x, w, off, y = make(len(lengths), lengths, n_in, n_out, dtype, act, scale, lead=3)
        check(dy, x, w, off, y, act, scale)
        _, _, db = grouped_linear_backward(dy, None, w, off, y, activation=act, scale=scale, wanted=(False, False, True))       # (by itself: not a part of dW's kernel)
        edges = off.tolist()
        (_, _), (_, _), (eb, sb) = exact(dy, x, w, off, y, act, scale)
        close(db, eb, sb, max(q - p for p, q in zip(edges[:-1], edges[1:])))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n_in,n_out,shift", [(64, 48, 0), (64, 48, 1), (61, 48, 0), (256, 136, 3), (256, 136, 8)])
@pytest.mark.parametrize("lengths", [[3, 0, 20, 90, 1], [200, 64, 0, 130, 500]])
def test_strides_alignment_and_rows_outside_of_the_groups(dtype, n_in, n_out, shift, lengths):
    dy, x, w, off, y = make(5, lengths, n_in, n_out, dtype, "tanh", 1.0, lead=2, tail=4)

    def wider(t, pitch):
        room = torch.full((t.shape[0], pitch), float("nan"), dtype=t.dtype, device="cuda")
        room[:, shift:shift + t.shape[1]] = t
        return room, room[:, shift:shift + t.shape[1]]
    # a layer of a wider parameter row and its gradient in a row like it, rows inside wider rows
    pitch = shift + n_out * n_in + n_out + 24
    theta = wider(w.flatten(1), pitch)[1].unflatten(1, (n_out, n_in))
    gradient = torch.full((5, pitch), float("nan"), dtype=dtype, device="cuda")
    dw, db = gradient[:, shift:shift + n_out * n_in].unflatten(1, (n_out, n_in)), gradient[:, shift + n_out * n_in:shift + n_out * n_in + n_out]
    room, dx = wider(torch.full_like(x, 7.0), shift + n_in + 5)
    check(wider(dy, shift + n_out + 3)[1], wider(x, shift + n_in + 8)[1], theta, off, wider(y, shift + n_out + 8)[1], "tanh", 1.0, out=(dx, dw, db))
    assert (dx[:2] == 7).all() and (dx[-4:] == 7).all()
    rest = torch.ones_like(room, dtype=torch.bool)
    rest[:, shift:shift + n_in] = False
    assert room[rest].isnan().all() and gradient[:, :shift].isnan().all() and gradient[:, shift + n_out * n_in + n_out:].isnan().all()


@pytest.mark.parametrize("dtype", [F32, F16])
@pytest.mark.parametrize("lengths,n_in,n_out", [([3, 0, 5, 1], 20, 12), ([300, 0, 77, 123], 136, 200), ([2000, 10, 1, 900], 16, 24)])
def test_weights_and_biases_that_groups_share_have_one_gradient(dtype, lengths, n_in, n_out):
    dy, x, w, off, _ = make(4, lengths, n_in, n_out, dtype, lead=3, tail=2)
    shared = w[:1].expand(4, -1, -1)
    for flag in (False, True):
        dx, dw, db = check(dy, x, shared, off, shared_bias=flag)
        assert dw.shape == (1, n_out, n_in) and db.shape == ((1 if flag else 4), n_out)
    dx, dw, db = check(dy, x, w, off, shared_bias=True)
    assert dw.shape == (4, n_out, n_in) and db.shape == (1, n_out)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lengths", [[3, 9, 0], [150, 260, 90]])
def test_each_gradient_by_itself_has_the_bits_it_has_with_the_others(dtype, lengths):
    dy, x, w, off, y = make(3, lengths, 200, 136, dtype, "relu")
    together = grouped_linear_backward(dy, x, w, off, y, activation="relu")
    for i in range(3):
        wanted = tuple(k == i for k in range(3))
        alone = grouped_linear_backward(dy, x if i == 1 else None, w, off, y, activation="relu", wanted=wanted)
        assert [a is not None for a in alone] == list(wanted)
        inside = slice(0, sum(lengths)) if i == 0 else slice(None)
        half = torch.finfo(dtype).eps
        assert (alone[i][inside].double() - together[i][inside].double()).abs().max() <= 2 * half * together[i][inside].double().abs().max()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("lengths,n_in,n_out", [([4, 3, 6], 24, 40), ([130, 70, 100], 136, 264)])
def test_infinities_and_nan_stay_in_their_groups_and_rows(dtype, lengths, n_in, n_out):
    dy, x, w, off, _ = make(3, lengths, n_in, n_out, dtype)
    a, b = lengths[0], lengths[0] + lengths[1]
    x[a - 1, 3], x[b, 5] = float("nan"), float("inf")                       # last row of the first group, first of the third
    dx, dw, db = grouped_linear_backward(dy, x, w, off)
    bad = ~dw.isfinite()
    assert bad[0, :, 3].all() and bad[2, :, 5].all() and int(bad.sum()) == 2 * n_out
    assert dx[:sum(lengths)].isfinite().all() and db.isfinite().all()
    dy, x, w, off, _ = make(3, lengths, n_in, n_out, dtype)
    dy[a - 1, 7], dy[b, 9] = float("inf"), float("nan")
    dx, dw, db = grouped_linear_backward(dy, x, w, off)
    bad = ~dw.isfinite()
    assert bad[0, 7].all() and bad[2, 9].all() and int(bad.sum()) == 2 * n_in
    assert not db[0, 7].isfinite() and not db[2, 9].isfinite() and int((~db.isfinite()).sum()) == 2
    bad = ~dx.isfinite()
    assert bad[a - 1].all() and bad[b].all() and int(bad.sum()) == 2 * n_in


@pytest.mark.parametrize("lengths,n_in,n_out", [([2, 0, 3, 1] * 8, 200, 136), ([22, 5, 31] * 30, 159, 902), ([40, 300, 17], 264, 128)])
def test_fp16_numbers_whose_second_part_has_few_bits(lengths, n_in, n_out):
    """dz / scale is two numbers of fp16: where it is small the second is a multiple of 2^-24, off by half of that at most, whatever dz is.  So a sum of products is off by
    another 2^-25 |scale| times the sum of the other operand's sizes."""
    scale = 2.0
    dy, x, w, off, y = make(len(lengths), lengths, n_in, n_out, F16, "tanh", scale)
    y = (scale * torch.tanh(2.5 * torch.atanh((y / scale).double().clamp(-0.99, 0.99)))).half()         # saturated
    dy = (dy.double() * 2.0 ** -6).half()
    got = grouped_linear_backward(dy, x, w, off, y, activation="tanh", scale=scale)
    for which, (want, s) in enumerate(exact(dy, x, w, off, y, "tanh", scale)):
        ones = torch.ones_like(dy)
        more = exact(ones, x, w, off, None, "none", 1.0)[which][1]       # sums of |weights|, |x|, 1
        k = n_out if which == 0 else max(lengths)
        off_by = slack(F16, k) * s + 2.0 ** -25 * scale * more
        err, bound = (got[which].double() - want).abs(), off_by + 2.0 ** -11 * (want.abs() + off_by) + 2.0 ** -24
        assert (err <= bound).all(), (which, float((err / bound).max()))


def test_offsets_that_fall_or_leave_the_rows_touch_nothing_outside():
    dy, x, w, off, _ = make(4, [40, 30, 20, 10], 72, 40, F32)
    for edges in ([-5, 40, 30, 200, 100], [100, 0, 50, 10, 100], [2 ** 31 - 1] * 5, [-2 ** 31] * 5):
        bad = torch.tensor(edges, dtype=torch.int32, device="cuda")
        room = torch.full((120, 72), 5.0, device="cuda")
        dx, dw, db = grouped_linear_backward(dy, x, w, bad, out=(room[10:110], None, None))
        torch.cuda.synchronize()
        assert (room[:10] == 5).all() and (room[110:] == 5).all()


def test_gradients_are_the_differences_of_the_forward():
    """Central differences of sum(d y) in 64 bits of the forward's formula at the call's inputs, and of the forward's own results."""
    act, scale = "tanh", 1.5
    dy, x, w, off, _ = make(2, [5, 9], 12, 8, F32)
    b = torch.randn(2, 8, device="cuda")
    y = grouped_linear(x, w, off, b, activation=act, scale=scale)
    dx, dw, db = grouped_linear_backward(dy, x, w, off, y, activation=act, scale=scale)

    def f(x, w, b):
        return float((grouped_linear(x, w, off, b, activation=act, scale=scale).double() * dy.double()).sum())
    step = 2.0 ** -6
    # (the third derivative of tanh is at most 2: a central difference is off by step^2 / 3 of the derivative's scale, fp32 rounding of f by 1e-6 / step)
    for which, at in ((0, (3, 5)), (0, (13, 0)), (1, (0, 2, 7)), (1, (1, 7, 11)), (2, (0, 3)), (2, (1, 0))):
        args = [x, w, b]
        ends = []
        for sign in (1.0, -1.0):
            moved = args[which].clone()
            moved[at] += sign * step
            ends.append(f(*[moved if k == which else t for k, t in enumerate(args)]))
        assert abs((ends[0] - ends[1]) / (2 * step) - float((dx, dw, db)[which][at])) < 2e-2


def test_refusals():
    dy, x, w, off, y = make(2, [3, 4], 8, 8, F32, "tanh")
    for call in (lambda: grouped_linear_backward(dy, x, w, off, activation="tanh"), lambda: grouped_linear_backward(dy, x, w, off, y, activation="gelu"),
                 lambda: grouped_linear_backward(dy, x, w, off, y, activation="tanh", scale=0.0), lambda: grouped_linear_backward(dy, None, w, off),
                 lambda: grouped_linear_backward(dy, x.half(), w, off), lambda: grouped_linear_backward(dy[:, :7], x, w, off), lambda: grouped_linear_backward(dy, x[:5], w, off),
                 lambda: grouped_linear_backward(dy, x, w, off[:2]), lambda: grouped_linear_backward(dy, x, w, off.float()), lambda: grouped_linear_backward(dy, x, w.transpose(1, 2)[:, :, ::2], off),
                 lambda: grouped_linear_backward(dy, x, w, off, out=(x, None, None)), lambda: grouped_linear_backward(dy, x, w, off, out=(None, w, None)),
                 lambda: grouped_linear_backward(dy, x, w, off, out=(None, torch.zeros(1, 8, 8, device="cuda"), None)), lambda: grouped_linear_backward(dy.cpu(), x, w, off),
                 lambda: grouped_linear_backward(dy, x, w, off, wanted=(True, True))):
        with pytest.raises(EvoError):
            call()


@pytest.mark.parametrize("dtype,act", [(BF16, "none"), (F16, "tanh"), (F32, "relu")])
@pytest.mark.parametrize("n_in,n_out", [(264, 136), (20, 24), (130, 61)])
def test_groups_of_more_rows_than_one_sum_may_have(dtype, act, n_in, n_out):
    """Numbers of one sign, where what the tensor core cuts off adds up: 20,000 rows in one group, others around it."""
    dy, x, w, off, y = make(3, [700, 20000, 300], n_in, n_out, dtype, act)
    dy, x, w = dy.abs() * 0.05, x.abs(), w.abs()
    check(dy, x, w, off, y, act, 1.0)
    many = 40                                                    # (as many groups as fill the GPU: no split)
    dy, x, w, off, y = make(many, [30] * 20 + [17000] + [50] * (many - 21), 264, 264, dtype, act)
    dy, x, w = dy.abs() * 0.05, x.abs(), w.abs()
    check(dy, x, w, off, y, act, 1.0)


def test_the_same_bits_every_time():
    for dtype, lengths, n_in, n_out in ((F32, [5, 3, 9] * 60, 72, 136), (BF16, [300, 10, 700], 136, 264), (F16, [4000], 40, 30), (F32, [900, 1300], 130, 70)):
        args = make(len(lengths), lengths, n_in, n_out, dtype, "tanh")
        dy, x, w, off, y = args
        first = [t.clone() for t in grouped_linear_backward(dy, x, w, off, y, activation="tanh")]
        for _ in range(5):
            again = grouped_linear_backward(dy, x, w, off, y, activation="tanh")
            assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_a_long_parameter_row_passes_32_bits():
    """Groups 2^27 numbers apart: the last one's weights and gradients lie beyond 2^31 bytes and, with 17 groups, beyond 2^31 numbers."""
    groups, pitch, n_in, n_out = 17, 1 << 27, 24, 40
    room, gradient = torch.empty(groups * pitch, dtype=BF16, device="cuda"), torch.empty(groups * pitch, dtype=BF16, device="cuda")
    theta, g = room.view(groups, pitch), gradient.view(groups, pitch)
    dy, x, w, off, _ = make(groups, [3] * (groups - 1) + [60], n_in, n_out, BF16)
    for at in (theta, g):
        at[:, :n_in * n_out] = w.flatten(1)
    weight, dw = theta[:, :n_in * n_out].unflatten(1, (n_out, n_in)), g[:, :n_in * n_out].unflatten(1, (n_out, n_in))
    check(dy, x, weight, off, out=(None, dw, g[:, n_in * n_out:n_in * n_out + n_out]))
