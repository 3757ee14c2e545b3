"""Rows sorted by member and back, against plain indexing and sums in 64 bits.

Tolerances: orders and copies are exact; a product with a weight is rounded to fp32 and then to the type.  combine adds `choices` products in fp32, each addition
off by half a unit of at most S = sum |w y|; a gradient of a weight adds `cols` products, in whatever order, off by cols 2^-24 of S = sum |d y| at worst."""
import math

import pytest
import torch

from paper_2202_05008_b200 import EvoError, combine_rows, combine_rows_backward, grouped_linear, mlp_actions, route_rows, take_rows

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def order(members, groups):
    """(offsets, source, place), by numpy-like loops over the sorted pairs."""
    flat = members.reshape(-1).cpu().tolist()
    lists = [[] for _ in range(groups)]
    for p, m in enumerate(flat):
        if 0 <= m < groups:
            lists[m].append(p)
    source = [p for own in lists for p in own]
    offsets, place = [0], [-1] * len(flat)
    for own in lists:
        offsets.append(offsets[-1] + len(own))
    for at, p in enumerate(source):
        place[p] = at
    return offsets, source + [-1] * (len(flat) - len(source)), place


def check_order(members, groups, routes):
    offsets, source, place = order(members, groups)
    assert routes.offsets.tolist() == offsets and routes.source.tolist() == source and routes.place.reshape(-1).tolist() == place
    assert routes.place.shape == members.shape and all(x.dtype == torch.int32 for x in routes)


# one block (with one to 32 warps), several, two passes; few and many members
@pytest.mark.parametrize("rows,choices", [(1, 1), (31, 1), (33, 2), (1, 700), (1000, 1), (3000, 3), (32768, 1), (32769, 1), (20011, 5), (140000, 3)])
@pytest.mark.parametrize("groups", [1, 2, 31, 500, 1023, 1024, 4096, 8191, 8192, 40000, 1 << 20])
def test_the_order_is_stable_and_complete(rows, choices, groups):
    if rows * choices > 50000 and groups not in (2, 500, 4096, 8192, 1 << 20):
        pytest.skip("the long list is taken with every kernel and not with every size")
    gen = torch.Generator(device="cuda").manual_seed(rows + groups)
    members = torch.randint(-2, groups + 2, (rows, choices), generator=gen, device="cuda")
    members = members.int() if rows % 2 else members
    check_order(members, groups, route_rows(members if choices > 1 else members[:, 0], groups)._replace(place=route_rows(members, groups).place))


@pytest.mark.parametrize("rows", [0, 1, 50, 40000])
@pytest.mark.parametrize("groups", [1, 7, 9000])
def test_lists_of_nobody_and_of_one_member(rows, groups):
    for value in (-1, groups, groups - 1, 0, 2 ** 40, -2 ** 40):
        members = torch.full((rows,), value, dtype=torch.int64, device="cuda")
        routes = route_rows(members, groups)
        live = rows if 0 <= value < groups else 0
        at = torch.arange(rows, device="cuda").int()
        assert routes.offsets.tolist() == [0 if live == 0 or g <= value else rows for g in range(groups + 1)]
        assert torch.equal(routes.place, at if live else torch.full_like(at, -1)) and torch.equal(routes.source, at if live else torch.full_like(at, -1))


def test_members_inside_wider_rows():
    wide = torch.randint(0, 20, (5000, 9), device="cuda", dtype=torch.int32)
    check_order(wide[:, 2:5], 20, route_rows(wide[:, 2:5], 20))
    check_order(wide[:, 3], 20, route_rows(wide[:, 3], 20))
    check_order(wide[::7, :2], 20, route_rows(wide[::7, :2], 20))


def make(rows, choices, cols, dtype, spare=5, dropped=0.2, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed + rows * 7 + cols)
    n = rows * choices
    place = torch.randperm(n + spare, generator=gen, device="cuda")[:n].int().view(rows, choices)
    place[torch.rand(rows, choices, generator=gen, device="cuda") < dropped] = -1
    if n > 3:
        place.view(-1)[n // 2] = n + spare                 # outside: none
    w = torch.randn(rows, choices, generator=gen, device="cuda")
    x = torch.randn(rows, cols, generator=gen, device="cuda").to(dtype)
    y = torch.randn(n + spare, cols, generator=gen, device="cuda").to(dtype)
    return place, w, x, y


def check_all(place, w, x, y, out=None, out_take=None, out_dy=None):
    rows, choices = place.shape
    total, cols = y.shape
    dtype, half = x.dtype, torch.finfo(x.dtype).eps / 2
    live = (place >= 0) & (place < total)
    row, j = torch.nonzero(live, as_tuple=True)
    at = place[row, j].long()
    for weights in (None, w):
        want = torch.full_like(y, 3.0)
        want[at] = x[row] if weights is None else (weights[row, j, None] * x[row].float()).to(dtype)
        got = take_rows(x, place, weights, out=torch.full_like(y, 3.0) if out_take is None else out_take.fill_(3.0))
        assert torch.equal(got, want)
        wd = torch.ones_like(w).double() if weights is None else w.double()
        sums, s = torch.zeros(rows, cols, dtype=torch.float64, device="cuda"), torch.zeros(rows, cols, dtype=torch.float64, device="cuda")
        sums.index_add_(0, row, wd[row, j, None] * y[at].double())
        s.index_add_(0, row, (wd[row, j, None] * y[at].double()).abs())
        got = combine_rows(y, place, weights, out=out)
        err, bound = (got.double() - sums).abs(), choices * 2.0 ** -24 * s * (1 + half) + half * sums.abs() + 1e-45 + (2.0 ** -25 if dtype == F16 else 0)
        assert (err <= bound).all(), float((err / bound).max())
    dy, dw = combine_rows_backward(x, y, place, w, out=torch.full_like(y, 3.0) if out_dy is None else out_dy.fill_(3.0))
    want = torch.full_like(y, 3.0)
    want[at] = (w[row, j, None] * x[row].float()).to(dtype)
    assert torch.equal(dy, want)
    sums, s = torch.zeros_like(w).double(), torch.zeros_like(w).double()
    sums[row, j], s[row, j] = (x[row].double() * y[at].double()).sum(1), (x[row].double() * y[at].double()).abs().sum(1)
    assert ((dw.double() - sums).abs() <= (cols + 1) * 2.0 ** -24 * s).all() and (dw[~live] == 0).all()


@pytest.mark.parametrize("rows,choices,cols", [(1, 1, 1), (1, 1, 4096), (7, 2, 3), (64, 2, 8), (300, 3, 28), (5, 9, 130), (40, 1, 1001), (33, 4, 2048), (3, 17, 513), (700, 8, 64),
                                               (2, 2, 20000), (4000, 1, 5), (9, 5, 255)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_sizes_and_types(rows, choices, cols, dtype):
    check_all(*make(rows, choices, cols, dtype))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [1, 7, 64, 96, 333])
@pytest.mark.parametrize("shift,pitch", [(0, 0), (1, 0), (2, 2), (3, 5), (4, 8), (8, 24)])
def test_strides_and_alignment(dtype, cols, shift, pitch):
    place, w, x, y = make(50, 3, cols, dtype)

    def wider(t, fill=float("nan")):
        room = torch.full((t.shape[0], shift + t.shape[1] + pitch), fill, dtype=t.dtype, device="cuda")
        room[:, shift:shift + t.shape[1]] = t
        return room, room[:, shift:shift + t.shape[1]]
    rooms = [wider(torch.zeros_like(x)), wider(torch.zeros_like(y)), wider(torch.zeros_like(y))]
    check_all(wider(place, -1)[1], wider(w)[1], wider(x)[1], wider(y)[1], *(view for _, view in rooms))
    for room, view in rooms:
        rest = torch.ones_like(room, dtype=torch.bool)
        rest[:, shift:shift + cols] = False
        assert room[rest].isnan().all()


def test_rows_without_a_place_and_no_rows():
    x, y = torch.randn(5, 12, device="cuda"), torch.randn(4, 12, device="cuda")
    none = torch.full((5, 2), -1, dtype=torch.int32, device="cuda")
    w = torch.full((5, 2), float("nan"), device="cuda")
    assert (combine_rows(y.fill_(float("inf")), none, w) == 0).all()
    out = torch.full((4, 12), 2.0, device="cuda")
    assert (take_rows(x, none, w, out=out) == 2).all()
    dy, dw = combine_rows_backward(x, y, none, w, out=out)
    assert (dy == 2).all() and (dw == 0).all()
    assert combine_rows(y, none[:0], w[:0]).shape == (0, 12) and take_rows(x[:0], none[:0]).shape == (0, 12)
    assert (combine_rows(y[:0], none, w) == 0).all()
    one = torch.zeros(5, dtype=torch.int32, device="cuda")
    one[1:] = -1
    assert torch.equal(combine_rows(x[2:], one)[0], x[2])


def test_infinities_go_where_they_belong():
    place = torch.tensor([[0, 1], [2, -1], [3, 4]], dtype=torch.int32, device="cuda")
    w = torch.tensor([[1.0, 0.0], [2.0, float("nan")], [0.5, 0.5]], device="cuda")
    y = torch.ones(5, 9, device="cuda")
    y[1, 3], y[2, 4], y[0, 0] = float("inf"), float("-inf"), float("nan")
    got = combine_rows(y, place, w)
    assert got[0, 3].isnan() and got[0, 0].isnan() and got[1, 4] == float("-inf")
    assert int(got.isfinite().sum()) == 27 - 3


def test_gradients_are_the_differences_of_the_forward():
    place, w, _, y = make(6, 3, 10, F32, dropped=0.3)
    d = torch.randn(6, 10, device="cuda")
    dy, dw = combine_rows_backward(d, y, place, w, out=torch.zeros_like(y))
    step = 2.0 ** -2                                         # (linear in each: the differences are exact but for rounding)

    def f(y, w):
        return float((combine_rows(y, place, w).double() * d.double()).sum())
    base = f(y, w)
    for i, c in ((0, 0), (5, 9), (11, 4), (17, 7)):
        moved = y.clone()
        moved[i, c] += step
        assert abs((f(moved, w) - base) / step - float(dy[i, c])) < 1e-4
    for i, j in ((0, 0), (3, 2), (5, 1)):
        moved = w.clone()
        moved[i, j] += step
        assert abs((f(y, moved) - base) / step - float(dw[i, j])) < 1e-4


def test_actions_of_members_for_observations_in_any_order():
    """route -> take -> the members' policies -> back: every row as its own member would have it."""
    members, sizes, rows = 9, (6, 20, 3), 200
    dim = sum((a + 1) * b for a, b in zip(sizes[:-1], sizes[1:]))
    theta = torch.randn(members, (dim + 3) // 4 * 4, device="cuda") * 0.3
    x, who = torch.randn(rows, 6, device="cuda"), torch.randint(0, members, (rows,), device="cuda")
    routes = route_rows(who, members)
    got = combine_rows(mlp_actions(theta, sizes, take_rows(x, routes.place), routes.offsets), routes.place)
    for m in range(members):
        mine = (who == m).nonzero()[:, 0]
        alone = mlp_actions(theta[m:m + 1], sizes, x[mine], torch.tensor([0, mine.numel()], dtype=torch.int32, device="cuda"))
        assert (got[mine] - alone).abs().max() <= 2e-6      # (another kernel may take other orders of the sums)


def test_refusals():
    x, place, w = torch.zeros(4, 8, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda")
    for call in (lambda: route_rows(place.float(), 3), lambda: route_rows(place, 0), lambda: route_rows(place, (1 << 20) + 1), lambda: route_rows(place.t(), 3),
                 lambda: route_rows(place.cpu(), 3), lambda: route_rows(place[None], 3), lambda: take_rows(x.double(), place), lambda: take_rows(x, place.long()),
                 lambda: take_rows(x[:3], place), lambda: take_rows(x, place, w.half()), lambda: take_rows(x, place, w[:3]), lambda: take_rows(x.t(), place),
                 lambda: take_rows(x, place, out=x), lambda: take_rows(x, place, out=torch.zeros(8, 7, device="cuda")), lambda: combine_rows(x, place, w, out=x),
                 lambda: combine_rows(x, place, w, out=torch.zeros(5, 8, device="cuda")), lambda: combine_rows_backward(x, x, place, None),
                 lambda: combine_rows_backward(x[:3], x, place, w), lambda: combine_rows_backward(x, x, place, w, out=x), lambda: combine_rows(x, place.t(), w)):
        with pytest.raises(EvoError):
            call()
