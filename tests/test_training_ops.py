"""Refusals of the C entry points that a mixture of members is trained with (no GPU needed: every check comes before the first CUDA call, and
the pointers are never used), and of the Python calls."""
import ctypes as C

import pytest
import torch

from paper_2202_05008_b200 import EvoError, build as B, operators
from paper_2202_05008_b200.binding import Grouped, GroupedGradient, PolicyRows, RoutePairs, RowSets, load_library

OK, INVALID, WORKSPACE = 0, 1, 3
FAR = 1 << 40          # addresses far apart: 1 FAR, 2 FAR, ...


@pytest.fixture(scope="module")
def lib():
    B.build_library()
    return load_library()


def _fill(structure, values, changes):
    p = structure()
    p.struct_size = C.sizeof(structure)
    for k, v in {**values, **changes}.items():
        setattr(p, k, v)
    return p


def _routes(**kw):
    return _fill(RoutePairs, dict(groups=10, choices=2, members_64=0, rows=100, d_members=FAR, ld_members=2, d_offsets=2 * FAR, d_source=3 * FAR,
                                  d_place=4 * FAR), kw)


@pytest.mark.parametrize("bad", [dict(struct_size=8), dict(groups=0), dict(groups=(1 << 20) + 1), dict(choices=0), dict(members_64=2), dict(rows=1 << 30),
                                 dict(rows=1 << 41), dict(rows=1 << 63), dict(ld_members=1), dict(d_members=None), dict(d_offsets=None), dict(d_place=None),
                                 dict(d_members=FAR + 2), dict(d_members=FAR + 4, members_64=1), dict(d_offsets=2 * FAR + 2), dict(d_source=3 * FAR + 1),
                                 dict(d_place=4 * FAR + 2), dict(d_place=FAR + 796), dict(d_source=FAR), dict(d_offsets=FAR + 4), dict(d_source=4 * FAR + 400),
                                 dict(d_offsets=3 * FAR + 796), dict(ld_members=1 << 41),
                                 dict(rows=1 << 40, choices=1 << 24, ld_members=1 << 24), dict(rows=1 << 33, choices=1 << 31, ld_members=1 << 32)])
def test_routes_that_are_refused(lib, bad):
    assert lib.evo_route_rows(C.byref(_routes(**bad)), FAR * 9, 1 << 40, None) == INVALID
    assert lib.evo_route_rows(None, FAR * 9, 1 << 40, None) == INVALID


def test_routes_workspace(lib):
    n = C.c_size_t(5)
    assert lib.evo_route_rows_bytes(C.byref(_routes()), C.byref(n)) == OK and n.value == 0
    assert lib.evo_route_rows_bytes(C.byref(_routes(rows=0)), C.byref(n)) == OK and n.value == 0
    assert lib.evo_route_rows_bytes(C.byref(_routes()), None) == INVALID and lib.evo_route_rows_bytes(None, C.byref(n)) == INVALID
    big = _routes(rows=1 << 20)
    assert lib.evo_route_rows_bytes(C.byref(big), C.byref(n)) == OK and n.value > 0
    assert lib.evo_route_rows(C.byref(big), FAR * 9, n.value - 1, None) == WORKSPACE
    assert lib.evo_route_rows(C.byref(big), None, n.value, None) == INVALID and lib.evo_route_rows(C.byref(big), FAR * 9 + 8, n.value, None) == INVALID
    assert lib.evo_route_rows_bytes(C.byref(_routes(groups=1 << 20, rows=(1 << 30) - 1)), C.byref(n)) == OK and n.value >= 2 * 4 * ((1 << 31) - 2)


def _sets(**kw):
    return _fill(RowSets, dict(type=0, choices=2, cols=30, rows=100, sorted_rows=150, d_place=FAR, ld_place=2, d_weights=2 * FAR, ld_weights=2, d_rows=3 * FAR,
                               ld_rows=30, d_sorted=4 * FAR, ld_sorted=32, d_sorted_gradient=5 * FAR, ld_sorted_gradient=31, d_weights_gradient=6 * FAR,
                               ld_weights_gradient=2), kw)


@pytest.mark.parametrize("bad", [dict(struct_size=4), dict(type=3), dict(choices=0), dict(cols=0), dict(cols=(1 << 20) + 1), dict(choices=(1 << 20) + 1),
                                 dict(sorted_rows=1 << 31), dict(rows=1 << 41), dict(ld_place=1), dict(ld_weights=1), dict(ld_rows=29), dict(ld_sorted=29),
                                 dict(d_place=None), dict(d_rows=None), dict(d_sorted=None), dict(d_place=FAR + 1), dict(d_weights=2 * FAR + 2),
                                 dict(d_rows=3 * FAR + 2), dict(d_sorted=4 * FAR + 1),
                                 dict(ld_rows=1 << 41), dict(rows=1 << 40, ld_rows=1 << 40)])
def test_rows_that_are_refused(lib, bad):
    for call in (lib.evo_take_rows, lib.evo_combine_rows, lib.evo_combine_rows_backward):
        assert call(C.byref(_sets(**bad)), None) == INVALID
        assert call(None, None) == INVALID


@pytest.mark.parametrize("bad", [dict(d_rows=4 * FAR + 4 * (149 * 32 + 29)), dict(d_sorted=3 * FAR), dict(d_sorted=3 * FAR - 4 * (149 * 32 + 29))])
def test_rows_that_overlap_are_refused(lib, bad):
    for call in (lib.evo_take_rows, lib.evo_combine_rows):
        assert call(C.byref(_sets(**bad)), None) == INVALID


@pytest.mark.parametrize("bad", [dict(d_sorted_gradient=None), dict(d_weights_gradient=None), dict(d_weights=None), dict(ld_sorted_gradient=29),
                                 dict(ld_weights_gradient=1), dict(d_sorted_gradient=4 * FAR), dict(d_weights_gradient=2 * FAR),
                                 dict(d_sorted_gradient=6 * FAR + 792), dict(d_sorted_gradient=3 * FAR + 4), dict(d_weights_gradient=FAR)])
def test_gradients_of_rows_that_are_refused(lib, bad):
    assert lib.evo_combine_rows_backward(C.byref(_sets(**bad)), None) == INVALID


def test_no_rows_are_no_work(lib):
    empty = _sets(rows=0)
    for call in (lib.evo_take_rows, lib.evo_combine_rows, lib.evo_combine_rows_backward):
        assert call(C.byref(empty), None) == OK
    assert lib.evo_take_rows(C.byref(_sets(sorted_rows=0, d_sorted=None)), None) == OK


def _forward(**kw):
    return _fill(Grouped, dict(type=0, groups=6, n_in=40, n_out=30, activation=1, scale=1.0, offsets_64=0, rows=100, d_x=FAR, ld_x=40, d_weight=2 * FAR, ld_weight=40,
                               weight_stride=1200, d_offsets=3 * FAR, d_y=4 * FAR, ld_y=30), kw)


def _gradient(**kw):
    return _fill(GroupedGradient, dict(sum_weight=0, sum_bias=0, d_dy=5 * FAR, ld_dy=30, d_dx=6 * FAR, ld_dx=40, d_dweight=7 * FAR, ld_dweight=40, dweight_stride=1200,
                                       d_dbias=8 * FAR, dbias_stride=30), kw)


def _backward(lib, f, p, work=FAR * 12, size=1 << 40):
    return lib.evo_grouped_linear_backward(C.byref(f), C.byref(p), work, size, None)


@pytest.mark.parametrize("bad", [dict(struct_size=4), dict(type=3), dict(groups=0), dict(groups=1 << 31), dict(n_in=0), dict(n_out=0), dict(n_in=(1 << 20) + 1),
                                 dict(activation=3), dict(offsets_64=2), dict(rows=1 << 41), dict(scale=float("inf")), dict(scale=0.0), dict(scale=1e-42), dict(ld_x=39), dict(ld_y=29),
                                 dict(ld_weight=39), dict(d_x=None), dict(d_weight=None), dict(d_y=None), dict(d_offsets=None), dict(d_x=FAR + 2),
                                 dict(d_offsets=3 * FAR + 2), dict(d_offsets=3 * FAR + 4, offsets_64=1), dict(ld_x=1 << 41), dict(weight_stride=1 << 41)])
def test_products_whose_gradient_is_refused(lib, bad):
    assert _backward(lib, _forward(**bad), _gradient()) == INVALID


@pytest.mark.parametrize("bad", [dict(struct_size=4), dict(sum_weight=2), dict(sum_bias=2), dict(d_dy=None), dict(ld_dy=29), dict(ld_dx=39), dict(ld_dweight=39),
                                 dict(dweight_stride=1199), dict(dbias_stride=29), dict(d_dx=6 * FAR + 1), dict(d_dx=FAR), dict(d_dx=5 * FAR), dict(d_dx=7 * FAR),
                                 dict(d_dweight=2 * FAR), dict(d_dweight=5 * FAR + 4), dict(d_dbias=3 * FAR), dict(d_dbias=4 * FAR), dict(d_dbias=7 * FAR),
                                 dict(d_dbias=7 * FAR + 4 * 1200, dbias_stride=1230), dict(d_dbias=7 * FAR + 4 * 1200, dbias_stride=1229, dweight_stride=1229),
                                 dict(d_dbias=7 * FAR + 4 * 1199, dbias_stride=1230, dweight_stride=1230), dict(d_dbias=7 * FAR + 4 * 1200, sum_bias=1)])
def test_gradients_of_products_that_are_refused(lib, bad):
    assert _backward(lib, _forward(), _gradient(**bad)) == INVALID
    assert lib.evo_grouped_linear_backward(None, C.byref(_gradient()), FAR * 12, 1 << 40, None) == INVALID
    assert lib.evo_grouped_linear_backward(C.byref(_forward()), None, FAR * 12, 1 << 40, None) == INVALID


def test_gradients_of_products_workspace_and_nothing_wanted(lib):
    n = C.c_size_t()
    assert _backward(lib, _forward(), _gradient(d_dx=None, d_dweight=None, d_dbias=None)) == OK
    big = _forward(groups=1, rows=100000, n_in=60, n_out=60, ld_x=60, ld_y=60, ld_weight=60)
    p = _gradient(ld_dy=60, ld_dx=60, ld_dweight=60)
    assert lib.evo_grouped_linear_backward_bytes(C.byref(big), C.byref(p), C.byref(n)) == OK and n.value > 0
    assert _backward(lib, big, p, size=n.value - 1) == WORKSPACE
    assert _backward(lib, big, p, work=None) == INVALID and _backward(lib, big, p, work=FAR * 12 + 16) == INVALID
    assert lib.evo_grouped_linear_backward_bytes(C.byref(big), C.byref(p), None) == INVALID


def _policy(**kw):
    return _fill(PolicyRows, dict(type=0, actions=12, actions_64=0, rows=100, clip_low=0.2, clip_high=0.2, kl=0.1, d_logits=FAR, ld_logits=12, d_action=2 * FAR,
                                  d_old_logp=3 * FAR, d_advantage=4 * FAR, d_ref_logp=5 * FAR, d_weights=6 * FAR, d_loss=7 * FAR, d_logp=8 * FAR,
                                  d_gradient=9 * FAR, ld_gradient=12), kw)


@pytest.mark.parametrize("bad", [dict(struct_size=4), dict(type=3), dict(actions=0), dict(actions=(1 << 20) + 1), dict(actions_64=2), dict(rows=1 << 41),
                                 dict(clip_low=-0.1), dict(clip_low=1.1), dict(clip_low=float("nan")), dict(clip_high=-1.0), dict(clip_high=float("inf")), dict(kl=-1.0),
                                 dict(kl=float("nan")), dict(d_ref_logp=None), dict(d_logits=None), dict(d_action=None), dict(d_old_logp=None), dict(d_advantage=None),
                                 dict(ld_logits=11), dict(ld_gradient=11), dict(d_logits=FAR + 2), dict(d_action=2 * FAR + 2), dict(d_action=2 * FAR + 4, actions_64=1),
                                 dict(d_weights=6 * FAR + 1), dict(d_loss=7 * FAR + 2), dict(d_logp=8 * FAR + 1), dict(d_gradient=FAR + 48), dict(d_gradient=FAR, ld_gradient=16),
                                 dict(d_gradient=2 * FAR), dict(d_loss=8 * FAR + 4), dict(d_logp=FAR + 4), dict(d_logp=3 * FAR), dict(d_loss=FAR + 44), dict(ld_logits=1 << 41)])
def test_policy_losses_that_are_refused(lib, bad):
    assert lib.evo_policy_loss(C.byref(_policy(**bad)), FAR * 12, 1 << 40, None) == INVALID
    assert lib.evo_policy_loss(None, FAR * 12, 1 << 40, None) == INVALID


def test_policy_loss_workspace(lib):
    n = C.c_size_t()
    assert lib.evo_policy_loss_bytes(C.byref(_policy()), C.byref(n)) == OK and n.value >= 800
    assert lib.evo_policy_loss(C.byref(_policy()), FAR * 12, n.value - 1, None) == WORKSPACE
    assert lib.evo_policy_loss(C.byref(_policy()), None, n.value, None) == INVALID
    assert lib.evo_policy_loss_bytes(C.byref(_policy(d_loss=None)), C.byref(n)) == OK and n.value == 0
    assert lib.evo_policy_loss(C.byref(_policy(d_loss=None, d_logp=None, d_gradient=None)), None, 0, None) == OK


def test_tensors_that_want_a_gradient_are_refused():
    x, place, w = torch.zeros(4, 3), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    off, weight, row = torch.tensor([0, 2, 4]), torch.zeros(2, 3, 3), torch.zeros(4)
    calls = [lambda g: operators.take_rows(g(x), place), lambda g: operators.take_rows(x, place, g(w)), lambda g: operators.combine_rows(g(x), place, w),
             lambda g: operators.combine_rows(x, place, g(w)), lambda g: operators.combine_rows_backward(x, g(x), place, w),
             lambda g: operators.combine_rows_backward(g(x), x, place, w), lambda g: operators.combine_rows_backward(x, x, place, g(w)),
             lambda g: operators.grouped_linear_backward(g(x), x, weight, off), lambda g: operators.grouped_linear_backward(x, g(x), weight, off),
             lambda g: operators.grouped_linear_backward(x, x, g(weight), off), lambda g: operators.grouped_linear_backward(x, x, weight, off, g(x)),
             lambda g: operators.policy_loss(g(x), place[:, 0], row, row), lambda g: operators.policy_loss(x, place[:, 0], row, row, weights=g(row))]
    for call in calls:
        with pytest.raises(EvoError) as e:
            call(lambda t: t.clone().requires_grad_())
        assert e.value.code == 1 and "backward" in str(e.value)
        with torch.no_grad(), pytest.raises(EvoError) as e:         # (these are not on a GPU, which is the next thing that is looked at)
            call(lambda t: t.clone().requires_grad_())
        assert "backward pass" not in str(e.value)


def test_waits_can_be_made_short_in_the_checked_build_alone(lib):
    for bad in ((9, 0), (32, 0), (20, 2)):
        assert lib.evo_debug_grouped_waits(*bad) == INVALID
    assert lib.evo_debug_grouped_waits(20, 1) == 7           # EVO_ERR_UNSUPPORTED
